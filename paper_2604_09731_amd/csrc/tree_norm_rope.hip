// tree_norm_rope: every head of the queries and keys divided by its root mean square, weighted, and rotated by its token's
// position, in one pass from a projection's output to what attention and the cache take.
//
//   y = x / sqrt(mean x^2 + eps) w;   pair i of y turned by position base^(-2 i / rotary_dim)
//
// Bound by memory: each element is read and written once.  A head lies in L lanes of a wavefront, two vectors of V elements a
// lane, which hold the two halves of V pairs, so that a pair is turned where it lies and a head's sum is a few moves between
// neighbours.  A wavefront takes up to kPassesOf times 64 / L heads of one token, all of their loads in flight together.
// The angles of a token are formed once a wavefront, a pair a lane, and handed round through LDS.  An angle is a count of quarter
// turns in binary64 (a binary32 product loses the fast pairs' phase at positions in the tens of thousands); what is left of it behind
// the whole quarters is off by 2^-26 of one in binary32, which sine and cosine in binary32 are taken of.
// 16384 tokens of 32 / 8 heads of 128, bf16: 65 us, 5.2 TB/s, the rate of a copy.  Vectors of 8 bytes and a wavefront for every place
// on the chip, which goes on to further tokens (kWavesPerCu): their registers leave five wavefronts a SIMD.  With vectors of 16 bytes,
// which halve the moves, three: 100 us; two passes in flight 77; a wavefront for every token, which forms the pairs' rates anew, 78 ..
// 156; two passes of 8-byte vectors 82.
#include <math.h>

#include "common.h"

namespace {

constexpr int kWave = 64, kWaves = 4, kThreads = kWave * kWaves;
constexpr int kMaxDim = 128, kMaxPairs = kMaxDim / 2;
// Heads of fewer than 128 (lanes of a head idle) gain from more in flight: bf16, 16384 tokens of 40 heads of 64, 80, 96, 128, four and
// five passes 31.0 / 28.8, 48.2 / 42.2, 53.5 / 51.3, 66 / 66 us; fp32, where five leave four wavefronts a SIMD, 68 / 70, 85 / 91, 99 / 103,
// 131 / 131.
template <typename T> constexpr int kPassesOf = sizeof(T) == 2 ? 5 : 4;
constexpr int kWavesPerCu = 20;

struct NormRopeArgs {
  const void* q;
  const void* k;
  const void* wq;
  const void* wk;
  void* q_out;
  void* k_out;
  const int32_t* position;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
  int32_t n_tokens, Hq, H, D, rot, interleaved;  // H: heads of queries and keys
  int32_t per, chunks;                           // passes over the heads that a wavefront makes of a token, wavefronts a token takes
  float eps;
  double log2_base;
};

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
  T x[V];
};
__device__ inline float wide(float x) { return x; }
__device__ inline float wide(__bf16 x) { return (float)x; }

// Over L neighbouring lanes.
template <int L>
__device__ inline float sum_lanes(float x) {
#pragma unroll
  for (int d = 1; d < L; d *= 2) x += __shfl_xor(x, d);
  return x;
}

template <typename T, int V, int L>
__global__ __launch_bounds__(kThreads) void tree_norm_rope_kernel(NormRopeArgs a) {
  typedef Vec<T, V> Chunk;
  constexpr int kPasses = kPassesOf<T>;
  constexpr int kHeads = kWave / L;
  __shared__ float s_cos[kWaves][kMaxPairs], s_sin[kWaves][kMaxPairs];
  const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int u = lane % L, half = a.rot / 2;
  const bool there = u * 2 * V < a.D, turns = u * 2 * V < a.rot;
  const int first = there ? (turns && !a.interleaved ? u * V : u * 2 * V) : 0;
  const int second = there ? first + (turns && !a.interleaved ? half : V) : V;
  Chunk wq[2], wk[2];  // (as they are in memory: half the registers)
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int d = (j == 0 ? first : second) + i;
      wq[j].x[i] = a.wq ? ((const T*)a.wq)[d] : (T)1.f;
      wk[j].x[i] = a.wk ? ((const T*)a.wk)[d] : (T)1.f;
    }
  // quarter turns a position of pair `lane`
  const double rate = lane < half ? exp2(-(2.0 * (double)lane / (double)a.rot) * a.log2_base) * 0.63661977236758134308 : 0.0;
  const float mean = 1.f / (float)a.D;
  const int64_t items = (int64_t)a.n_tokens * a.chunks;
  for (int64_t item = (int64_t)blockIdx.x * kWaves + wv; item < items; item += (int64_t)gridDim.x * kWaves) {
    const int token = (int)(item / a.chunks), pass0 = (int)(item % a.chunks) * a.per;
    Chunk x[kPasses][2];
    T* to[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int head = (pass0 + p) * kHeads + lane / L;
      const bool on = p < a.per && head < a.H && there;
      const bool is_q = head < a.Hq;
      const T* from = is_q ? (const T*)a.q + token * a.q_stride + (int64_t)head * a.D
                           : (const T*)a.k + token * a.k_stride + (int64_t)(head - a.Hq) * a.D;
      to[p] = !on ? nullptr : (is_q ? (T*)a.q_out + token * a.q_out_stride + (int64_t)head * a.D
                                    : (T*)a.k_out + token * a.k_out_stride + (int64_t)(head - a.Hq) * a.D);
      x[p][0] = on ? *(const Chunk*)(from + first) : Chunk{};
      x[p][1] = on ? *(const Chunk*)(from + second) : Chunk{};
    }
    if (lane < half) {
      const double quarters = (double)a.position[token] * rate, whole = rint(quarters);
      const float rest = (float)(quarters - whole) * 0.5f;
      const int quadrant = (int)(whole - 4.0 * floor(whole * 0.25));
      const float s = sinpif(rest), c = cospif(rest);
      const float sn = quadrant & 1 ? c : s, cs = quadrant & 1 ? s : c;
      s_sin[wv][lane] = quadrant & 2 ? -sn : sn;
      s_cos[wv][lane] = quadrant == 1 || quadrant == 2 ? -cs : cs;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float cs[V], sn[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      cs[i] = turns ? s_cos[wv][u * V + i] : 1.f;
      sn[i] = turns ? s_sin[wv][u * V + i] : 0.f;
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      if (p >= a.per) break;
      const bool is_q = (pass0 + p) * kHeads + lane / L < a.Hq;
      float y[2][V], sum = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          y[j][i] = wide(x[p][j].x[i]);
          sum = fmaf(y[j][i], y[j][i], sum);
        }
      sum = sum_lanes<L>(sum);
      float inv = rsqrtf(fmaf(sum, mean, a.eps));
      if (__any(!(sum < INFINITY))) {  // squares past binary32: again with everything 2^-70 of itself
        float low = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) low = fmaf(y[j][i] * 0x1p-70f, y[j][i] * 0x1p-70f, low);
        low = sum_lanes<L>(low);
        if (!(sum < INFINITY)) {
          inv = rsqrtf(fmaf(low, mean, a.eps * 0x1p-70f * 0x1p-70f));
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) y[j][i] *= 0x1p-70f;
        }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) y[j][i] *= inv * wide(is_q ? wq[j].x[i] : wk[j].x[i]);
      Chunk z[2];
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < V; ++i) {  // pair i: elements 2 i and 2 i + 1 of the two vectors behind one another
          const float even = y[2 * i / V][2 * i % V], odd = y[(2 * i + 1) / V][(2 * i + 1) % V];
          z[2 * i / V].x[2 * i % V] = (T)(turns ? even * cs[i] - odd * sn[i] : even);
          z[(2 * i + 1) / V].x[(2 * i + 1) % V] = (T)(turns ? even * sn[i] + odd * cs[i] : odd);
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          z[0].x[i] = (T)(turns ? y[0][i] * cs[i] - y[1][i] * sn[i] : y[0][i]);
          z[1].x[i] = (T)(turns ? y[0][i] * sn[i] + y[1][i] * cs[i] : y[1][i]);
        }
      }
      if (to[p]) {
        *(Chunk*)(to[p] + first) = z[0];
        *(Chunk*)(to[p] + second) = z[1];
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");  // the angles are read before the next token's are written
    __builtin_amdgcn_wave_barrier();
  }
}

template <typename T, int V, int L>
int32_t launch(NormRopeArgs a, int32_t num_cus, hipStream_t stream) {
  constexpr int kPasses = kPassesOf<T>;
  const int passes = (a.H + kWave / L - 1) / (kWave / L);
  const int64_t waves = (int64_t)(num_cus > 0 ? num_cus : 256) * kWavesPerCu;
  // A wavefront to a pass while that leaves some of the chip's wavefronts over, else as many passes as share their angles.
  a.per = (int64_t)a.n_tokens * passes <= waves / 2 ? 1 : (passes + (passes + kPasses - 1) / kPasses - 1) / ((passes + kPasses - 1) / kPasses);
  a.chunks = (passes + a.per - 1) / a.per;
  const int64_t items = (int64_t)a.n_tokens * a.chunks, groups = ((items < waves ? items : waves) + kWaves - 1) / kWaves;
  hipLaunchKernelGGL((tree_norm_rope_kernel<T, V, L>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}

template <typename T>
int32_t launch_type(const NormRopeArgs& a, bool vectors, int32_t num_cus, hipStream_t stream) {
  if (!vectors) return launch<T, 1, 64>(a, num_cus, stream);
  return a.D <= 64 ? launch<T, 4, 8>(a, num_cus, stream) : launch<T, 4, 16>(a, num_cus, stream);
}

int32_t check(const norm_rope_params& p) {
  if (p.dtype != SMART_F32 && p.dtype != SMART_BF16) return SMART_EINVAL;
  if (p.n_tokens < 0 || p.num_q_heads < 0 || p.num_kv_heads < 0 || (int64_t)p.num_q_heads + p.num_kv_heads < 1) return SMART_EINVAL;
  if ((int64_t)p.num_q_heads + p.num_kv_heads > 65535) return SMART_EINVAL;
  if (p.head_dim < 2 || p.head_dim > kMaxDim || p.head_dim % 2) return SMART_EINVAL;
  if (p.rotary_dim < 2 || p.rotary_dim > p.head_dim || p.rotary_dim % 2) return SMART_EINVAL;
  if (p.pairing != SMART_ROPE_HALF_SPLIT && p.pairing != SMART_ROPE_INTERLEAVED) return SMART_EINVAL;
  if (!(p.base > 0.0) || !(p.base < 1e300) || !(p.eps >= 0x1p-126f) || !(p.eps < 1e30f)) return SMART_EINVAL;
  const int64_t q_row = (int64_t)p.num_q_heads * p.head_dim, k_row = (int64_t)p.num_kv_heads * p.head_dim;
  if (p.q_stride < q_row || p.q_out_stride < q_row || p.k_stride < k_row || p.k_out_stride < k_row) return SMART_EINVAL;
  // (in place: a row where it was)
  if (p.d_q && p.d_q == p.d_q_out && p.q_stride != p.q_out_stride) return SMART_EINVAL;
  if (p.d_k && p.d_k == p.d_k_out && p.k_stride != p.k_out_stride) return SMART_EINVAL;
  if (p.n_tokens == 0) return SMART_OK;
  if (!p.d_position || (p.num_q_heads > 0 && (!p.d_q || !p.d_q_out)) || (p.num_kv_heads > 0 && (!p.d_k || !p.d_k_out))) return SMART_EINVAL;
  const uintptr_t unit = p.dtype == SMART_F32 ? 3 : 1;
  if (((uintptr_t)p.d_q | (uintptr_t)p.d_k | (uintptr_t)p.d_q_out | (uintptr_t)p.d_k_out | (uintptr_t)p.d_q_weight | (uintptr_t)p.d_k_weight) & unit)
    return SMART_EINVAL;
  return SMART_OK;
}

// Whether all heads can be read and written in vectors of n elements (and the pairs' halves lie in whole vectors).
bool vectors_of(const norm_rope_params& p, int64_t n) {
  const uintptr_t bytes = (uintptr_t)n * (p.dtype == SMART_F32 ? 4 : 2) - 1;
  const uintptr_t at = (p.num_q_heads ? (uintptr_t)p.d_q | (uintptr_t)p.d_q_out : 0) | (p.num_kv_heads ? (uintptr_t)p.d_k | (uintptr_t)p.d_k_out : 0);
  const int64_t strides = (p.num_q_heads ? p.q_stride | p.q_out_stride : 0) | (p.num_kv_heads ? p.k_stride | p.k_out_stride : 0);
  return (at & bytes) == 0 && strides % n == 0 && p.head_dim % (2 * n) == 0 && p.rotary_dim % (2 * n) == 0;
}

}  // namespace

extern "C" int32_t tree_norm_rope(smart_ctx* ctx, void* stream, const norm_rope_params* params) {
  if (!ctx || !params) return SMART_EINVAL;
  const norm_rope_params& p = *params;
  int32_t rc = check(p);
  if (rc != SMART_OK || p.n_tokens == 0) return rc;
  NormRopeArgs a;
  a.q = p.d_q;
  a.k = p.d_k;
  a.wq = p.d_q_weight;
  a.wk = p.d_k_weight;
  a.q_out = p.d_q_out;
  a.k_out = p.d_k_out;
  a.position = p.d_position;
  a.q_stride = p.q_stride;
  a.k_stride = p.k_stride;
  a.q_out_stride = p.q_out_stride;
  a.k_out_stride = p.k_out_stride;
  a.n_tokens = p.n_tokens;
  a.Hq = p.num_q_heads;
  a.H = p.num_q_heads + p.num_kv_heads;
  a.D = p.head_dim;
  a.rot = p.rotary_dim;
  a.interleaved = p.pairing == SMART_ROPE_INTERLEAVED;
  a.eps = p.eps;
  a.log2_base = log2(p.base);
  int prev = 0;
  SMART_HIP_CHECK(hipGetDevice(&prev));
  if (prev != ctx->device) SMART_HIP_CHECK(hipSetDevice(ctx->device));
  hipStream_t s = (hipStream_t)stream;
  const int32_t cus = ctx->num_cus;
  if (p.dtype == SMART_F32) rc = launch_type<float>(a, vectors_of(p, 4), cus, s);
  else rc = launch_type<__bf16>(a, vectors_of(p, 4), cus, s);
  if (prev != ctx->device) (void)hipSetDevice(prev);
  return rc;
}
