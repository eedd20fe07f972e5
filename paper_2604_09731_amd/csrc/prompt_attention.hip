// prompt_attention: causal attention of packed prompts, the prefill that lays down what tree_verify_attention streams.
//
// Per (prompt, kv head g) the rows are (token, query head of the group) pairs, rho = token * G + head, so that the heads that
// share keys share the key tiles, and a row tile spans few tokens (few keys behind the diagonal).  A workgroup takes kRows
// consecutive rows, a wavefront 32 R of them, and streams the keys up to its last token past them: one pass with the running
// maximum and sum of a softmax, keys and values staged through LDS.
//   * Scores are kept transposed (keys x rows): a row's softmax stays inside a lane and its partner in the other half of
//     the wavefront, and the probabilities come out in the operand layout of the second product.
//   * Row tiles are handed out from the longest down: what is dispatched last is short.
//   * Bound by the matrix cores: 4 D flops per (row, key).
//   * Values of later tokens are multiplied by probabilities of zero where a tile crosses the diagonal; if that makes a row
//     infinite or NaN the row is evaluated once more, key by key, over its own keys only (walk).
#include <math.h>

#include "common.h"
#include "wave.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short shortx4;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(8))) float floatx8;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) uint32_t uintx4;
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int kWave = 64;
constexpr int kWaves = 4;
constexpr int kThreads = kWave * kWaves;
constexpr int kTile = 32;  // keys and rows of a score tile
constexpr float kLog2e = 1.4426950408889634f;
// The reference of the exponentials follows the running maximum only when that has moved more than 2^kRescaleStep above it.
constexpr float kRescaleStep = 8.f;

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  const int32_t* cu;
  int64_t q_stride, k_stride, v_stride, out_stride;
  int32_t batch, total_tokens, Hq, Hkv, G;
  float scale, c;  // c: in powers of two
};

__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline int wave_sum(int v) {
  int64_t total;
  smart::wave_excl_scan(v, threadIdx.x & (kWave - 1), &total);
  return (int)total;
}

// Key (of 32) that register r of a lane in half h holds.
__device__ inline int key_of(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// ---- which rows a workgroup takes ------------------------------------------------------------------------------------
struct Item {
  int base, len, tile;  // tile < 0: none
};

// Prompts' row tiles: tiles_b = ceil(len_b G / rows).  Up to 64 prompts: level by level from the longest prompt's last tile
// down, so that no long tile is dispatched after short ones.  C(L) = sum_b max(0, tiles_b - L) tiles lie at level L and above.
template <int kRows>
__device__ inline Item find_item(const PromptArgs& a, int rank) {
  const int lane = threadIdx.x & (kWave - 1);
  __shared__ int64_t s_sum[kThreads];
  __shared__ int s_bad;
  __shared__ Item s_item;
  auto length = [&](int b, int* base) {  // -1: no prompt of these offsets
    *base = a.cu[b];
    const int next = a.cu[b + 1];
    return *base < 0 || next < *base || next > a.total_tokens ? -1 : next - *base;
  };
  auto tiles_of = [&](int len) { return (int)(((int64_t)len * a.G + kRows - 1) / kRows); };
  Item it{0, 0, -1};
  if (a.batch <= kWave) {
    int base = 0;
    const int len = lane < a.batch ? length(lane, &base) : 0;
    if (__any(len < 0)) return it;
    const int tiles = tiles_of(len);
    if (wave_sum(tiles) <= rank) return it;
    int lo = 0, hi = tiles;  // C(hi) <= rank < C(lo); the same in all lanes, which take part in the sums together
    for (int o = 32; o > 0; o >>= 1) hi = max(hi, __shfl_xor(hi, o));
    hi = __builtin_amdgcn_readfirstlane(hi);
    int above = 0;  // C(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1, c = wave_sum(max(0, tiles - mid));
      if (c <= rank) hi = mid, above = c;
      else lo = mid;
    }
    const uint64_t there = __ballot(tiles > lo);  // the level's prompts
    int skip = rank - above;
    uint64_t left = there;
    while (skip-- > 0) left &= left - 1;
    if (!left) return it;
    const int b = __ffsll((unsigned long long)left) - 1;
    it.base = __builtin_amdgcn_readlane(base, b);
    it.len = __builtin_amdgcn_readlane(len, b);
    it.tile = lo;
    return it;
  }
  // more prompts: one after the other, each from its last tile down
  const int tid = threadIdx.x, each = (a.batch + kThreads - 1) / kThreads;
  if (tid == 0) s_bad = 0, s_item = it;
  __syncthreads();
  int64_t mine = 0;
  for (int b = tid * each; b < min(a.batch, (tid + 1) * each); ++b) {
    int base;
    const int len = length(b, &base);
    if (len < 0) s_bad = 1;
    else mine += tiles_of(len);
  }
  s_sum[tid] = mine;
  __syncthreads();
  if (s_bad) return it;
  int64_t before = 0;
  for (int i = 0; i < tid; ++i) before += s_sum[i];
  if (rank >= before && rank < before + mine)
    for (int b = tid * each; b < min(a.batch, (tid + 1) * each); ++b) {
      int base;
      const int len = length(b, &base), tiles = tiles_of(len);
      if (rank < before + tiles) {
        s_item = Item{base, len, tiles - 1 - (int)(rank - before)};
        break;
      }
      before += tiles;
    }
  __syncthreads();
  return s_item;
}

// ---- staging: global memory -> registers -> LDS, in 16-byte chunks of rows ----------------------------------------------
// Chunk c of row `key` lies at position c ^ swizzle(key): 16 consecutive rows put the same chunk at 16 positions of a 256-byte
// line (the score product reads a row per lane), and the output product's reads are free of bank conflicts too.
template <typename T, int D>
__device__ inline int swizzle(int key) {
  if (sizeof(T) == 4) return (key & 7) | ((((key >> 2) ^ (key >> 3)) & 1) << 3);
  if (D == 128) return ((key & 7) << 1) | ((key >> 3) & 1);
  return (((key >> 1) & 3) << 1) | ((key >> 3) & 1);
}

template <typename T, int D>
struct Stage {
  static constexpr int kE = 16 / (int)sizeof(T);
  static constexpr int kRowChunks = D / kE;
  static constexpr int kKeys = sizeof(T) == 2 ? 64 : 32;
  static constexpr int kChunks = kKeys * kRowChunks;  // of K, and of V
  static constexpr int kPer = kChunks / kThreads;
  uintx4 k[kPer], v[kPer];

  // Rows past the prompt's end repeat its last one (their scores are masked).
  __device__ void load(const T* kp, const T* vp, const PromptArgs& a, int key0, int len, int tid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = i * kThreads + tid, key = p / kRowChunks, c = (p % kRowChunks) ^ swizzle<T, D>(key);
      const int64_t t = min(key0 + key, len - 1);
      k[i] = *(const uintx4*)(kp + t * a.k_stride + c * kE);
      v[i] = *(const uintx4*)(vp + t * a.v_stride + c * kE);
    }
  }
  __device__ void store(uintx4* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      lds[i * kThreads + tid] = k[i];
      lds[kChunks + i * kThreads + tid] = v[i];
    }
  }
};

// ---- the two products of a wavefront's rows with 32 staged keys ----------------------------------------------------------
template <typename T, int D> struct Products;

template <int D>
struct Products<__bf16, D> {
  typedef bf16x8 Query[D / 16];
  static constexpr int kRowChunks = D / 8;
  __device__ static void load_query(Query& q, const __bf16* row, int h) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) q[ks] = *(const bf16x8*)(row + 16 * ks + 8 * h);
  }
  template <int R>
  __device__ static void scores(floatx16 (&s)[R], const uintx4* kt, const Query (&q)[R], int lane) {
    const int h = lane >> 5, j = lane & 31;
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = (floatx16)(0.f);
    bf16x8 kx[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      kx[ks] = __builtin_bit_cast(bf16x8, kt[j * kRowChunks + ((2 * ks + h) ^ swizzle<__bf16, D>(j))]);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int r = 0; r < R; ++r) s[r] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kx[ks], q[r][ks], s[r], 0, 0, 0);
  }
  // p[r]: the probabilities; rounded[r] becomes the sum of those that enter the product (this lane's).
  template <int R>
  __device__ static void output(floatx16 (&o)[R][D / 32], const uintx4* vt, const floatx16 (&p)[R], float (&rounded)[R], int lane) {
    const int h = lane >> 5, li = lane & 15, jh = (lane >> 4) & 1;
#pragma unroll
    for (int r = 0; r < R; ++r) rounded[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 pb[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        floatx8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p[r][8 * kk + e];
        pb[r] = __builtin_convertvector(x, bf16x8);
        const floatx8 y = __builtin_convertvector(pb[r], floatx8);
        rounded[r] += ((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]));
      }
#pragma unroll
      for (int jt = 0; jt < D / 32; ++jt) {
        // transposing reads: sixteen lanes fetch four rows of sixteen elements, lane i receives column i
        shortx4 part[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int token = 16 * kk + 8 * half + 4 * h + (li >> 2), chunk = 4 * jt + 2 * jh + ((li & 3) >> 1);
          const char* at = (const char*)(vt + token * kRowChunks + (chunk ^ swizzle<__bf16, D>(token))) + 8 * (li & 1);
          part[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)at);
        }
        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int r = 0; r < R; ++r) o[r][jt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pb[r], o[r][jt], 0, 0, 0);
      }
    }
  }
};

template <int D>
struct Products<float, D> {
  typedef floatx4 Query[D / 8];
  static constexpr int kRowChunks = D / 4;
  __device__ static void load_query(Query& q, const float* row, int h) {
#pragma unroll
    for (int s = 0; s < D / 8; ++s) q[s] = *(const floatx4*)(row + 8 * s + 4 * h);
  }
  template <int R>
  __device__ static void scores(floatx16 (&s)[R], const uintx4* kt, const Query (&q)[R], int lane) {
    const int h = lane >> 5, j = lane & 31;
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = (floatx16)(0.f);
#pragma unroll
    for (int x = 0; x < D / 8; ++x) {  // contraction step (x, e): the halves hold head dims 8 x + e and 8 x + 4 + e
      const floatx4 k = __builtin_bit_cast(floatx4, kt[j * kRowChunks + ((2 * x + h) ^ swizzle<float, D>(j))]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], q[r][x][e], s[r], 0, 0, 0);
    }
  }
  template <int R>
  __device__ static void output(floatx16 (&o)[R][D / 32], const uintx4* vt, const floatx16 (&p)[R], float (&rounded)[R], int lane) {
    const int h = lane >> 5, j = lane & 31;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rounded[r] = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) rounded[r] += p[r][i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {  // register i of the halves: two keys
      const int key = key_of(i, h);
#pragma unroll
      for (int jt = 0; jt < D / 32; ++jt) {
        const float v = ((const float*)(vt + key * kRowChunks + ((8 * jt + (j >> 2)) ^ swizzle<float, D>(key))))[j & 3];
#pragma unroll
        for (int r = 0; r < R; ++r) o[r][jt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[r][i], o[r][jt], 0, 0, 0);
      }
    }
  }
};

__device__ inline float widen(float x) { return x; }
__device__ inline float widen(__bf16 x) { return (float)x; }
__device__ inline void store4(float* p, floatx4 x) { *(floatx4*)p = x; }
__device__ inline void store4(__bf16* p, floatx4 x) { *(bf16x4*)p = __builtin_convertvector(x, bf16x4); }

// One row again, key by key, by the whole wavefront: for rows that are hardly ever seen, small and not fast.
template <typename T, int D>
__device__ void walk(const PromptArgs& a, int base, int token, int head, int lane) {
  constexpr int K = D / kWave;
  const int g = head / a.G;
  const T* q = (const T*)a.q + (int64_t)(base + token) * a.q_stride + (int64_t)head * D;
  float x[K], acc[K], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < K; ++i) x[i] = widen(q[lane + i * kWave]), acc[i] = 0.f;
  for (int u = 0; u <= token; ++u) {
    const T* k = (const T*)a.k + (int64_t)(base + u) * a.k_stride + (int64_t)g * D;
    const T* v = (const T*)a.v + (int64_t)(base + u) * a.v_stride + (int64_t)g * D;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) dot += x[i] * widen(k[lane + i * kWave]);
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
    if (dot == -INFINITY) continue;
    const float m_new = fmaxf(m, dot), p = exp2f((dot - m_new) * a.c), al = m_new == m ? 1.f : exp2f((m - m_new) * a.c);
    l = l * al + p;
    m = m_new;
#pragma unroll
    for (int i = 0; i < K; ++i) acc[i] = acc[i] * al + p * widen(v[lane + i * kWave]);
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* out = (T*)a.out + (int64_t)(base + token) * a.out_stride + (int64_t)head * D;
#pragma unroll
  for (int i = 0; i < K; ++i) out[lane + i * kWave] = (T)(acc[i] * inv);
}

template <typename T, int D, int R>
__global__ __launch_bounds__(kThreads, 1) void prompt_attention_kernel(PromptArgs a) {
  constexpr int kRows = kWaves * kTile * R;
  typedef Products<T, D> P;
  typedef Stage<T, D> S;
  __shared__ uintx4 lds[2][2 * S::kChunks];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), h = lane >> 5, j = lane & 31;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  // consecutive workgroups go to different L2s: the row tiles of one kv head sit behind as few of them as possible
  const int g = blockIdx.x % a.Hkv, rank = blockIdx.x / a.Hkv;
  const Item it = find_item<kRows>(a, rank);
  if (it.tile < 0 || it.len <= 0) return;
  const int base = __builtin_amdgcn_readfirstlane(it.base), len = __builtin_amdgcn_readfirstlane(it.len);
  const int rows = len * a.G, row0 = __builtin_amdgcn_readfirstlane(it.tile) * kRows;
  const int mine = row0 + wv * kTile * R;  // this wavefront's first row
  const int keys = (min(row0 + kRows, rows) - 1) / a.G + 1;  // keys of the workgroup
  const int last = (min(mine + kTile * R, rows) - 1) / a.G;  // the last key of the wavefront (with rows)

  typename P::Query q[R];
  floatx16 o[R][D / 32];
  float m[R], l[R], exact[R];
  int token[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int rho = min(mine + kTile * r + j, rows - 1);  // padding rows repeat the last real row; never written
    token[r] = rho / a.G;
    P::load_query(q[r], (const T*)a.q + (int64_t)(base + token[r]) * a.q_stride + (int64_t)(g * a.G + rho % a.G) * D, h);
#pragma unroll
    for (int jt = 0; jt < D / 32; ++jt) o[r][jt] = (floatx16)(0.f);
    m[r] = -INFINITY;
    l[r] = exact[r] = 0.f;
  }
  const T* kp = (const T*)a.k + (int64_t)base * a.k_stride + (int64_t)g * D;
  const T* vp = (const T*)a.v + (int64_t)base * a.v_stride + (int64_t)g * D;
  const int steps = (keys + S::kKeys - 1) / S::kKeys;
  S stage;
  stage.load(kp, vp, a, 0, len, tid);
  for (int t = 0; t < steps; ++t) {
    uintx4* at = lds[t & 1];
    stage.store(at, tid);
    if (t + 1 < steps) stage.load(kp, vp, a, (t + 1) * S::kKeys, len, tid);
    __syncthreads();  // the stage is full, and everyone is done with the other one
    if (mine >= rows) continue;
    for (int x = 0; x < S::kKeys; x += kTile) {
      const int key0 = t * S::kKeys + x;
      if (key0 > last) break;
      floatx16 s[R];
      P::scores(s, at + x * S::kRowChunks, q, lane);
      float rounded[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int first = (min(mine + kTile * r, rows - 1)) / a.G;  // the row tile's first token
        if (key0 + kTile - 1 > first) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (key0 + key_of(i, h) > token[r]) s[r][i] = -INFINITY;
        }
        float mx = s[r][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[r][i]);
        const float m_new = fmaxf(m[r], max_halves(mx));
        if (__any((m_new - m[r]) * a.c > kRescaleStep)) {
          const float alpha = __builtin_amdgcn_exp2f((m[r] - (m_new == -INFINITY ? 0.f : m_new)) * a.c);
          l[r] *= alpha;
          exact[r] *= alpha;
#pragma unroll
          for (int jt = 0; jt < D / 32; ++jt) o[r][jt] *= alpha;
          m[r] = m_new;
        }
        const float mc = m[r] == -INFINITY ? 0.f : m[r] * a.c;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[r][i] = __builtin_amdgcn_exp2f(fmaf(s[r][i], a.c, -mc));
          sum += s[r][i];
        }
        exact[r] += sum;
      }
      P::output(o, at + S::kChunks + x * S::kRowChunks, s, rounded, lane);
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] += rounded[r];
    }
  }
  if (mine >= rows) return;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int rho = mine + kTile * r + j;
    const bool there = rho < rows;
    const float sum = sum_halves(l[r]), inv = sum > 0.f ? 1.f / sum : 0.f;
    const float all = sum_halves(exact[r]);
    const int head = g * a.G + (there ? rho : rows - 1) % a.G;
    float bad = 0.f;
#pragma unroll
    for (int jt = 0; jt < D / 32; ++jt)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        floatx4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = o[r][jt][4 * i4 + i] * inv;
          bad = fmaf(x[i], 0.f, bad);
        }
        if (there) store4((T*)a.out + (int64_t)(base + token[r]) * a.out_stride + (int64_t)head * D + 32 * jt + 8 * i4 + 4 * h, x);
      }
    if (a.lse && there && h == 0) a.lse[(int64_t)(base + token[r]) * a.Hq + head] = all > 0.f ? m[r] * a.scale + logf(all) : -INFINITY;
    // an infinity or NaN that does not come from NaN scores (those stay NaN whichever way they are summed)
    uint64_t again = __ballot(there && bad != 0.f && sum < INFINITY);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    while (again) {
      const int i = __ffsll((unsigned long long)again) - 1;
      again &= again - 1;
      const int row = mine + kTile * r + i;
      walk<T, D>(a, base, row / a.G, g * a.G + row % a.G, lane);
    }
  }
}

template <typename T, int D, int R>
int32_t launch(const PromptArgs& a, hipStream_t stream) {
  constexpr int kRows = kWaves * kTile * R;
  const int64_t tiles = (int64_t)a.total_tokens * a.G / kRows + a.batch;  // sum of ceil(len G / rows) is at most that
  const int64_t grid = tiles * a.Hkv;
  if (grid > 0x7FFFFFFF) return SMART_EINVAL;
  hipLaunchKernelGGL((prompt_attention_kernel<T, D, R>), dim3((unsigned)grid), dim3(kThreads), 0, stream, a);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}

int32_t check(const prompt_params& p) {
  if (p.dtype != SMART_F32 && p.dtype != SMART_BF16) return SMART_EINVAL;
  if (p.batch < 0 || p.total_tokens < 0 || p.num_q_heads <= 0 || p.num_kv_heads <= 0 || p.num_q_heads % p.num_kv_heads != 0)
    return SMART_EINVAL;
  if (p.head_dim != 64 && p.head_dim != 128) return SMART_EINVAL;
  if (!(p.softmax_scale > 0.f) || !(p.softmax_scale < 1e30f)) return SMART_EINVAL;
  if ((int64_t)p.total_tokens * p.num_q_heads > 0x7FFFFFFF) return SMART_EINVAL;
  const int64_t unit = p.dtype == SMART_F32 ? 4 : 8, q_row = (int64_t)p.num_q_heads * p.head_dim, kv_row = (int64_t)p.num_kv_heads * p.head_dim;
  if (p.q_stride < q_row || p.out_stride < q_row || p.k_stride < kv_row || p.v_stride < kv_row) return SMART_EINVAL;
  if (p.q_stride % unit || p.k_stride % unit || p.v_stride % unit || p.out_stride % unit) return SMART_EINVAL;
  if (p.batch == 0 || p.total_tokens == 0) return SMART_OK;
  if (!p.d_q || !p.d_k || !p.d_v || !p.d_cu_tokens || !p.d_out) return SMART_EINVAL;
  if (((uintptr_t)p.d_q | (uintptr_t)p.d_k | (uintptr_t)p.d_v | (uintptr_t)p.d_out) & 15u) return SMART_EINVAL;
  return SMART_OK;
}

}  // namespace

extern "C" int32_t prompt_attention(smart_ctx* ctx, void* stream, const prompt_params* params) {
  if (!ctx || !params) return SMART_EINVAL;
  const prompt_params& p = *params;
  int32_t rc = check(p);
  if (rc != SMART_OK || p.batch == 0 || p.total_tokens == 0) return rc;
  PromptArgs a;
  a.q = p.d_q;
  a.k = p.d_k;
  a.v = p.d_v;
  a.out = p.d_out;
  a.lse = p.d_lse;
  a.cu = p.d_cu_tokens;
  a.q_stride = p.q_stride;
  a.k_stride = p.k_stride;
  a.v_stride = p.v_stride;
  a.out_stride = p.out_stride;
  a.batch = p.batch;
  a.total_tokens = p.total_tokens;
  a.Hq = p.num_q_heads;
  a.Hkv = p.num_kv_heads;
  a.G = p.num_q_heads / p.num_kv_heads;
  a.scale = p.softmax_scale;
  a.c = p.softmax_scale * kLog2e;
  int prev = 0;
  SMART_HIP_CHECK(hipGetDevice(&prev));
  if (prev != ctx->device) SMART_HIP_CHECK(hipSetDevice(ctx->device));
  hipStream_t s = (hipStream_t)stream;
  if (p.dtype == SMART_F32) rc = p.head_dim == 128 ? launch<float, 128, 1>(a, s) : launch<float, 64, 1>(a, s);
  else rc = p.head_dim == 128 ? launch<__bf16, 128, 1>(a, s) : launch<__bf16, 64, 1>(a, s);
  if (prev != ctx->device) (void)hipSetDevice(prev);
  return rc;
}
