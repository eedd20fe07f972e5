// prompt_attention: causal attention of packed prompts, the prefill that lays down what tree_verify_attention streams.
//
// Per (prompt, kv head g) the rows are (token, query head of the group) pairs, rho = token * G + head, so that the heads that
// share keys share the key tiles, and a row tile spans few tokens (few keys behind the diagonal).  A workgroup takes
// consecutive rows, a wavefront 16 or a few times 16 of them, and streams the keys up to its last token past them, 64 at a
// time: one pass with the running maximum and sum of a softmax, keys and values staged through LDS.
//   * Scores are kept transposed (keys x rows): a row's softmax stays inside the four lanes of a column, and the
//     probabilities come out in the operand layout of the second product.
//   * Row tiles are handed out from the longest down, of up to 64 prompts: what is dispatched last is short.
//   * Bound by the matrix cores: 4 D flops per (row, key).
//   * With a window (prompt_attention_window) a row tile streams the first tokens that stay visible and what the windows of its rows
//     hold, as one axis without the gap between them (Span); every variant is compiled for both.  16384 tokens, 64 / 8 heads of 128,
//     window 4096 1.80 ms (1.07 PFLOP/s of what is seen, without a window 1.15); 5 prompts of 300 .. 5000, 32 / 8 heads, window 1024
//     248 us (720 TFLOP/s; the same prompts without 420, 890): 17 stages a row tile, of which the masked ones at both ends and the
//     tile's own beginning and end weigh more; fp32, 8 of 128 .. 1536, 8 / 2 heads of 64, window 200 34 us (61 TFLOP/s): four stages for
//     218 keys, and 825 tiles on 512 places.
//   * Values of later tokens are multiplied by probabilities of zero where a tile crosses the diagonal; a row that comes out
//     infinite or NaN is evaluated once more over its own keys only (evaluate_again).
#include <math.h>

#include "common.h"
#include "wave.h"

namespace {

using smart::add_pair;
using smart::max_quarters;
using smart::sum_quarters;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short shortx4;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(8))) float floatx8;
typedef __attribute__((ext_vector_type(4))) uint32_t uintx4;
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f;
// The reference of the exponentials follows the running maximum only when that has moved more than 2^kRescaleStep above it.
constexpr float kRescaleStep = 8.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNoScore = -3e38f;  // a reference below all scores, and finite: scores of -inf give weights of zero against it

struct PromptArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  const int32_t* cu;
  int64_t q_stride, k_stride, v_stride, out_stride;
  int32_t batch, total_tokens, Hq, Hkv, G;
  int32_t window, sinks;  // 0 in calls without a window; less than total_tokens in all
  uint32_t num_cus;
  float scale, c;  // c: in powers of two
};

// `op` over the 64 lanes, the same in all of them: lanes 1, 2, 4 and 8 apart by data-parallel moves, 16 and 32 apart by swaps.
template <typename Op>
__device__ inline int wave_all(int v, Op op) {
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true));   // quads: 1, 0, 3, 2
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true));   // 2, 3, 0, 1
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true));  // half rows mirrored
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true));  // rows mirrored
  const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = op((int)r[0], (int)r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return __builtin_amdgcn_readfirstlane(op((int)h[0], (int)h[1]));
}
__device__ inline int wave_sum(int v) {
  return wave_all(v, [](int x, int y) { return x + y; });
}

// ---- which rows a workgroup takes ------------------------------------------------------------------------------------
struct Item {
  int base, len, tile;  // tile < 0: none
};

// Prompts' row tiles: tiles_b = ceil(len_b G / rows).  Up to 64 prompts: level by level from the longest prompt's last tile
// down, so that no long tile is dispatched after short ones.  C(L) = sum_b max(0, tiles_b - L) tiles lie at level L and above.
template <int kRows, int kThreads>
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
    hi = wave_all(hi, [](int x, int y) { return max(x, y); });
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
  // More prompts: one after the other, each from its last tile down, and all offsets in every workgroup.  64 prompts of 300 tokens, 32
  // / 8 heads of 128, 160 us, 65 214; 64 of 100 before one of 4000 214, behind it 206; 1000 of 1 .. 8 tokens 19, 20000 2867.
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

// The keys that rows of tokens first .. need, numbered without the gap between the first tokens, which all see, and the first one's
// window: key v is token v, or v + shift from the gap on.  A row of token t, which is key t - shift, sees the keys up to its own
// that are no more than a window behind it or among the first `sinks`.  A stage with keys from both sides of the gap is addressed
// from the prompt's first token; where 32 bits do not reach that far the gap begins with a stage (the keys before it are hidden).
template <bool kWindow>
struct Span {
  int shift = 0, gap = 0, sinks = 0, window = 0;
  __device__ Span(const PromptArgs& a, int first, int len) {
    if (!kWindow) return;
    const int begin = first - a.window + 1;
    const bool reaches = max(a.k_stride, a.v_stride) * len < (int64_t)1 << 30;
    sinks = a.sinks;
    window = a.window;
    const int until = reaches ? sinks : (sinks + 63) & ~63;
    if (begin > until) shift = begin - until, gap = until;
  }
  __device__ int token(int v) const { return kWindow && v >= gap ? v + shift : v; }
  // key: of the row itself
  __device__ bool hidden(int v, int key) const { return v > key || (kWindow && v >= sinks && v <= key - window); }
};

// ---- staging: global memory -> registers -> LDS, in 16-byte chunks of rows ----------------------------------------------
// Chunk c of row `key` lies at position c ^ swizzle(key), so that the reads of both products (a row per lane; four rows of
// sixteen elements per sixteen lanes) are free of bank conflicts.  (Bit 2 of the key takes no part: rows four apart are read by
// the same lanes, at a constant distance.)
template <typename T, int D>
__device__ inline int swizzle(int key) {
  if (sizeof(T) == 4) return (key & 7) | ((((key >> 2) ^ (key >> 3)) & 1) << 3);
  if (D == 128) return ((key & 3) << 1) | ((key >> 3) & 1);
  return (key & 2) | ((key >> 3) & 1);
}

template <typename T, int D, int kThreads>
struct Stage {
  static constexpr int kE = 16 / (int)sizeof(T);
  static constexpr int kRowChunks = D / kE;
  static constexpr int kKeys = 64;
  static constexpr int kChunks = kKeys * kRowChunks;  // of K, and of V
  static constexpr int kPer = kChunks / kThreads;
  uintx4 k[kPer], v[kPer];

  uint32_t ko[kPer], vo[kPer];  // bytes from a stage's first row (check keeps strides below 2^24 elements)

  // The rows of a stage, of which `rows` exist: those past the prompt's end repeat its last one (their scores are masked).
  __device__ void place(const PromptArgs& a, int rows, int tid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = i * kThreads + tid, key = p / kRowChunks, c = (p % kRowChunks) ^ swizzle<T, D>(key), row = min(key, rows - 1);
      ko[i] = ((uint32_t)row * (uint32_t)a.k_stride + c * kE) * (uint32_t)sizeof(T);
      vo[i] = ((uint32_t)row * (uint32_t)a.v_stride + c * kE) * (uint32_t)sizeof(T);
    }
  }
  // The same of a stage with tokens from both sides of a window's gap, from the prompt's first token.
  __device__ void place_both(const PromptArgs& a, const Span<true>& span, int key0, int len, int tid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = i * kThreads + tid, key = p / kRowChunks, c = (p % kRowChunks) ^ swizzle<T, D>(key);
      const int row = min(span.token(key0 + key), len - 1);
      ko[i] = ((uint32_t)row * (uint32_t)a.k_stride + c * kE) * (uint32_t)sizeof(T);
      vo[i] = ((uint32_t)row * (uint32_t)a.v_stride + c * kE) * (uint32_t)sizeof(T);
    }
  }
  // Stages are requested in order; the last one may be short.
  template <bool kWindow>
  __device__ void load(const T* kp, const T* vp, const PromptArgs& a, const Span<kWindow>& span, int key0, int len, int tid) {
    int token0 = key0;
    if constexpr (kWindow) {
      asm volatile("" : "+v"(tid));  // (offsets are derived anew where they change, so that nothing of them lives in registers until there)
      const bool both = key0 < span.gap && key0 + kKeys > span.gap;
      token0 = both ? 0 : span.token(key0);
      if (both) place_both(a, span, key0, len, tid);
      else if (key0 == 0 || key0 - kKeys < span.gap || token0 + kKeys > len) place(a, len - token0, tid);
    } else {
      if (key0 == 0 || key0 + kKeys > len) place(a, len - key0, tid);
    }
    const char *kb = (const char*)(kp + token0 * a.k_stride), *vb = (const char*)(vp + token0 * a.v_stride);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      k[i] = *(const uintx4*)(kb + ko[i]);
      v[i] = *(const uintx4*)(vb + vo[i]);
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

__device__ inline floatx4 four(const float* p) { return *(const floatx4*)p; }
__device__ inline floatx4 four(const __bf16* p) { return __builtin_convertvector(*(const bf16x4*)p, floatx4); }
__device__ inline void put_four(float* p, floatx4 x) { *(floatx4*)p = x; }
__device__ inline void put_four(__bf16* p, floatx4 x) { *(bf16x4*)p = __builtin_convertvector(x, bf16x4); }

// Sixteen rows of a wavefront again, of which those in `which` are written: binary32 products straight from global memory, 16 keys
// a step, weights of at most 1 against the running maximum (the kernels' own may be 2^kRescaleStep, which can take a sum of large
// values past binary32).  A key whose value holds an infinity or NaN is multiplied apart from the others of its step, and only rows in
// which its score is not -infinity take that product.
// Rows that are infinite or NaN by their own keys come here too.  So one bad value of an early token sends every later row of its kv
// head here, and this has to be of the order of the call itself: with an infinity in the first token of all kv heads 3000 tokens of
// 16 / 4 heads take 575 us instead of 73 (bf16, head dim 128), 309 instead of 46 (64), 476 instead of 200 (fp32, 64).
template <typename T, int D, bool kWindow>
__device__ void evaluate_again(const PromptArgs& a, int base, int g, int mine, int rows, uint32_t which, int lane) {
  asm volatile("" : "+v"(lane));  // (everything is derived anew, so that nothing lives in registers until here)
  const int w = lane >> 4, i = lane & 15;
  const int rho = min(mine + i, rows - 1), token = rho / a.G, head = g * a.G + rho % a.G;
  const Span<kWindow> span(a, mine / a.G, rows / a.G);
  const int last = (min(mine + 16, rows) - 1) / a.G - span.shift, own = token - span.shift;
  const T* qp = (const T*)a.q + (int64_t)(base + token) * a.q_stride + (int64_t)head * D + 4 * w;
  const T* kp = (const T*)a.k + (int64_t)base * a.k_stride + (int64_t)g * D + 4 * w;
  const T* vp = (const T*)a.v + (int64_t)base * a.v_stride + (int64_t)g * D + 4 * i;
  floatx4 q[D / 16], o[D / 64][4];  // laid out as in prompt_f32_kernel
#pragma unroll
  for (int x = 0; x < D / 16; ++x) q[x] = four(qp + 16 * x);
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[x][e] = (floatx4)(0.f);
  float m = -INFINITY, l = 0.f;
  for (int key0 = 0; key0 <= last; key0 += 16) {  // (keys behind the last one are that one again, and masked)
    floatx4 v[4][D / 64], s = (floatx4)(0.f);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int x = 0; x < D / 64; ++x) v[r][x] = four(vp + span.token(min(key0 + 4 * w + r, last)) * a.v_stride + 64 * x);
    const T* kr = kp + span.token(min(key0 + i, last)) * a.k_stride;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      const floatx4 k = four(kr + 16 * x);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[x][e], s, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (span.hidden(key0 + 4 * w + r, own)) s[r] = -INFINITY;
    const float now = fmaxf(m, max_quarters(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
    if (__any(now != m)) {
      const float alpha = now == m ? 1.f : exp2f((m - now) * a.c);
      l *= alpha;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] *= alpha;
      m = now;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint64_t counts = __ballot(s[r] != -INFINITY);  // bit 16 u + i: key 4 u + r of the step in row i
      const float p = exp2f((s[r] - (m == -INFINITY ? 0.f : m)) * a.c);
      l += p;
      uint32_t top = 0;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(v[r][x][e]) & 0x7FFFFFFFu);
      for (uint64_t bad = __ballot(top >= 0x7F800000u); bad;) {
        const int u = (__ffsll((unsigned long long)bad) - 1) >> 4;
        bad &= ~(0xFFFFull << (16 * u));
        const bool here = w == u, take = (counts >> (16 * u + i) & 1ull) != 0;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const floatx4 alone = __builtin_amdgcn_mfma_f32_16x16x4f32(here ? v[r][x][e] : 0.f, p, (floatx4)(0.f), 0, 0, 0);
            if (take) o[x][e] += alone;
            v[r][x][e] = here ? 0.f : v[r][x][e];
          }
      }
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][x][e], p, o[x][e], 0, 0, 0);
    }
  }
  const float sum = sum_quarters(l), inv = sum > 0.f ? 1.f / sum : 0.f;
  if ((which >> i & 1u) == 0u) return;
  T* out = (T*)a.out + (int64_t)(base + token) * a.out_stride + (int64_t)head * D + 16 * w;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      floatx4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = o[x][e][r] * inv;
      put_four(out + 64 * x + 4 * r, y);
    }
}

// ---- fp32 -----------------------------------------------------------------------------------------------------------------
// A wavefront's 16 rows against 32 staged keys, in 16 x 16 tiles.  Lane (quarter w, i) of a score tile: row i and keys 4 w + 0 ..
// 3, which are the ones it contributes to the output product, register by register.  Both products contract over what 16-byte
// reads bring: a score's step (x, e) over the head dims 16 x + 4 w + e, and row i of output tile (x, e) is head dim 64 x + 4 i + e.
// Two wavefronts share rows and take the two halves of every stage, so that a compute unit has two on each matrix core even
// where it has one row tile, and a long prompt's last tile, which nothing can follow, takes half as long.  8 / 2 heads of 64:
// 6600 tokens of 8 prompts 103 us (102 TFLOP/s; with 32 x 32 tiles, 128 rows and no sharing 148; 64 rows without sharing 110), one
// prompt of 1536 62 (129, 72), of 300 16.6 (29, 17.7), 4 of 4096 571 (653, 579); head dim 128, 4 of 2048 324 (335, 341).  Left without
// the softmax it takes 6 % less, without staging 8 %; the rest is what the ends of the row tiles leave idle.
template <int D, bool kWindow>
__global__ __launch_bounds__(512, D == 64 ? 4 : 2) void prompt_f32_kernel(PromptArgs a) {
  constexpr int kThreads = 512, kTileRows = 16, kRowWaves = kThreads / kWave / 2, kRows = kRowWaves * kTileRows;
  typedef Stage<float, D, kThreads> S;
  __shared__ uintx4 lds[2][2 * S::kChunks];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = lane >> 4, i16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wv = wave % kRowWaves, part = wave / kRowWaves;
  const int g = blockIdx.x % a.Hkv, rank = blockIdx.x / a.Hkv;
  const Item it = find_item<kRows, kThreads>(a, rank);
  if (it.tile < 0 || it.len <= 0) return;
  const int base = __builtin_amdgcn_readfirstlane(it.base), len = __builtin_amdgcn_readfirstlane(it.len);
  const int rows = len * a.G, row0 = __builtin_amdgcn_readfirstlane(it.tile) * kRows;
  const int mine = row0 + wv * kTileRows;                    // this wavefront's first row
  const Span<kWindow> span(a, row0 / a.G, len);
  const int keys = (min(row0 + kRows, rows) - 1) / a.G + 1 - span.shift;  // keys of the workgroup
  const int last = (min(mine + kTileRows, rows) - 1) / a.G - span.shift;  // the last key of the wavefront (with rows)
  const int first = min(mine, rows - 1) / a.G - span.shift;               // and its first row's own

  const int rho = min(mine + i16, rows - 1);  // padding rows repeat the last real row; never written
  const int token = rho / a.G, head = g * a.G + rho % a.G;
  floatx4 q[D / 16];
#pragma unroll
  for (int x = 0; x < D / 16; ++x)
    q[x] = *(const floatx4*)((const float*)a.q + (int64_t)(base + token) * a.q_stride + (int64_t)head * D + 16 * x + 4 * w);
  floatx4 o[D / 64][4];
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[x][e] = (floatx4)(0.f);
  float m = -INFINITY, l = 0.f;
  const float* kp = (const float*)a.k + (int64_t)base * a.k_stride + (int64_t)g * D;
  const float* vp = (const float*)a.v + (int64_t)base * a.v_stride + (int64_t)g * D;
  const int steps = (keys + S::kKeys - 1) / S::kKeys;
  S stage;
  stage.load(kp, vp, a, span, 0, len, tid);
  for (int t = 0; t < steps; ++t) {
    uintx4* at = lds[t & 1];
    stage.store(at, tid);
    if (t + 1 < steps) stage.load(kp, vp, a, span, (t + 1) * S::kKeys, len, tid);
    __syncthreads();  // the stage is full, and everyone is done with the other one
    const int key0 = t * S::kKeys + 32 * part;
    const uintx4 *kt0 = at + 32 * part * S::kRowChunks, *vt = kt0 + S::kChunks;
    if (mine >= rows || key0 > last) continue;
    if (kWindow && key0 >= span.sinks && key0 + 31 <= first - span.window) continue;
    floatx4 s[2];
    s[0] = s[1] = (floatx4)(0.f);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      floatx4 k[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
        k[kt] = __builtin_bit_cast(floatx4, kt0[(16 * kt + i16) * S::kRowChunks + ((4 * x + w) ^ swizzle<float, D>(16 * kt + i16))]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[kt][e], q[x][e], s[kt], 0, 0, 0);
    }
    if (key0 + 31 > first || (kWindow && key0 + 31 >= span.sinks && key0 <= last - span.window)) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (span.hidden(key0 + 16 * (r >> 2) + 4 * w + (r & 3), token - span.shift)) s[r >> 2][r & 3] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int r = 1; r < 8; ++r) mx = fmaxf(mx, s[r >> 2][r & 3]);
    const float m_new = fmaxf(m, max_quarters(mx));
    if (__any((m_new - m) * a.c > kRescaleStep)) {
      const float alpha = __builtin_amdgcn_exp2f((m - (m_new == -INFINITY ? 0.f : m_new)) * a.c);
      l *= alpha;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] *= alpha;
      m = m_new;
    }
    const float mc = m == -INFINITY ? 0.f : m * a.c;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[r >> 2][r & 3], a.c, -mc));
      s[r >> 2][r & 3] = p;
      l += p;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const int key = 16 * (r >> 2) + 4 * w + (r & 3);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        const floatx4 v = __builtin_bit_cast(floatx4, vt[key * S::kRowChunks + ((16 * x + i16) ^ swizzle<float, D>(key))]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], s[r >> 2][r & 3], o[x][e], 0, 0, 0);
      }
    }
  }
  // The odd halves of the stages join the even ones.
  __syncthreads();
  floatx4* const mo = (floatx4*)lds[0];
  float* const ml = (float*)(mo + D / 16 * kRowWaves * kWave);
  const int at = wv * kWave + lane;
  if (part) {
#pragma unroll
    for (int x = 0; x < D / 16; ++x) mo[x * kRowWaves * kWave + at] = o[x / 4][x % 4];
    ml[at] = m;
    ml[kRowWaves * kWave + at] = l;
  }
  __syncthreads();
  if (part || mine >= rows) return;
  const float m2 = ml[at], top = fmaxf(m, m2);
  const float w1 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.c);
  const float w2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - top) * a.c);
  l = l * w1 + ml[kRowWaves * kWave + at] * w2;
  m = top;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x / 4][x % 4] = o[x / 4][x % 4] * w1 + mo[x * kRowWaves * kWave + at] * w2;
  const bool there = mine + i16 < rows;
  const float sum = sum_quarters(l), inv = sum > 0.f ? 1.f / sum : 0.f;
  float bad = 0.f;
#pragma unroll
  for (int x = 0; x < D / 64; ++x)
#pragma unroll
    for (int r = 0; r < 4; ++r) {  // row 4 w + r of the four tiles
      floatx4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = o[x][e][r] * inv;
        bad = fmaf(y[e], 0.f, bad);
      }
      if (there)
        *(floatx4*)((float*)a.out + (int64_t)(base + token) * a.out_stride + (int64_t)head * D + 64 * x + 16 * w + 4 * r) = y;
    }
  if (a.lse && there && w == 0) a.lse[(int64_t)(base + token) * a.Hq + head] = sum == 0.f ? -INFINITY : m * a.scale + logf(sum);
  uint64_t again = __ballot(there && bad != 0.f && sum < INFINITY);
  again = (again | again >> 16 | again >> 32 | again >> 48) & 0xFFFFull;
  if (again) evaluate_again<float, D, kWindow>(a, base, g, mine, rows, (uint32_t)again, lane);
}

// ---- bf16 -----------------------------------------------------------------------------------------------------------------
__device__ inline float highest(const floatx8& x) {
  return fmaxf(fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(x[3], x[4])), fmaxf(fmaxf(x[5], x[6]), x[7]));
}

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) uintx4 lds_uintx4;

// A wavefront's 16 N rows: products of 16 x 16 tiles, 32 keys at a time.  Lane (quarter w, i): of a score tile, row i and four
// keys; the two score tiles of a step are made of keys 8 w + 0 .. 3 and 8 w + 4 .. 7, so that a lane's eight probabilities are
// the eight consecutive keys that it contributes to the output product.
template <int D, int N, bool kLse, bool kWindow>
struct RowsBf16 {
  bf16x8 q[N][D / 32];
  floatx4 o[N][D / 16];
  float mc[N], l[N], exact[N];  // the reference (in powers of two); the sums of the rounded weights and of the unrounded ones
  int token[N];
  uint32_t ka[D / 32], va[D / 16];  // byte offsets in a stage of this lane's vectors

  __device__ void begin(const PromptArgs& a, int base, int g, int mine, int rows, int lane, int value_offset) {
    const int w = lane >> 4, i = lane & 15;
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const int rho = min(mine + 16 * r + i, rows - 1);  // padding rows repeat the last real row; never written
      token[r] = rho / a.G;
      const __bf16* qp = (const __bf16*)a.q + (int64_t)(base + token[r]) * a.q_stride + (int64_t)(g * a.G + rho % a.G) * D + 8 * w;
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) q[r][ks] = *(const bf16x8*)(qp + 32 * ks);
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) o[r][dt] = (floatx4)(0.f);
      mc[r] = kNoScore;
      l[r] = exact[r] = 0.f;
    }
    const int k_key = 8 * (i >> 2) + (i & 3), v_key = 8 * w + (i >> 2);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) ka[ks] = k_key * (2 * D) + ((4 * ks + w) ^ swizzle<__bf16, D>(k_key)) * 16;
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
      va[dt] = value_offset + v_key * (2 * D) + ((2 * dt + ((i & 3) >> 1)) ^ swizzle<__bf16, D>(v_key)) * 16 + 8 * (i & 1);
  }
  // The operands of the products with keys 32 x .. of the stage at `at`.
  __device__ void read_keys(bf16x8 (&k)[D / 32][2], lds_char* at, int x) const {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int half = 0; half < 2; ++half)
        k[ks][half] = __builtin_bit_cast(bf16x8, *(lds_uintx4*)(at + ka[ks] + (32 * x + 4 * half) * (2 * D)));
  }
  __device__ void read_values(bf16x8 (&v)[D / 16], lds_char* at, int x) const {
    // transposing reads: sixteen lanes fetch four rows of sixteen elements, lane i receives column i
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
      shortx4 four[2];
#pragma unroll
      for (int half = 0; half < 2; ++half)
        four[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(at + va[dt] + (32 * x + 4 * half) * (2 * D)));
      v[dt] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(four[0], four[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
  __device__ void scores(floatx4 (&s)[N][2], const bf16x8 (&k)[D / 32][2]) const {
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int r = 0; r < N; ++r)
          s[r][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[ks][half], q[r][ks], ks == 0 ? (floatx4)(0.f) : s[r][half], 0, 0, 0);
  }
  __device__ void mask(floatx4 (&s)[N][2], const Span<kWindow>& span, int key0, int lane) const {
    if (kWindow) asm volatile("" : "+v"(lane));  // (as in load)
    const int at = key0 + 8 * (lane >> 4);
#pragma unroll
    for (int r = 0; r < N; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e > token[r] - span.shift - at || (kWindow && e >= span.sinks - at && e <= token[r] - span.shift - span.window - at))
          s[r][e >> 2][e & 3] = -INFINITY;
  }
  // Scores -> probabilities as the output product takes them.  The values are requested between the exponentials: a wavefront
  // that asks for all of them at once waits until the LDS has taken the requests of all wavefronts.
  __device__ void softmax(bf16x8 (&pb)[N], const floatx4 (&s)[N][2], float c, bf16x8 (&v)[D / 16], lds_char* at, int part) {
    floatx8 e2[N];
    if (__any(exponents(e2, s, c))) rescale(e2, s, c);
    __builtin_amdgcn_sched_barrier(0);
    read_values(v, at, part);
    weights(pb, e2);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, N + (kLse ? 1 : 0), 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // The reference of the exponentials stays while no score is more than 2^kRescaleStep above it; a lane looks at its own scores only,
  // and where one is (true), the rows' maxima are taken.
  __device__ bool exponents(floatx8 (&e2)[N], const floatx4 (&s)[N][2], float c) const {
    bool move = false;
#pragma unroll
    for (int r = 0; r < N; ++r) {
#pragma unroll
      for (int e = 0; e < 8; ++e) e2[r][e] = fmaf(s[r][e >> 2][e & 3], c, -mc[r]);
      move = move || highest(e2[r]) > kRescaleStep;
    }
    return move;
  }
  __device__ void rescale(floatx8 (&e2)[N], const floatx4 (&s)[N][2], float c) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      floatx8 raw;
#pragma unroll
      for (int e = 0; e < 8; ++e) raw[e] = s[r][e >> 2][e & 3];
      const float now = fmaxf(mc[r], max_quarters(highest(raw)) * c), alpha = __builtin_amdgcn_exp2f(mc[r] - now);
      l[r] *= alpha;
      exact[r] *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) o[r][dt] *= alpha;
      mc[r] = now;
#pragma unroll
      for (int e = 0; e < 8; ++e) e2[r][e] = fmaf(raw[e], c, -now);
    }
  }
  // A weight enters the output product as one bf16.  Three parts would hold its 24 bits, and make four products of the two that a
  // (row, key) takes, where the matrix cores are what bounds the call.  It is off by 2^-8 of itself at most; the sum that divides is
  // that of the rounded weights, so a row is off by 2 2^-8 of its weighted mean |V| at most, about what rounding the result may cost.
  // (Against 64 bits on normal values: root mean square 0.0020 of the output's, 0.0016 of them from rounding the result.)
  __device__ void weights(bf16x8 (&pb)[N], const floatx8 (&e2)[N]) {
#pragma unroll
    for (int r = 0; r < N; ++r) {
      floatx8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(e2[r][e]);
      if (kLse) exact[r] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      pb[r] = __builtin_convertvector(p, bf16x8);
      const uintx4 pairs = __builtin_bit_cast(uintx4, pb[r]);
#pragma unroll
      for (int e = 0; e < 4; ++e) l[r] = add_pair(pairs[e], l[r]);
    }
  }
  // The output product, while the keys 32 x .. of the stage at `at` are fetched.
  __device__ void output(const bf16x8 (&v)[D / 16], const bf16x8 (&pb)[N], bf16x8 (&k)[D / 32][2], lds_char* at, int part) {
    read_keys(k, at, part);
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
      for (int r = 0; r < N; ++r) o[r][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[dt], pb[r], o[r][dt], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, N, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ void finish(const PromptArgs& a, int base, int g, int mine, int rows, int lane) {
    const int w = lane >> 4, i = lane & 15;
    uint64_t all_again = 0;  // (afterwards, when nothing else is held in registers)
#pragma unroll
    for (int r = 0; r < N; ++r) {
      const int rho = mine + 16 * r + i;
      const bool there = rho < rows;
      const float sum = sum_quarters(l[r]), inv = sum > 0.f ? 1.f / sum : 0.f;
      const int head = g * a.G + (there ? rho : rows - 1) % a.G;
      __bf16* out = (__bf16*)a.out + (int64_t)(base + token[r]) * a.out_stride + (int64_t)head * D + 4 * w;
      float bad = 0.f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        const floatx4 x = o[r][dt] * inv;
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = fmaf(x[e], 0.f, bad);
        if (there) *(bf16x4*)(out + 16 * dt) = __builtin_convertvector(x, bf16x4);
      }
      if (kLse) {
        const float all = sum_quarters(exact[r]);
        if (there && w == 0) a.lse[(int64_t)(base + token[r]) * a.Hq + head] = all == 0.f ? -INFINITY : mc[r] * kLn2 + logf(all);
      }
      // an infinity or NaN that does not come from NaN scores (those stay NaN whichever way they are summed)
      uint64_t again = __ballot(there && bad != 0.f && sum < INFINITY);
      again |= again >> 32;
      all_again |= ((again | again >> 16) & 0xFFFFull) << (16 * r);
    }
    for (int r = 0; all_again; ++r, all_again >>= 16)
      if (all_again & 0xFFFFull) evaluate_again<__bf16, D, kWindow>(a, base, g, mine + 16 * r, rows, (uint32_t)(all_again & 0xFFFFull), lane);
  }
};

// A stage is 64 keys, two parts of 32.  Stage t lies in buffer t % 2.  It is written behind the barrier of stage t - 2, when nobody
// reads that one any more, out of registers that were requested a stage earlier, and first read (the keys of its first part)
// behind the barrier of stage t - 1.
template <int D, int kWaves, int N, bool kLse, bool kWindow>
__global__ __launch_bounds__(kWaves* kWave, D == 64 && N == 2 ? 3 : 2) void prompt_bf16_kernel(PromptArgs a) {
  constexpr int kThreads = kWaves * kWave, kMine = 16 * N, kRows = kWaves * kMine;
  typedef Stage<__bf16, D, kThreads> S;
  static_assert(S::kKeys == 64, "two parts a stage");
  __shared__ uintx4 lds[2][2 * S::kChunks];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  // consecutive workgroups go to different L2s: the row tiles of one kv head sit behind as few of them as possible
  uint32_t id = blockIdx.x;
  // Where two workgroups share a compute unit the second one on each is as long as the first is short: 32 / 8 heads, one prompt of
  // 2048 tokens 57.3 us in order, 51.8 so; of 1024 24.5 and 23.0; 8262 tokens of five 165 and 160.
  if (kWaves == 4 && id >= a.num_cus && id < 2 * a.num_cus && 2 * a.num_cus <= gridDim.x) id = 3 * a.num_cus - 1 - id;
  const int g = id % a.Hkv, rank = id / a.Hkv;
  const Item it = find_item<kRows, kThreads>(a, rank);
  if (it.tile < 0 || it.len <= 0) return;
  const int base = __builtin_amdgcn_readfirstlane(it.base), len = __builtin_amdgcn_readfirstlane(it.len);
  const int rows = len * a.G, row0 = __builtin_amdgcn_readfirstlane(it.tile) * kRows;
  const int mine = row0 + wv * kMine;                                       // this wavefront's first row
  const Span<kWindow> span(a, row0 / a.G, len);
  const int keys = (min(row0 + kRows, rows) - 1) / a.G + 1 - span.shift;                 // keys of the workgroup
  const int last = mine < rows ? (min(mine + kMine, rows) - 1) / a.G - span.shift : -1;  // the last key of the wavefront
  const int first = min(mine, rows - 1) / a.G - span.shift;                              // its first row's own
  const int steps = (keys + S::kKeys - 1) / S::kKeys;

  const __bf16* kp = (const __bf16*)a.k + (int64_t)base * a.k_stride + (int64_t)g * D;
  const __bf16* vp = (const __bf16*)a.v + (int64_t)base * a.v_stride + (int64_t)g * D;
  S stage;
  stage.load(kp, vp, a, span, 0, len, tid);
  RowsBf16<D, N, kLse, kWindow> x;
  x.begin(a, base, g, mine, rows, lane, S::kChunks * 16);
  stage.store(lds[0], tid);
  if (steps > 1) {
    stage.load(kp, vp, a, span, S::kKeys, len, tid);
    stage.store(lds[1], tid);
    if (steps > 2) stage.load(kp, vp, a, span, 2 * S::kKeys, len, tid);
  }
  __syncthreads();

  lds_char* at = (lds_char*)lds[0];
  lds_char* other = (lds_char*)lds[1];
  int t = 0;
  auto fill = [&]() {  // behind the barrier of stage t
    if (t + 2 < steps) {
      stage.store(lds[t & 1], tid);
      if (t + 3 < steps) stage.load(kp, vp, a, span, (t + 3) * S::kKeys, len, tid);
    }
  };
  auto next_stage = [&]() {
    lds_char* const was = at;
    at = other;
    other = was;
    ++t;
  };
  bf16x8 k[D / 32][2], v[D / 16], pb[N];
  floatx4 s[N][2];
  x.read_keys(k, at, 0);
  x.scores(s, k);
  // Stages of which some row sees part (with a window also none); wavefronts that are done keep the stages coming.
  auto edge = [&](int until) {
    while (t < until) {
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        const int key0 = t * S::kKeys + 32 * part;
        const bool more = key0 <= last, seen = more && !(kWindow && key0 >= span.sinks && key0 + 31 <= first - span.window);
        if (seen) {
          x.mask(s, span, key0, lane);
          x.softmax(pb, s, a.c, v, at, part);
        }
        if (part == 1) {
          __syncthreads();
          fill();
        }
        if (seen) x.output(v, pb, k, part == 0 ? at : other, 1 - part);
        else if (kWindow && more) x.read_keys(k, part == 0 ? at : other, 1 - part);
        if (more) x.scores(s, k);
      }
      next_stage();
    }
  };
  // Stages that all rows of the wavefront see whole.
  auto inside = [&](int until) {
    while (t < until) {
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        x.softmax(pb, s, a.c, v, at, part);
        if (part == 1) {
          __syncthreads();
          fill();
        }
        __builtin_amdgcn_s_setprio(1);
        x.output(v, pb, k, part == 0 ? at : other, 1 - part);  // (behind the last stage of no use, but there to be read)
        x.scores(s, k);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
      }
      next_stage();
    }
  };
  const int whole = mine < rows ? (first + 1) / S::kKeys : 0;
  if constexpr (kWindow) {
    // Where the windows begin; between the edges; the diagonal and the prompt's end.  (One loop of each kind: a second copy of the
    // edges' takes registers that the loops do not have.)
    for (int pass = 0; pass < 2; ++pass) {
      inside(pass == 1 ? whole : 0);
      edge(pass == 1 ? steps : min(steps, last >= span.window ? (last - span.window) / S::kKeys + 1 : 0));
    }
  } else {
    inside(whole);
    edge(steps);  // the diagonal and the prompt's end
  }
  if (mine < rows) x.finish(a, base, g, mine, rows, lane);
}

// Row tiles of the given height that any offsets can make: sum of ceil(len G / rows) is at most that.
int64_t most_tiles(const PromptArgs& a, int rows) { return (int64_t)a.total_tokens * a.G / rows + a.batch; }

template <typename Kernel>
int32_t launch(Kernel kernel, int threads, int rows, const PromptArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(kernel, dim3((unsigned)(most_tiles(a, rows) * a.Hkv)), dim3(threads), 0, stream, a);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}

template <int D, int kWaves, int N, bool kWindow>
int32_t launch_rows(const PromptArgs& a, hipStream_t stream) {
  return a.lse ? launch(prompt_bf16_kernel<D, kWaves, N, true, kWindow>, kWaves * kWave, kWaves * 16 * N, a, stream)
               : launch(prompt_bf16_kernel<D, kWaves, N, false, kWindow>, kWaves * kWave, kWaves * 16 * N, a, stream);
}

// Taller row tiles read the LDS less often per product, but there have to be enough of them to fill the chip and to let the short
// ones fill in behind the long.  us with tiles of 64 / 128 / 256 rows (four wavefronts; 256 rows of head dim 128 eight), 32 / 8
// heads: one prompt of 37 tokens 5.2 / 6.6 / 7.9, of 512 13.2 / 17.8 / 22.3, of 1500 36.2 / 43.5 / 47.0, of 2048 57.1 / 52.7 / 61.3, of
// 4096 194 / 140 / 133; 12 of 341 .. 1024 92.6 / 70.7 / 73.5; 8262 tokens of five 223 / 166 / 165; 16384 tokens, 64 heads 5647 / 3987 /
// 3690; head dim 64, 8 heads, one of 4096 34.6 / 46.1 / 74.0, 64 of 1 .. 300 14.7 / 11.7 / 14.9, 4 of 1024 .. 2048 26.4 / 34.3 / 52.4;
// 32 heads, 4 of 4096 383 / 309 / 289.  (Two teams of wavefronts on one row tile, with half of the keys each, are ahead for a few
// prompts of few heads only: one of 4096, 8 heads of 64, 27 for 35 us; one of 2048, 32 heads of 128, 51; 8262 tokens 212.)
// With a window a tile of more tokens than a sixth of it (of 256 rows: than a 64th) streams too many keys that few of its rows see, and
// nothing is longest: 64 rows for longer.  One prompt of 8192 tokens, 32 / 8 heads of 128, windows of 100, 500 and 2000, tiles of 64 / 128
// / 256 rows: 43 / 51 / 61, 85 / 80 / 91, 187 / 141 / 149; 64 / 8 heads 82 / 76 / 99, 149 / 133 / 152, 362 / 273 / 270; 16384 tokens, window
// 4096 2660 / 1947 / 1800; 8 / 8 heads of 64 11 / 18 / 31, 19 / 26 / 51, 37 / 47 / 88; 2048 tokens, 32 / 8 heads of 128, window 2000 26 /
// 34 / 39.
int tile_rows(const PromptArgs& a, bool f32) {
  const int64_t rows = (int64_t)a.total_tokens * a.Hq, cus = a.num_cus;
  if (a.window > 0 && !f32) {
    const int64_t reach = (int64_t)a.window * a.G;
    return rows <= 256 * cus || reach < 6 * 128 ? 64 : (rows < 4 * 256 * cus || reach < 64 * 256 ? 128 : 256);
  }
  return f32 || rows <= 192 * cus ? 64 : (rows < 4 * 256 * cus ? 128 : 256);
}
int tile_threads(int rows, bool f32, int D) { return f32 || (rows == 256 && D == 128) ? 512 : 256; }

template <int D, bool kWindow>
int32_t launch_bf16(const PromptArgs& a, int rows, hipStream_t stream) {
  if (rows == 64) return launch_rows<D, 4, 1, kWindow>(a, stream);
  if (rows == 128) return launch_rows<D, 4, 2, kWindow>(a, stream);
  return launch_rows<D, D == 128 ? 8 : 4, D == 128 ? 2 : 4, kWindow>(a, stream);
}

template <bool kWindow>
int32_t launch_any(const PromptArgs& a, bool f32, int D, int rows, int threads, hipStream_t stream) {
  if (f32)
    return D == 128 ? launch(prompt_f32_kernel<128, kWindow>, threads, rows, a, stream) : launch(prompt_f32_kernel<64, kWindow>, threads, rows, a, stream);
  return D == 128 ? launch_bf16<128, kWindow>(a, rows, stream) : launch_bf16<64, kWindow>(a, rows, stream);
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
  // (rows of a stage, 64 of them, are addressed in 32 bits)
  if (p.k_stride >= (1 << 24) || p.v_stride >= (1 << 24)) return SMART_EINVAL;
  if (p.q_stride % unit || p.k_stride % unit || p.v_stride % unit || p.out_stride % unit) return SMART_EINVAL;
  if (p.batch == 0 || p.total_tokens == 0) return SMART_OK;
  if (!p.d_q || !p.d_k || !p.d_v || !p.d_cu_tokens || !p.d_out) return SMART_EINVAL;
  if (((uintptr_t)p.d_q | (uintptr_t)p.d_k | (uintptr_t)p.d_v | (uintptr_t)p.d_out) & 15u) return SMART_EINVAL;
  return SMART_OK;
}

// window 0: none
int32_t prompt(smart_ctx* ctx, void* stream, const prompt_params& p, int32_t window, int32_t sinks) {
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
  // (the last token of the longest prompt there can be sees the first `sinks` and the last `window`: with all of them nothing is hidden)
  const bool hides = window > 0 && (int64_t)window + sinks < p.total_tokens;
  a.window = hides ? window : 0;
  a.sinks = hides ? sinks : 0;
  a.num_cus = ctx->num_cus > 0 ? ctx->num_cus : 256;
  a.scale = p.softmax_scale;
  a.c = p.softmax_scale * kLog2e;
  const bool f32 = p.dtype == SMART_F32;
  const int rows = tile_rows(a, f32), threads = tile_threads(rows, f32, p.head_dim);
  if (most_tiles(a, rows) * a.Hkv > 0xFFFFFFFFll / threads) return SMART_EINVAL;  // (a grid's threads are counted in 32 bits)
  int prev = 0;
  SMART_HIP_CHECK(hipGetDevice(&prev));
  if (prev != ctx->device) SMART_HIP_CHECK(hipSetDevice(ctx->device));
  hipStream_t s = (hipStream_t)stream;
  rc = hides ? launch_any<true>(a, f32, p.head_dim, rows, threads, s) : launch_any<false>(a, f32, p.head_dim, rows, threads, s);
  if (prev != ctx->device) (void)hipSetDevice(prev);
  return rc;
}

}  // namespace

extern "C" int32_t prompt_attention(smart_ctx* ctx, void* stream, const prompt_params* params) {
  if (!ctx || !params) return SMART_EINVAL;
  return prompt(ctx, stream, *params, 0, 0);
}

extern "C" int32_t prompt_attention_window(smart_ctx* ctx, void* stream, const prompt_params* params, int32_t window, int32_t sinks) {
  if (!ctx || !params || window < 1 || sinks < 0) return SMART_EINVAL;
  return prompt(ctx, stream, *params, window, sinks);
}
