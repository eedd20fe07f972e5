// The 4-bit cache: kv_cache_write_fp4, kv_cache_read_fp4, tree_commit_fp4.
//
// Elements move in eights: a lane holds 8 head dims of a token and kv head (16 bytes of bf16, 4 bytes of codes), and the four
// lanes of a quad the 32 that share a scale; they agree on the largest absolute value by two exchanges.  fp4.h has the format
// and the rounding.
#include "common.h"
#include "fp4.h"
#include "tree_commit.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnit = 32;                // elements that share a scale
constexpr int kEight = 8;                // elements of a lane
constexpr int kTokens = 8;               // tokens of a wavefront, 8 lanes each
constexpr int kDims = 64 / kTokens * kEight;  // and elements that it takes of each

struct Eight {
  float x[kEight];
};

__device__ inline void load_eight(Eight& u, const float* p) {
#pragma unroll
  for (int i = 0; i < kEight / 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(p)[i];
    u.x[4 * i] = v.x, u.x[4 * i + 1] = v.y, u.x[4 * i + 2] = v.z, u.x[4 * i + 3] = v.w;
  }
}
__device__ inline void load_eight(Eight& u, const uint16_t* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u.x[2 * j] = __uint_as_float(w[j] << 16);
    u.x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
}
__device__ inline void store_eight(const Eight& u, float* p) {
#pragma unroll
  for (int i = 0; i < kEight / 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(u.x[4 * i], u.x[4 * i + 1], u.x[4 * i + 2], u.x[4 * i + 3]);
}
__device__ inline void store_eight(const Eight& u, uint16_t* p) {  // exact: the values have two significant bits
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(u.x[2 * j]) >> 16 | (__float_as_uint(u.x[2 * j + 1]) & 0xFFFF0000u);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

template <int kPattern>
__device__ inline uint32_t quad_max(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kPattern, 0xF, 0xF, true));
}

struct Codes {
  uint32_t w, scale;
};
// All four lanes of a quad take part.
__device__ inline Codes encode(const Eight& u) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kEight; ++i) top = max(top, __float_as_uint(u.x[i]) & 0x7FFFFFFFu);
  top = quad_max<0xB1>(top);  // lanes 1, 0, 3, 2
  top = quad_max<0x4E>(top);  // lanes 2, 3, 0, 1
  Codes c;
  c.scale = smart::fp4_scale_byte(top);
  c.w = c.scale == 255u ? 0u : smart::fp4_codes8(u.x, smart::fp4_scale(c.scale));
  return c;
}
__device__ inline void decode(Eight& u, const Codes& c) {
  const float s = smart::fp4_scale(c.scale);
  const smart::fp4_floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, s, 0);
  const smart::fp4_floatx2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, s, 1);
  const smart::fp4_floatx2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, s, 2);
  const smart::fp4_floatx2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w, s, 3);
  u.x[0] = a[0], u.x[1] = a[1], u.x[2] = b[0], u.x[3] = b[1];
  u.x[4] = d[0], u.x[5] = d[1], u.x[6] = e[0], u.x[7] = e[1];
}

// Pages of a cache: K and V lie alike.
struct Pages {
  int Hkv, D, block_size, num_blocks;
  int64_t block_stride, head_stride;  // bytes
};

// Where the 8 elements e .. e + 7 of a slot's Hkv x D lie: the page's offset in the cache, and the head dim.
struct Place {
  int64_t page;
  int d;
};
__device__ inline Place place(const Pages& pg, int64_t block, int e) {
  const int g = (int)((uint32_t)e / (uint32_t)pg.D);
  return Place{block * pg.block_stride + g * pg.head_stride, e - g * pg.D};
}
// The block and slot of a slot id; false for one that names no slot.
__device__ inline bool find_slot(const Pages& pg, int64_t id, int64_t* block, int* slot) {
  if (id < 0 || id >= (int64_t)pg.num_blocks * pg.block_size) return false;
  *block = id >> 32 ? id / pg.block_size : (int64_t)((uint32_t)id / (uint32_t)pg.block_size);
  *slot = (int)(id - *block * pg.block_size);
  return true;
}

// One lane of a quad writes the scale.
__device__ inline void put_k(uint8_t* page, int bs, int D, int slot, int d, const Codes& c) {
  *reinterpret_cast<uint32_t*>(page + smart::fp4_k_code(bs, slot, d)) = c.w;
  if ((d & (kUnit - 1)) == 0) page[smart::fp4_k_scale(bs, D, slot, d)] = (uint8_t)c.scale;
}
__device__ inline void put_v(uint8_t* page, int bs, int D, int slot, int d, const Codes& c) {
  *reinterpret_cast<uint16_t*>(page + smart::fp4_v_code(D, slot, d)) = (uint16_t)c.w;
  *reinterpret_cast<uint16_t*>(page + smart::fp4_v_code(D, slot, d + 4)) = (uint16_t)(c.w >> 16);
  if ((d & (kUnit - 1)) == 0) page[smart::fp4_v_scale(bs, D, slot, d)] = (uint8_t)c.scale;
}
__device__ inline Codes get_k(const uint8_t* page, int bs, int D, int slot, int d) {
  return Codes{*reinterpret_cast<const uint32_t*>(page + smart::fp4_k_code(bs, slot, d)), page[smart::fp4_k_scale(bs, D, slot, d)]};
}
__device__ inline Codes get_v(const uint8_t* page, int bs, int D, int slot, int d) {
  const uint32_t lo = *reinterpret_cast<const uint16_t*>(page + smart::fp4_v_code(D, slot, d));
  const uint32_t hi = *reinterpret_cast<const uint16_t*>(page + smart::fp4_v_code(D, slot, d + 4));
  return Codes{lo | hi << 16, page[smart::fp4_v_scale(bs, D, slot, d)]};
}

// Both directions: a wavefront takes 64 elements of K and of V of 8 tokens.  Eight lanes read or write 128 bytes of a row of
// bf16; a page's V vector, 8 consecutive tokens by 4 head dims, is written by 8 lanes of one store.  Bytes bound both: 8190 tokens
// of 8 heads of 128, 42 MB each, 10.6 and 10.0 us (one thread a unit, with 64 bytes
// between the lanes: 12.7 and 16.4); fp32, 76 MB, 29.2 together (42.5).  Two or four times as much a wavefront is no faster.
template <typename T>
__global__ __launch_bounds__(kThreads) void kv_cache_write_fp4_kernel(Pages pg, int n_tokens, const T* __restrict__ k_src,
                                                                      const T* __restrict__ v_src,
                                                                      const int64_t* __restrict__ slot_mapping,
                                                                      uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, row = pg.Hkv * pg.D;
  const int64_t t = (int64_t)blockIdx.x * kTokens + (lane >> 3);
  const int e = ((int)blockIdx.y * kWaves + wv) * kDims + (lane & 7) * kEight;
  if (t >= n_tokens || e >= row) return;
  const int64_t id = slot_mapping[t];
  Eight k, v;
  load_eight(k, k_src + t * row + e);
  load_eight(v, v_src + t * row + e);
  int64_t block;
  int slot;
  if (!find_slot(pg, id, &block, &slot)) return;
  const Place p = place(pg, block, e);
  put_k(k_cache + p.page, pg.block_size, pg.D, slot, p.d, encode(k));
  put_v(v_cache + p.page, pg.block_size, pg.D, slot, p.d, encode(v));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_cache_read_fp4_kernel(Pages pg, int n_tokens, const uint8_t* __restrict__ k_cache,
                                                                     const uint8_t* __restrict__ v_cache,
                                                                     const int64_t* __restrict__ slot_mapping, T* __restrict__ k_dst,
                                                                     T* __restrict__ v_dst) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, row = pg.Hkv * pg.D;
  const int64_t t = (int64_t)blockIdx.x * kTokens + (lane >> 3);
  const int e = ((int)blockIdx.y * kWaves + wv) * kDims + (lane & 7) * kEight;
  if (t >= n_tokens || e >= row) return;
  int64_t block;
  int slot;
  Codes k{0u, 127u}, v = k;  // no slot: zeros
  if (find_slot(pg, slot_mapping[t], &block, &slot)) {
    const Place p = place(pg, block, e);
    k = get_k(k_cache + p.page, pg.block_size, pg.D, slot, p.d);
    v = get_v(v_cache + p.page, pg.block_size, pg.D, slot, p.d);
  }
  Eight x;
  decode(x, k);
  store_eight(x, k_dst + t * row + e);
  decode(x, v);
  store_eight(x, v_dst + t * row + e);
}

// One workgroup per (path index i, sequence b); workgroup i = 0 reports the sequence's verdict (commit_row).
template <typename T>
__global__ __launch_bounds__(kThreads) void tree_commit_fp4_kernel(Pages pg, smart::CommitInputs in, const T* __restrict__ k_tree,
                                                                   const T* __restrict__ v_tree, uint8_t* __restrict__ k_cache,
                                                                   uint8_t* __restrict__ v_cache,
                                                                   int32_t* __restrict__ new_prefix_len,
                                                                   int32_t* __restrict__ status) {
  const int i = blockIdx.x, b = blockIdx.y;
  const int base = in.cu_nodes[b];
  const smart::CommitRow r = smart::commit_row(in, i, b, base, in.cu_nodes[b + 1] - base, threadIdx.x & 63);
  if (i == 0 && threadIdx.x == 0) {
    status[b] = r.verdict;
    new_prefix_len[b] = r.verdict == SMART_OK ? r.start + r.accepted + 1 : r.start;
  }
  if (r.verdict != SMART_OK || i > r.accepted) return;
  const int slot = (r.start + i) % pg.block_size, row = pg.Hkv * pg.D;
  const int64_t src = ((int64_t)base + r.node) * row;
  for (int u = threadIdx.x * kEight; u < 2 * row; u += kThreads * kEight) {
    const bool values = u >= row;
    const int e = values ? u - row : u;
    Eight x;
    load_eight(x, (values ? v_tree : k_tree) + src + e);
    const Codes c = encode(x);
    const Place p = place(pg, r.block, e);
    if (values) put_v(v_cache + p.page, pg.block_size, pg.D, slot, p.d, c);
    else put_k(k_cache + p.page, pg.block_size, pg.D, slot, p.d, c);
  }
}

// The grid of a copy of n_tokens rows; false if there is none.
bool copy_grid(int32_t n_tokens, int32_t num_kv_heads, int32_t head_dim, dim3* grid) {
  const int64_t x = ((int64_t)n_tokens + kTokens - 1) / kTokens, piece = kWaves * kDims;
  const int64_t y = ((int64_t)num_kv_heads * head_dim + piece - 1) / piece;
  if (y > 65535 || x * kThreads > 0xFFFFFFFFll) return false;  // (a grid's threads are counted in 32 bits)
  *grid = dim3((unsigned)x, (unsigned)y);
  return true;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The arguments that all three calls share.
bool pages_ok(int32_t dtype, int32_t num_kv_heads, int32_t head_dim, int32_t block_size, int32_t num_blocks, const void* k_cache,
              const void* v_cache, int64_t block_stride, int64_t head_stride) {
  if (dtype != SMART_F32 && dtype != SMART_BF16) return false;
  // (offsets inside a page and the elements of a row are counted in 32 bits)
  if (num_kv_heads <= 0 || head_dim <= 0 || block_size <= 0 || num_blocks < 0 || (int64_t)head_dim * block_size >= (1 << 30) ||
      (int64_t)num_kv_heads * head_dim >= (1 << 26))
    return false;
  return smart::fp4_cache_ok(block_size, head_dim, k_cache, v_cache, block_stride, head_stride);
}

}  // namespace

extern "C" int32_t kv_cache_write_fp4(smart_ctx* ctx, void* stream, int32_t src_dtype, int32_t n_tokens, int32_t num_kv_heads,
                                      int32_t head_dim, int32_t block_size, int32_t num_blocks, const void* d_k_src,
                                      const void* d_v_src, const int64_t* d_slot_mapping, void* d_k_cache, void* d_v_cache,
                                      int64_t cache_block_stride, int64_t cache_head_stride) {
  if (!ctx || n_tokens < 0 || !pages_ok(src_dtype, num_kv_heads, head_dim, block_size, num_blocks, d_k_cache, d_v_cache,
                                        cache_block_stride, cache_head_stride))
    return SMART_EINVAL;
  if (n_tokens == 0) return SMART_OK;
  if (!d_k_src || !d_v_src || !d_slot_mapping || !d_k_cache || !d_v_cache || !aligned16(d_k_src) || !aligned16(d_v_src))
    return SMART_EINVAL;
  dim3 grid;
  if (!copy_grid(n_tokens, num_kv_heads, head_dim, &grid)) return SMART_EINVAL;
  const Pages pg{num_kv_heads, head_dim, block_size, num_blocks, cache_block_stride, cache_head_stride};
  if (src_dtype == SMART_F32)
    hipLaunchKernelGGL(kv_cache_write_fp4_kernel<float>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg, n_tokens,
                       (const float*)d_k_src, (const float*)d_v_src, d_slot_mapping, (uint8_t*)d_k_cache, (uint8_t*)d_v_cache);
  else
    hipLaunchKernelGGL(kv_cache_write_fp4_kernel<uint16_t>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg,
                       n_tokens, (const uint16_t*)d_k_src, (const uint16_t*)d_v_src, d_slot_mapping, (uint8_t*)d_k_cache,
                       (uint8_t*)d_v_cache);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}

extern "C" int32_t kv_cache_read_fp4(smart_ctx* ctx, void* stream, int32_t dst_dtype, int32_t n_tokens, int32_t num_kv_heads,
                                     int32_t head_dim, int32_t block_size, int32_t num_blocks, const void* d_k_cache,
                                     const void* d_v_cache, int64_t cache_block_stride, int64_t cache_head_stride,
                                     const int64_t* d_slot_mapping, void* d_k_dst, void* d_v_dst) {
  if (!ctx || n_tokens < 0 || !pages_ok(dst_dtype, num_kv_heads, head_dim, block_size, num_blocks, d_k_cache, d_v_cache,
                                        cache_block_stride, cache_head_stride))
    return SMART_EINVAL;
  if (n_tokens == 0) return SMART_OK;
  if (!d_k_dst || !d_v_dst || !d_slot_mapping || !d_k_cache || !d_v_cache || !aligned16(d_k_dst) || !aligned16(d_v_dst))
    return SMART_EINVAL;
  dim3 grid;
  if (!copy_grid(n_tokens, num_kv_heads, head_dim, &grid)) return SMART_EINVAL;
  const Pages pg{num_kv_heads, head_dim, block_size, num_blocks, cache_block_stride, cache_head_stride};
  if (dst_dtype == SMART_F32)
    hipLaunchKernelGGL(kv_cache_read_fp4_kernel<float>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg, n_tokens,
                       (const uint8_t*)d_k_cache, (const uint8_t*)d_v_cache, d_slot_mapping, (float*)d_k_dst, (float*)d_v_dst);
  else
    hipLaunchKernelGGL(kv_cache_read_fp4_kernel<uint16_t>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg,
                       n_tokens, (const uint8_t*)d_k_cache, (const uint8_t*)d_v_cache, d_slot_mapping, (uint16_t*)d_k_dst,
                       (uint16_t*)d_v_dst);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}

extern "C" int32_t tree_commit_fp4(smart_ctx* ctx, void* stream, int32_t src_dtype, int32_t batch, int32_t max_depth,
                                   int32_t num_kv_heads, int32_t head_dim, int32_t block_size, int32_t max_blocks_per_seq,
                                   int32_t num_blocks, const int32_t* d_cu_nodes, const int32_t* d_accept_len,
                                   const int32_t* d_accept_path, const void* d_k_tree, const void* d_v_tree,
                                   const int32_t* d_block_table, const int32_t* d_prefix_len, void* d_k_cache, void* d_v_cache,
                                   int64_t cache_block_stride, int64_t cache_head_stride, int32_t* d_new_prefix_len,
                                   int32_t* d_status) {
  if (!ctx || batch < 0 || max_depth < 0 || max_depth > SMART_MAX_NODES || max_blocks_per_seq < 0 ||
      !pages_ok(src_dtype, num_kv_heads, head_dim, block_size, num_blocks, d_k_cache, d_v_cache, cache_block_stride,
                cache_head_stride))
    return SMART_EINVAL;
  if (batch == 0) return SMART_OK;
  if (batch > 65535) return SMART_EINVAL;  // grid y
  if (!d_cu_nodes || !d_accept_len || !d_accept_path || !d_k_tree || !d_v_tree || !d_block_table || !d_prefix_len || !d_k_cache ||
      !d_v_cache || !d_new_prefix_len || !d_status || d_new_prefix_len == d_prefix_len || !aligned16(d_k_tree) ||
      !aligned16(d_v_tree))
    return SMART_EINVAL;
  const Pages pg{num_kv_heads, head_dim, block_size, num_blocks, cache_block_stride, cache_head_stride};
  const smart::CommitInputs in{max_depth,  block_size,   max_blocks_per_seq, num_blocks,    d_cu_nodes,
                               d_accept_len, d_accept_path, d_block_table,      d_prefix_len};
  const dim3 grid(max_depth + 1, batch);
  if (src_dtype == SMART_F32)
    hipLaunchKernelGGL(tree_commit_fp4_kernel<float>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg, in, (const float*)d_k_tree,
                       (const float*)d_v_tree, (uint8_t*)d_k_cache, (uint8_t*)d_v_cache, d_new_prefix_len, d_status);
  else
    hipLaunchKernelGGL(tree_commit_fp4_kernel<uint16_t>, grid, dim3(kThreads), 0, (hipStream_t)stream, pg, in,
                       (const uint16_t*)d_k_tree, (const uint16_t*)d_v_tree, (uint8_t*)d_k_cache, (uint8_t*)d_v_cache,
                       d_new_prefix_len, d_status);
  SMART_HIP_CHECK(hipGetLastError());
  return SMART_OK;
}
