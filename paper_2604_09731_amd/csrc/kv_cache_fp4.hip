// The 4-bit cache: kv_cache_write_fp4, kv_cache_read_fp4, tree_commit_fp4.
//
// A unit is the 32 head dims of one token and kv head that share a scale, of K or of V: one thread reads them, finds their
// largest absolute value, and converts them with the processor's instructions (fp4.h has the format and the rounding).
#include "common.h"
#include "fp4.h"
#include "tree_commit.h"

namespace {

constexpr int kThreads = 256;
constexpr int kUnit = 32;  // elements that share a scale

struct Unit {
  float x[kUnit];
};

__device__ inline void load_unit(Unit& u, const float* p) {
#pragma unroll
  for (int i = 0; i < kUnit / 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(p)[i];
    u.x[4 * i] = v.x, u.x[4 * i + 1] = v.y, u.x[4 * i + 2] = v.z, u.x[4 * i + 3] = v.w;
  }
}
__device__ inline void load_unit(Unit& u, const uint16_t* p) {
#pragma unroll
  for (int i = 0; i < kUnit / 8; ++i) {
    const uint4 v = reinterpret_cast<const uint4*>(p)[i];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u.x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
      u.x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
}
__device__ inline void store_unit(const Unit& u, float* p) {
#pragma unroll
  for (int i = 0; i < kUnit / 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(u.x[4 * i], u.x[4 * i + 1], u.x[4 * i + 2], u.x[4 * i + 3]);
}
__device__ inline void store_unit(const Unit& u, uint16_t* p) {  // exact: the values have two significant bits
#pragma unroll
  for (int i = 0; i < kUnit / 8; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __float_as_uint(u.x[8 * i + 2 * j]) >> 16 | (__float_as_uint(u.x[8 * i + 2 * j + 1]) & 0xFFFF0000u);
    reinterpret_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

struct Codes {
  uint32_t w[4];
  uint32_t scale;
};
__device__ inline Codes encode(const Unit& u) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) top = max(top, __float_as_uint(u.x[i]) & 0x7FFFFFFFu);
  Codes c;
  c.scale = smart::fp4_scale_byte(top);
  const float s = smart::fp4_scale(c.scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) c.w[i] = c.scale == 255u ? 0u : smart::fp4_codes8(u.x + 8 * i, s);
  return c;
}
__device__ inline void decode(Unit& u, const Codes& c) {
  const float s = smart::fp4_scale(c.scale);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const smart::fp4_floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w[i], s, 0);
    const smart::fp4_floatx2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w[i], s, 1);
    const smart::fp4_floatx2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w[i], s, 2);
    const smart::fp4_floatx2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c.w[i], s, 3);
    u.x[8 * i] = a[0], u.x[8 * i + 1] = a[1], u.x[8 * i + 2] = b[0], u.x[8 * i + 3] = b[1];
    u.x[8 * i + 4] = d[0], u.x[8 * i + 5] = d[1], u.x[8 * i + 6] = e[0], u.x[8 * i + 7] = e[1];
  }
}

__device__ inline void put_k(uint8_t* page, int bs, int D, int slot, int d, const Codes& c) {
  *reinterpret_cast<uint4*>(page + smart::fp4_k_vector(bs, slot, d)) = make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]);
  page[smart::fp4_k_scale(bs, D, slot, d)] = (uint8_t)c.scale;
}
__device__ inline void put_v(uint8_t* page, int bs, int D, int slot, int d, const Codes& c) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *reinterpret_cast<uint16_t*>(page + smart::fp4_v_code(D, slot, d + 4 * i)) = (uint16_t)(c.w[i >> 1] >> (16 * (i & 1)));
  page[smart::fp4_v_scale(bs, D, slot, d)] = (uint8_t)c.scale;
}
__device__ inline Codes get_k(const uint8_t* page, int bs, int D, int slot, int d) {
  const uint4 v = *reinterpret_cast<const uint4*>(page + smart::fp4_k_vector(bs, slot, d));
  return Codes{{v.x, v.y, v.z, v.w}, page[smart::fp4_k_scale(bs, D, slot, d)]};
}
__device__ inline Codes get_v(const uint8_t* page, int bs, int D, int slot, int d) {
  Codes c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = *reinterpret_cast<const uint16_t*>(page + smart::fp4_v_code(D, slot, d + 8 * i));
    const uint32_t hi = *reinterpret_cast<const uint16_t*>(page + smart::fp4_v_code(D, slot, d + 8 * i + 4));
    c.w[i] = lo | hi << 16;
  }
  c.scale = page[smart::fp4_v_scale(bs, D, slot, d)];
  return c;
}

// Pages of a cache: K and V lie alike.
struct Pages {
  int Hkv, D, block_size, num_blocks;
  int64_t block_stride, head_stride;  // bytes
};

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_cache_write_fp4_kernel(Pages pg, int64_t n_units, const T* __restrict__ k_src,
                                                                      const T* __restrict__ v_src,
                                                                      const int64_t* __restrict__ slot_mapping,
                                                                      uint8_t* __restrict__ k_cache, uint8_t* __restrict__ v_cache) {
  const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (u >= 2 * n_units) return;
  const bool values = u >= n_units;
  const int64_t at = values ? u - n_units : u;
  const int row = pg.Hkv * (pg.D / kUnit);
  const int64_t t = at / row;
  const int e = (int)(at - t * row), g = e / (pg.D / kUnit), d = (e - g * (pg.D / kUnit)) * kUnit;
  const int64_t slot_id = slot_mapping[t];
  if (slot_id < 0 || slot_id >= (int64_t)pg.num_blocks * pg.block_size) return;
  const int64_t block = slot_id / pg.block_size;
  const int slot = (int)(slot_id - block * pg.block_size);
  Unit x;
  load_unit(x, (values ? v_src : k_src) + at * kUnit);
  const Codes c = encode(x);
  uint8_t* page = (values ? v_cache : k_cache) + block * pg.block_stride + g * pg.head_stride;
  if (values) put_v(page, pg.block_size, pg.D, slot, d, c);
  else put_k(page, pg.block_size, pg.D, slot, d, c);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void kv_cache_read_fp4_kernel(Pages pg, int64_t n_units, const uint8_t* __restrict__ k_cache,
                                                                     const uint8_t* __restrict__ v_cache,
                                                                     const int64_t* __restrict__ slot_mapping, T* __restrict__ k_dst,
                                                                     T* __restrict__ v_dst) {
  const int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (u >= 2 * n_units) return;
  const bool values = u >= n_units;
  const int64_t at = values ? u - n_units : u;
  const int row = pg.Hkv * (pg.D / kUnit);
  const int64_t t = at / row;
  const int e = (int)(at - t * row), g = e / (pg.D / kUnit), d = (e - g * (pg.D / kUnit)) * kUnit;
  const int64_t slot_id = slot_mapping[t];
  Unit x;
  if (slot_id < 0 || slot_id >= (int64_t)pg.num_blocks * pg.block_size) {
#pragma unroll
    for (int i = 0; i < kUnit; ++i) x.x[i] = 0.f;
  } else {
    const int64_t block = slot_id / pg.block_size;
    const int slot = (int)(slot_id - block * pg.block_size);
    const uint8_t* page = (values ? v_cache : k_cache) + block * pg.block_stride + g * pg.head_stride;
    decode(x, values ? get_v(page, pg.block_size, pg.D, slot, d) : get_k(page, pg.block_size, pg.D, slot, d));
  }
  store_unit(x, (values ? v_dst : k_dst) + at * kUnit);
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
  const int slot = (r.start + i) % pg.block_size, per_head = pg.D / kUnit, row = pg.Hkv * per_head;
  const int64_t src = ((int64_t)base + r.node) * row * kUnit;
  for (int u = threadIdx.x; u < 2 * row; u += kThreads) {
    const bool values = u >= row;
    const int e = values ? u - row : u, g = e / per_head, d = (e - g * per_head) * kUnit;
    Unit x;
    load_unit(x, (values ? v_tree : k_tree) + src + (int64_t)e * kUnit);
    const Codes c = encode(x);
    uint8_t* page = (values ? v_cache : k_cache) + (int64_t)r.block * pg.block_stride + g * pg.head_stride;
    if (values) put_v(page, pg.block_size, pg.D, slot, d, c);
    else put_k(page, pg.block_size, pg.D, slot, d, c);
  }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The arguments that all three calls share.
bool pages_ok(int32_t dtype, int32_t num_kv_heads, int32_t head_dim, int32_t block_size, int32_t num_blocks, const void* k_cache,
              const void* v_cache, int64_t block_stride, int64_t head_stride) {
  if (dtype != SMART_F32 && dtype != SMART_BF16) return false;
  // (offsets inside a page and the units of a row are counted in 32 bits)
  if (num_kv_heads <= 0 || head_dim <= 0 || block_size <= 0 || num_blocks < 0 || (int64_t)head_dim * block_size >= (1 << 30) ||
      (int64_t)num_kv_heads * head_dim >= (1 << 30))
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
  const int64_t units = (int64_t)n_tokens * num_kv_heads * (head_dim / kUnit), groups = (2 * units + kThreads - 1) / kThreads;
  if (groups > 0x7FFFFFFF) return SMART_EINVAL;
  const Pages pg{num_kv_heads, head_dim, block_size, num_blocks, cache_block_stride, cache_head_stride};
  if (src_dtype == SMART_F32)
    hipLaunchKernelGGL(kv_cache_write_fp4_kernel<float>, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, pg, units,
                       (const float*)d_k_src, (const float*)d_v_src, d_slot_mapping, (uint8_t*)d_k_cache, (uint8_t*)d_v_cache);
  else
    hipLaunchKernelGGL(kv_cache_write_fp4_kernel<uint16_t>, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, pg,
                       units, (const uint16_t*)d_k_src, (const uint16_t*)d_v_src, d_slot_mapping, (uint8_t*)d_k_cache,
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
  const int64_t units = (int64_t)n_tokens * num_kv_heads * (head_dim / kUnit), groups = (2 * units + kThreads - 1) / kThreads;
  if (groups > 0x7FFFFFFF) return SMART_EINVAL;
  const Pages pg{num_kv_heads, head_dim, block_size, num_blocks, cache_block_stride, cache_head_stride};
  if (dst_dtype == SMART_F32)
    hipLaunchKernelGGL(kv_cache_read_fp4_kernel<float>, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, pg, units,
                       (const uint8_t*)d_k_cache, (const uint8_t*)d_v_cache, d_slot_mapping, (float*)d_k_dst, (float*)d_v_dst);
  else
    hipLaunchKernelGGL(kv_cache_read_fp4_kernel<uint16_t>, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, pg,
                       units, (const uint8_t*)d_k_cache, (const uint8_t*)d_v_cache, d_slot_mapping, (uint16_t*)d_k_dst,
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
