// The library's host code on a machine without a GPU: the HIP calls it makes are defined here (an executable's symbols come
// before those of the HIP runtime), so that the test sees which kernel every call launches, and on what grid.
#define __HIP_PLATFORM_AMD__
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "smart_tree.h"

struct Launch {
  const void* kernel;
  dim3 grid, block;
};
static Launch last;
static int launches;

extern "C" {
hipError_t hipGetDeviceCount(int* n) { *n = 1; return hipSuccess; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
  memset(p, 0, sizeof *p);
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipGetSymbolAddress(void** p, const void*) { *p = nullptr; return hipErrorInvalidSymbol; }
hipError_t hipMalloc(void** p, size_t) { *p = malloc(64); return hipSuccess; }
hipError_t hipFree(void* p) { free(p); return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  last = Launch{f, grid, block};
  ++launches;
  return hipSuccess;
}
static dim3 pushed_grid, pushed_block;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  pushed_grid = grid;
  pushed_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* m, hipStream_t* s) {
  *grid = pushed_grid;
  *block = pushed_block;
  *m = 0;
  *s = nullptr;
  return hipSuccess;
}
}

static int failures;

// A window and first tokens that are together as many as the call's tokens, or more, hide nothing: the same kernel on the same grid.
static void full_window(smart_ctx* ctx, int dtype, int tokens, int hq, int hkv, int dim, bool lse) {
  alignas(256) static char somewhere[256];
  prompt_params p;
  memset(&p, 0, sizeof p);
  p.dtype = dtype;
  p.batch = 1;
  p.total_tokens = tokens;
  p.num_q_heads = hq;
  p.num_kv_heads = hkv;
  p.head_dim = dim;
  p.softmax_scale = 0.125f;
  p.q_stride = p.out_stride = (int64_t)hq * dim;
  p.k_stride = p.v_stride = (int64_t)hkv * dim;
  p.d_q = p.d_k = p.d_v = somewhere;
  p.d_out = somewhere;
  p.d_cu_tokens = (const int32_t*)somewhere;
  p.d_lse = lse ? (float*)somewhere : nullptr;
  launches = 0;
  int32_t rc = prompt_attention(ctx, nullptr, &p);
  const Launch plain = last;
  for (int32_t window : {1, (tokens + 1) / 2, tokens, tokens + 1, 0x7FFFFFFF})
    for (int32_t sinks : {window < tokens ? tokens - window : 0, 0x7FFFFFFF}) {
      rc |= prompt_attention_window(ctx, nullptr, &p, window, sinks);
      if (last.kernel != plain.kernel || last.grid.x != plain.grid.x || last.block.x != plain.block.x) {
        printf("dtype %d, %d tokens, %d / %d heads of %d, window %d, sinks %d: another kernel or grid (%u x %u, %u x %u without)\n", dtype,
               tokens, hq, hkv, dim, window, sinks, last.grid.x, last.block.x, plain.grid.x, plain.block.x);
        ++failures;
        return;
      }
    }
  if (rc != SMART_OK || launches != 11) printf("%d tokens: rc %d, %d launches\n", tokens, rc, launches), ++failures;
}

int main() {
  smart_ctx* ctx = nullptr;
  if (smart_create(&ctx, 0) != SMART_OK) return 1;
  for (int dtype : {SMART_BF16, SMART_F32})
    for (int dim : {64, 128})
      for (bool lse : {false, true})
        for (int tokens : {1, 64, 300, 1500, 2048, 5000, 8192, 16384}) {
          full_window(ctx, dtype, tokens, 32, 8, dim, lse);
          full_window(ctx, dtype, tokens, 64, 64, dim, lse);
          full_window(ctx, dtype, tokens, 8, 1, dim, lse);
        }
  smart_destroy(ctx);
  if (!failures) printf("launch driver ok\n");
  return failures != 0;
}
