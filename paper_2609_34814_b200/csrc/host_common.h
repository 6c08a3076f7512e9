// Host-side helpers shared by the entry points: thread-local error text and launch counter.
#pragma once
#include <cstdarg>
#include <cstdio>
#include <cuda.h>
#include <cuda_runtime.h>
#include "waveal.h"

namespace waveal {

char* last_error_buffer();          // thread-local, 512 bytes
int32_t& launch_counter();          // thread-local

inline waveal_status fail(waveal_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(last_error_buffer(), 512, fmt, ap);
  va_end(ap);
  return s;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// SMs of the current device (looked up once a device); 0: not available
inline int sm_count() {
  static int counts[64] = {};
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev < 64 && counts[dev]) return counts[dev];
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  if (dev < 64) counts[dev] = n;
  return n;
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's cuTensorMapEncodeTiled (the library is not linked to the driver); NULL: not available
inline EncodeTiledFn tensor_map_encoder() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

#ifdef __CUDACC__
// The kernels of one call that follow each other on the stream: each is launched while the one before it
// drains (programmatic dependent launch), sets itself up, and waits before it touches what that one
// writes.  Every kernel launched this way waits, so whoever follows the last one follows all of them.
// The first kernel of a call is launched the ordinary way: it starts when all earlier work has ended.
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <class... Params, class... Args>
inline cudaError_t launch_chained(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream,
                                  Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}
#endif

// what append and attention ask of the cache and of the batch
inline waveal_status check_cache(const waveal_cache_desc* c) {
  if (c->n_pages <= 0 || c->kv_heads <= 0) return fail(WAVEAL_ERR_INVALID_ARG, "n_pages and kv_heads must be positive");
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return fail(WAVEAL_ERR_UNSUPPORTED, "page_size %d (supported: powers of two, 16 .. 65536)", c->page_size);
  if (c->kv_heads > (1 << 20)) return fail(WAVEAL_ERR_UNSUPPORTED, "more than 2^20 heads");
  if (c->dtype != WAVEAL_BF16 && c->dtype != WAVEAL_FP16)
    return fail(WAVEAL_ERR_UNSUPPORTED, "dtype %d (a cache holds WAVEAL_BF16 or WAVEAL_FP16)", c->dtype);
  return WAVEAL_OK;
}

inline waveal_status check_batch(const waveal_batch_desc* b) {
  if (b->batch < 0 || b->tokens < 0 || b->max_pages < 0 || b->prefix_len < 0)
    return fail(WAVEAL_ERR_INVALID_ARG, "batch, tokens, max_pages and prefix_len must not be negative");
  if (b->table_stride < b->max_pages) return fail(WAVEAL_ERR_INVALID_ARG, "table_stride is smaller than max_pages");
  return WAVEAL_OK;
}

#define WAVEAL_CUDA_OK(expr)                                                                 \
  do {                                                                                       \
    cudaError_t e__ = (expr);                                                                \
    if (e__ != cudaSuccess)                                                                  \
      return ::waveal::fail(WAVEAL_ERR_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e__)); \
  } while (0)

}  // namespace waveal
