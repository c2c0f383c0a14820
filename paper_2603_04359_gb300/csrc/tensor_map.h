// The driver's encoder of tensor maps, reached without linking against libcuda.
#pragma once
#include <mutex>

#include <cuda.h>
#include <cuda_runtime.h>

namespace cat {
namespace {   // (each file's own: a shared static would be one for all loaded copies of the library)

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn driver_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(p);
  });
  return fn;
}

// The encoder wants a context that is current in the calling thread.  A launch makes the device's so by itself, but the maps
// come before it: where a thread has had no CUDA work yet, the current device's context is made current here.
CUresult encode_tiled(CUtensorMap* map, CUtensorMapDataType type, cuuint32_t rank, void* base, const cuuint64_t* dims,
                             const cuuint64_t* strides, const cuuint32_t* box, const cuuint32_t* steps,
                             CUtensorMapInterleave interleave, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion l2,
                             CUtensorMapFloatOOBfill fill) {
  const EncodeTiledFn fn = driver_encode_fn();
  CUresult r = fn(map, type, rank, base, dims, strides, box, steps, interleave, swizzle, l2, fill);
  int dev = 0;
  if (r == CUDA_ERROR_INVALID_CONTEXT && cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess)
    r = fn(map, type, rank, base, dims, strides, box, steps, interleave, swizzle, l2, fill);
  return r;
}

// Null where the driver has no such function.
EncodeTiledFn encode_fn() { return driver_encode_fn() ? encode_tiled : nullptr; }

}  // namespace
}  // namespace cat
