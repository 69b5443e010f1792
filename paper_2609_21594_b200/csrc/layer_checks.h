// What the entry points of the layer operators share: checks of arguments, and what a call does before and after its launches.
#pragma once

#include <initializer_list>

#include "boxes.h"
#include "layer_ops.h"

namespace muon {

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline bool known_dtype(int32_t d) { return d == MUON_DTYPE_BF16 || d == MUON_DTYPE_FP32; }

inline size_t bytes_of(int32_t d) { return d == MUON_DTYPE_BF16 ? 2 : 4; }

// The context's device must be current; its SM count comes with the answer.
inline int device_of(const muon_ctx* ctx, int* sms) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != ctx->device) return MUON_ERR_CUDA;
  return cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess ? MUON_OK : MUON_ERR_CUDA;
}

inline int launched(muon_ctx* ctx, int n) {
  if (n < 0) {
    (void)cudaGetLastError();      // a refused launch is this call's error, not the next one's
    return n;
  }
  ctx->launches += n;
  return MUON_OK;
}

inline Box rows_of(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t elem) {
  const int64_t e = int64_t(elem);
  return Box(p, 1, 1, rows, cols * e, 0, 0, ld * e);
}

// Whether a result lies over an input or over another result.  The first result may be one of `in_place` exactly.
inline bool results_clash(std::initializer_list<Box> results, std::initializer_list<Box> inputs, std::initializer_list<Box> in_place = {}) {
  for (const Box* r = results.begin(); r != results.end(); ++r) {
    for (const Box& in : inputs)
      if (boxes_meet(*r, in)) return true;
    for (const Box& in : in_place)
      if (!(r == results.begin() && same_box(*r, in)) && boxes_meet(*r, in)) return true;
    for (const Box* other = results.begin(); other != r; ++other)
      if (boxes_meet(*r, *other)) return true;
  }
  return false;
}

}  // namespace muon
