// Launch interface of the kernels on lists of tensors (gfx950 only): the norm of gradients, gradients scaled to a highest norm,
// Adam's step.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "qsv.h"
#include "qsv_requests.h"

namespace qsv {

// Bytes of workspace that the two launches need, whatever the list.
size_t norm_scratch_bytes();
// outs NULL: in place; max_norm +inf: the norm alone where outs is NULL too, otherwise copies.
hipError_t launch_clip(const qsv_tensor* grads, const qsv_tensor* outs, int64_t n, double max_norm, float* norm, void* scratch, hipStream_t st);

struct AdamRates { double lr, b1, b2, eps, c1, c2; };      // c1, c2: 1 - b^t
hipError_t launch_adam_clipped(const qsv_adam_tensor* t, int64_t n, double max_norm, const AdamRates& by, float* norm, void* scratch, hipStream_t st);

}  // namespace qsv
