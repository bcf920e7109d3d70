// Internal declarations of the gradient norm and clipping kernels.
#pragma once

#include "saef_internal.h"

namespace saef {

// Device-side view of a saef_grads.
struct GradsDev {
  void* const* ptr;  // [K L] first element of tensor l of worker k
  double* part;      // [K n_tiles] a tensor's part of a run, at its first tile there
  double* run_sums;  // [K runs] sum of each run
  int64_t runs;      // runs of run_tiles tiles, a wave each (0: one launch, a
                     // workgroup to a worker; part and run_sums are unused)
  int32_t run_tiles;
  int32_t cached;    // the norm's loads stay in the last-level cache
  int32_t K;
  int32_t dtype;
};

// Tiles of a worker whose norms one workgroup takes, at most: two a wave (32 tiles
// of 2048 elements, 4 workers: 4.9 us a call against 7.0 for two launches; 64 tiles
// 6.8 against 7.1, 100 small ones 10.0 against 7.0).
constexpr int kSmallTiles = 32;

// norms[k] = the 2-norm (inf: the largest magnitude) of worker k's gradient;
// tensor_norms[k][l] alike per tensor when non-null.  Enqueues one or
// two kernels.
hipError_t launch_grad_norm(const DevLayout& lay, const GradsDev& g, bool inf, float* norms,
                            float* tensor_norms, hipStream_t s);

// out == nullptr: gradients scaled in place; else out[k] (fp32 rows of d_pad).
hipError_t launch_clip(const DevLayout& lay, const GradsDev& g, float max_norm,
                       const float* norms, float* out, hipStream_t s);

}  // namespace saef
