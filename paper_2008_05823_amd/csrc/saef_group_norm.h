// Internal declarations of the group norm kernels.
#pragma once

#include "saef_internal.h"

namespace saef {

// Activations (SAEF_ACT_* of the C ABI).
constexpr int kActNone = 0;
constexpr int kActRelu = 1;
constexpr int kActSilu = 2;

// Shape of a group norm over K workers' N samples of P pixels by C channels
// in G groups, channels last, and how its kernels cut the work.
struct GroupNormDev {
  int64_t N, P;
  int32_t K, C, G, Cg;
  float eps;
  int32_t vec;     // elements of a load: 16 bytes' worth, or 1
  int32_t slab;    // channels of a workgroup: C, or a multiple of vec
  int32_t slabs;   // ceil(C / slab)
  int32_t splits;  // workgroups over the pixels of a sample
  int64_t split_pixels;  // pixels of each
  int32_t backwards;  // the second pass goes through the samples backwards
  float* part;     // [K N splits C 2] backward sums per channel
  double* pieces;  // [K N splits (G + slabs - 1) 2] sums per group and slab
};

constexpr int kParamWaves = 16;  // of a workgroup that adds up 64 channels of dgamma and dbeta

// How a kernel that reads its features once cuts the work: workgroups of
// `threads` threads, each holding `vectors` 16-byte vectors, take slabs of
// `slab` channels of whole groups, or of all groups where vectors do not divide
// the channels.  threads == 0: the shape does not fit.
struct GroupNormHeld {
  int32_t threads, vectors, slab, slabs;
};

// LDS of such a workgroup; at most 64 KB may be asked for.
size_t group_norm_held_lds(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                           bool back);
constexpr size_t kMostLds = 65536;

hipError_t launch_group_norm_forward(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                                     int act, const void* x, const float* gamma,
                                     const float* beta, int64_t ld, void* y, float* mean,
                                     float* rstd, hipStream_t s);

hipError_t launch_group_norm_backward(const GroupNormDev& d, const GroupNormHeld& held, int dtype,
                                      int act, const void* dy, const void* x, const float* gamma,
                                      const float* beta, int64_t ld, const float* mean,
                                      const float* rstd, void* dx, float* dgamma, float* dbeta,
                                      int64_t ldg, hipStream_t s);

}  // namespace saef
