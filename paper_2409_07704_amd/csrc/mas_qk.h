// Parameters and launchers of the norm-and-rotation kernels (mas_qk.hip), shared
// with the host entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mas_heads.h"

namespace mas {

constexpr int32_t kQkMaxD = 256;

struct QkParams {
  HeadView q, k;            // inputs
  HeadView qo, ko;          // forward: outputs; backward: gradients of the outputs
  HeadView dq, dk;          // backward: gradients of the inputs
  const float *wq, *wk;     // [D] or null
  const float *cos, *sin;   // [P][R / 2]
  const int32_t* pos;       // [B][T] or null: the token's index
  const int32_t* t_x;       // [B] or null: T
  float* part;              // backward: [blocks][2][D] partial sums of dwq, dwk
  float *dwq, *dwk;         // [D] or null
  int32_t B, T, Hq, Hk, D, R, P, interleaved;
  int32_t align;            // every head starts on a multiple of this many elements (a power of two)
  float eps;
};

hipError_t launch_qk(const QkParams& p, int dtype, hipStream_t stream);
hipError_t launch_qk_backward(const QkParams& p, int dtype, hipStream_t stream);
// Workgroups of the backward pass, and so the partial sums of the weights' gradients.
int32_t qk_backward_blocks(int32_t B, int32_t T, int32_t heads);

}  // namespace mas
