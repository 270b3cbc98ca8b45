// Parameters and launcher of the aligned loss (mas_loss.hip), shared with the
// host entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mas {

struct LossParams {
  const float *mu, *log_sigma, *z;  // log_sigma nullable
  const int32_t* row_start;
  const float* item_weight;         // nullable
  float *loss, *dmu, *dlog_sigma, *dz;  // the gradients nullable
  float* part_loss;                 // [B][chunks][slabs]
  float* part;                      // [B][chunks][2][2][D]: sums of the rows that a chunk's ends cut
  int32_t B, T, S, D;
  int32_t* part_row;                // [B][chunks] the row that begins in the chunk and goes on after it, or -1
  int32_t frames, chunks, slabs;    // frames a workgroup, workgroups an item; blocks of channels
};

// Device workspace for any alignment of the tensors.
size_t loss_workspace_bytes(int32_t B, int32_t T, int32_t S, int32_t D);
// vec: channels and tensors are whole, aligned 16-byte pieces.
hipError_t launch_loss(LossParams p, bool vec, void* workspace, hipStream_t stream);

}  // namespace mas
