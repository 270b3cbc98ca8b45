// Parameters and launchers of the attention kernels (mas_attention.hip), shared
// with the host entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mas_heads.h"

namespace mas {

constexpr int32_t kAttnMaxD = 128;

struct AttnParams {
  HeadView q, k, v, out, dout, dq, dk, dv;
  const int32_t* t_q;        // [B] or null
  const int32_t* t_k;        // [B] or null
  const float* slope;        // [Hq] or null
  const int32_t* doc_start;  // [B][N + 1] or null
  const int32_t* prefix;     // [B][N] ([B] without doc_start) or null
  float* lse;                // [B][Hq][Tq] or null
  float* part;               // split forward: [splits][pairs * tiles * 32][D + 2], the sums, the maximum, the total
  float2* stat;              // backward: [B][Hk][Tq * G] log-sum-exp in powers of two, and delta
  int2* see;                 // backward: [B][Tq] keys a token sees
  int32_t B, Tq, Tk, Hq, Hk, D, G, N;
  int32_t rows;              // Tq * G: the rows that share a key head, row = token * G + head of the group
  int32_t causal;
  int32_t vec;               // rows of every tensor are whole, aligned 16-byte pieces
  int32_t tiles, splits, span;  // row (or key) tiles; parts of the key axis, and the keys of each
  int32_t pairs;             // B * Hk
  int32_t spread;            // workgroups of a pair are eight apart
  uint32_t g_mul;            // row / G = g_mul ? mulhi(row, g_mul) : row >> g_shift
  int32_t g_shift;
  float scale, cap;
};

// How the forward pass is laid out on the chip.
struct AttnPlan {
  bool small;  // workgroups of 32 rows whose four waves take turns at the keys
  int32_t waves;  // else: of 32 rows each in a workgroup
  int32_t tiles, splits, span;
};
AttnPlan attention_plan(int32_t pairs, int32_t rows, int32_t Tk, int32_t D, bool fp32, float cap);
size_t attention_part_bytes(const AttnPlan& plan, int32_t pairs, int32_t D);

hipError_t launch_attention(AttnParams p, int dtype, const AttnPlan& plan, hipStream_t stream);
hipError_t launch_attention_backward(AttnParams p, int dtype, hipStream_t stream);

}  // namespace mas
