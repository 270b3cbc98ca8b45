// Host entry points of the operators around the alignment (C ABI declared in
// include/mas.h): attention, the norm and rotation of its queries and keys, the
// aligned loss.
//
// Every entry point validates its arguments on the host, then only enqueues
// kernels on the caller's stream; nothing synchronises or copies to the host.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "mas.h"
#include "mas_attention.h"
#include "mas_layout.h"
#include "mas_loss.h"
#include "mas_qk.h"

namespace mas {
namespace {

// Workgroups of a launch at most: far below 2^32 threads.
constexpr double kMaxBlocks = 1 << 22;

int elem_bytes(int32_t dtype) { return dtype == MAS_F32 ? 4 : 2; }

HeadView view(const mas_heads* h) { return h ? HeadView{static_cast<char*>(h->data), h->stride_b, h->stride_t, h->stride_h} : HeadView{nullptr, 0, 0, 0}; }

bool given(const mas_heads* h) { return h && h->data; }

// The largest power of two, at most 16 bytes, that every head of the tensor starts
// on a multiple of, in elements.
int alignment(const mas_heads& h, int bytes) {
  const uintptr_t a = (uintptr_t)h.data | (uintptr_t)(h.stride_b * bytes) | (uintptr_t)(h.stride_t * bytes) | (uintptr_t)(h.stride_h * bytes) | 16;
  return (int)((a & (~a + 1)) / bytes);
}

bool elements_ok(const mas_heads& h, int bytes) { return (uintptr_t)h.data % bytes == 0; }

mas_status check_desc(const mas_attention_desc* d) {
  if (!d) return MAS_ERR_NULL_POINTER;
  if (d->dtype != MAS_F32 && d->dtype != MAS_F16 && d->dtype != MAS_BF16) return MAS_ERR_BAD_VALUE;
  if (d->B < 1 || d->Tq < 1 || d->Tk < 1 || d->Hq < 1 || d->Hk < 1 || d->Hq % d->Hk != 0) return MAS_ERR_BAD_SHAPE;
  if (d->D < 1 || d->D > kAttnMaxD) return MAS_ERR_BAD_SHAPE;
  const double G = d->Hq / d->Hk, rows = d->Tq * G, pairs = (double)d->B * d->Hk + 8;
  // Rows and keys are 32-bit numbers with room for a tile beyond them, row / G is a
  // multiplication that is right for row G < 2^32, and a grid holds kMaxBlocks.
  if (rows > (1 << 30) || d->Tk > (1 << 30) || rows * G >= 4294967296.0) return MAS_ERR_BAD_SHAPE;
  if (pairs * std::ceil(rows / 32) > kMaxBlocks || pairs * std::ceil(d->Tk / 32.0) > kMaxBlocks) return MAS_ERR_BAD_SHAPE;
  if ((d->doc_start || d->prefix) && (d->N < 1 || d->N > (1 << 30) || (!d->doc_start && d->N != 1))) return MAS_ERR_BAD_SHAPE;
  if (!std::isfinite(d->scale) || !std::isfinite(d->cap) || d->cap < 0.0f) return MAS_ERR_BAD_VALUE;
  if (d->prefix && !d->causal) return MAS_ERR_BAD_VALUE;
  return MAS_OK;
}

AttnParams params(const mas_attention_desc& d) {
  AttnParams p = {};
  p.t_q = d.t_q;
  p.t_k = d.t_k;
  p.slope = d.slope;
  p.doc_start = d.doc_start;
  p.prefix = d.prefix;
  p.B = d.B;
  p.Tq = d.Tq;
  p.Tk = d.Tk;
  p.Hq = d.Hq;
  p.Hk = d.Hk;
  p.D = d.D;
  p.G = d.Hq / d.Hk;
  p.N = d.N;
  p.rows = d.Tq * p.G;
  p.pairs = d.B * d.Hk;
  p.causal = d.causal != 0;
  p.scale = d.scale;
  // Caps past these make pre and mul of the kernels infinite or nothing.  A cap of 1e30
  // bends only scores whose neighbours in fp32 are 1e16 apart and more, one of 1e-30
  // leaves scores that are all equal in fp32.
  p.cap = d.cap > 1e30f ? 0.0f : d.cap > 0.0f && d.cap < 1e-30f ? 1e-30f : d.cap;
  while ((1 << p.g_shift) < p.G) ++p.g_shift;
  if ((1 << p.g_shift) != p.G) p.g_mul = (uint32_t)(4294967296ull / p.G) + 1;
  return p;
}

size_t stat_bytes(const mas_attention_desc& d) {
  return (size_t)d.B * d.Hq * d.Tq * sizeof(float2) + (size_t)d.B * d.Tq * sizeof(int2);
}

size_t round_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

bool workspace_ok(const void* ws, size_t bytes, size_t need) { return need == 0 || (ws && (uintptr_t)ws % kAlign == 0 && bytes >= need); }

bool vectors(const mas_attention_desc& d, std::initializer_list<const mas_heads*> all) {
  const int bytes = elem_bytes(d.dtype);
  if (d.D * bytes % 16 != 0) return false;
  for (const mas_heads* h : all)
    if (alignment(*h, bytes) * bytes < 16) return false;
  return true;
}

mas_status check_qk(const mas_qk_desc* d, const mas_heads* q, const mas_heads* k) {
  if (!d) return MAS_ERR_NULL_POINTER;
  if (d->dtype != MAS_F32 && d->dtype != MAS_F16 && d->dtype != MAS_BF16) return MAS_ERR_BAD_VALUE;
  if (d->B < 1 || d->T < 1 || d->Hq < 1 || d->Hk < 0 || d->D < 1 || d->D > kQkMaxD) return MAS_ERR_BAD_SHAPE;
  if (d->R < 0 || d->R > d->D || d->R % 2 != 0 || (d->R > 0 && d->P < 1)) return MAS_ERR_BAD_SHAPE;
  if ((double)d->B * d->T > (1 << 24) || (double)d->Hq + d->Hk > 65536) return MAS_ERR_BAD_SHAPE;
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return MAS_ERR_BAD_VALUE;
  if (!given(q) || (d->Hk > 0 && !given(k)) || (d->R > 0 && (!d->cos || !d->sin))) return MAS_ERR_NULL_POINTER;
  return MAS_OK;
}

QkParams params(const mas_qk_desc& d, std::initializer_list<const mas_heads*> all) {
  QkParams p = {};
  p.wq = d.wq;
  p.wk = d.wk;
  p.cos = d.cos;
  p.sin = d.sin;
  p.pos = d.pos;
  p.t_x = d.t_x;
  p.B = d.B;
  p.T = d.T;
  p.Hq = d.Hq;
  p.Hk = d.Hk;
  p.D = d.D;
  p.R = d.R;
  p.P = d.P > 0 ? d.P : 1;
  p.interleaved = d.interleaved != 0;
  p.eps = d.eps;
  p.align = 16;
  for (const mas_heads* h : all)
    if (given(h)) {
      const int a = alignment(*h, elem_bytes(d.dtype));
      p.align = a < p.align ? a : p.align;
    }
  return p;
}

}  // namespace
}  // namespace mas

using namespace mas;

extern "C" {

size_t mas_attention_workspace_bytes(const mas_attention_desc* desc, int32_t backward) {
  if (check_desc(desc) != MAS_OK) return 0;
  const int32_t pairs = desc->B * desc->Hk;
  const AttnPlan plan = attention_plan(pairs, desc->Tq * (desc->Hq / desc->Hk), desc->Tk, desc->D, desc->dtype == MAS_F32, desc->cap);
  size_t n = attention_part_bytes(plan, pairs, desc->D);
  if (backward && stat_bytes(*desc) > n) n = stat_bytes(*desc);
  return round_up(n > 0 ? n : 1);
}

mas_status mas_attention(const mas_attention_desc* desc, const mas_heads* q, const mas_heads* k, const mas_heads* v,
                         const mas_heads* out, float* lse_out, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  if (!desc || !given(q) || !given(k) || !given(v) || !given(out)) return MAS_ERR_NULL_POINTER;
  const mas_status s = check_desc(desc);
  if (s != MAS_OK) return s;
  for (const mas_heads* h : {q, k, v, out})
    if (!elements_ok(*h, elem_bytes(desc->dtype))) return MAS_ERR_BAD_VALUE;
  AttnParams p = params(*desc);
  const AttnPlan plan = attention_plan(p.pairs, p.rows, p.Tk, p.D, desc->dtype == MAS_F32, p.cap);
  if (!workspace_ok(workspace, workspace_bytes, attention_part_bytes(plan, p.pairs, p.D))) return MAS_ERR_WORKSPACE;
  p.q = view(q);
  p.k = view(k);
  p.v = view(v);
  p.out = view(out);
  p.lse = lse_out;
  p.part = static_cast<float*>(workspace);
  p.vec = vectors(*desc, {q, k, v, out});
  return launch_attention(p, desc->dtype, plan, stream) == hipSuccess ? MAS_OK : MAS_ERR_HIP;
}

mas_status mas_attention_backward(const mas_attention_desc* desc, const mas_heads* dout, const mas_heads* q,
                                  const mas_heads* k, const mas_heads* v, const mas_heads* out, const float* lse,
                                  const mas_heads* dq, const mas_heads* dk, const mas_heads* dv, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream) {
  if (!desc || !lse) return MAS_ERR_NULL_POINTER;
  for (const mas_heads* h : {dout, q, k, v, out, dq, dk, dv})
    if (!given(h)) return MAS_ERR_NULL_POINTER;
  const mas_status s = check_desc(desc);
  if (s != MAS_OK) return s;
  for (const mas_heads* h : {dout, q, k, v, out, dq, dk, dv})
    if (!elements_ok(*h, elem_bytes(desc->dtype))) return MAS_ERR_BAD_VALUE;
  if (!workspace_ok(workspace, workspace_bytes, stat_bytes(*desc))) return MAS_ERR_WORKSPACE;
  AttnParams p = params(*desc);
  p.q = view(q);
  p.k = view(k);
  p.v = view(v);
  p.out = view(out);
  p.dout = view(dout);
  p.dq = view(dq);
  p.dk = view(dk);
  p.dv = view(dv);
  p.lse = const_cast<float*>(lse);
  p.stat = static_cast<float2*>(workspace);
  p.see = reinterpret_cast<int2*>(p.stat + (size_t)p.B * p.Hq * p.Tq);
  p.vec = vectors(*desc, {dout, q, k, v, out, dq, dk, dv});
  return launch_attention_backward(p, desc->dtype, stream) == hipSuccess ? MAS_OK : MAS_ERR_HIP;
}

mas_status mas_qk_norm_rope(const mas_qk_desc* desc, const mas_heads* q, const mas_heads* k, const mas_heads* q_out,
                            const mas_heads* k_out, hipStream_t stream) {
  const mas_status s = check_qk(desc, q, k);
  if (s != MAS_OK) return s;
  if (!given(q_out) || (desc->Hk > 0 && !given(k_out))) return MAS_ERR_NULL_POINTER;
  if (desc->Hk == 0) k = k_out = nullptr;
  for (const mas_heads* h : {q, k, q_out, k_out})
    if (given(h) && !elements_ok(*h, elem_bytes(desc->dtype))) return MAS_ERR_BAD_VALUE;
  QkParams p = params(*desc, {q, k, q_out, k_out});
  p.q = view(q);
  p.k = view(k);
  p.qo = view(q_out);
  p.ko = view(k_out);
  return launch_qk(p, desc->dtype, stream) == hipSuccess ? MAS_OK : MAS_ERR_HIP;
}

size_t mas_qk_norm_rope_workspace_bytes(int32_t B, int32_t T, int32_t Hq, int32_t Hk, int32_t D) {
  if (B < 1 || T < 1 || Hq < 1 || Hk < 0 || D < 1 || D > kQkMaxD || (double)B * T > (1 << 24) || (double)Hq + Hk > 65536)
    return 0;
  return round_up((size_t)qk_backward_blocks(B, T, Hq + Hk) * 2 * D * sizeof(float));
}

mas_status mas_qk_norm_rope_backward(const mas_qk_desc* desc, const mas_heads* dq_out, const mas_heads* dk_out,
                                     const mas_heads* q, const mas_heads* k, const mas_heads* dq, const mas_heads* dk,
                                     float* dwq, float* dwk, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
  const mas_status s = check_qk(desc, q, k);
  if (s != MAS_OK) return s;
  if (!given(dq_out) || !given(dq) || (desc->Hk > 0 && (!given(dk_out) || !given(dk)))) return MAS_ERR_NULL_POINTER;
  if (desc->Hk == 0) k = dk_out = dk = nullptr;
  for (const mas_heads* h : {q, k, dq_out, dk_out, dq, dk})
    if (given(h) && !elements_ok(*h, elem_bytes(desc->dtype))) return MAS_ERR_BAD_VALUE;
  if (!workspace_ok(workspace, workspace_bytes, mas_qk_norm_rope_workspace_bytes(desc->B, desc->T, desc->Hq, desc->Hk, desc->D)))
    return MAS_ERR_WORKSPACE;
  QkParams p = params(*desc, {q, k, dq_out, dk_out, dq, dk});
  p.q = view(q);
  p.k = view(k);
  p.qo = view(dq_out);
  p.ko = view(dk_out);
  p.dq = view(dq);
  p.dk = view(dk);
  p.dwq = dwq;
  p.dwk = dwk;
  p.part = static_cast<float*>(workspace);
  return launch_qk_backward(p, desc->dtype, stream) == hipSuccess ? MAS_OK : MAS_ERR_HIP;
}

static bool loss_shape_ok(int32_t B, int32_t T, int32_t S, int32_t D) {
  if (B < 1 || T < 1 || S < 1 || D < 1 || D > (1 << 16)) return false;
  // The smallest run of frames and block of channels of a workgroup is 16 x 64.
  if ((double)B * std::ceil(S / 16.0) * std::ceil(D / 64.0) > kMaxBlocks || (double)B * (T + 1.0) > kMaxBlocks) return false;
  return (double)T < (1 << 30) && (double)S < (1 << 30);
}

size_t mas_align_loss_workspace_bytes(int32_t B, int32_t T, int32_t S, int32_t D) {
  return loss_shape_ok(B, T, S, D) ? round_up(loss_workspace_bytes(B, T, S, D)) : 0;
}

mas_status mas_align_loss(const float* mu, const float* log_sigma, const float* z, const int32_t* row_start,
                          const float* item_weight, int32_t B, int32_t T, int32_t S, int32_t D, float* loss_out,
                          float* dmu_out, float* dlog_sigma_out, float* dz_out, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  if (!mu || !z || !row_start || !loss_out) return MAS_ERR_NULL_POINTER;
  if (!loss_shape_ok(B, T, S, D)) return MAS_ERR_BAD_SHAPE;
  if (!workspace_ok(workspace, workspace_bytes, loss_workspace_bytes(B, T, S, D))) return MAS_ERR_WORKSPACE;
  LossParams p = {};
  p.mu = mu;
  p.log_sigma = log_sigma;
  p.z = z;
  p.row_start = row_start;
  p.item_weight = item_weight;
  p.loss = loss_out;
  p.dmu = dmu_out;
  p.dlog_sigma = dlog_sigma_out;
  p.dz = dz_out;
  p.B = B;
  p.T = T;
  p.S = S;
  p.D = D;
  const uintptr_t a = (uintptr_t)mu | (uintptr_t)log_sigma | (uintptr_t)z | (uintptr_t)dmu_out | (uintptr_t)dlog_sigma_out | (uintptr_t)dz_out;
  return launch_loss(p, a % 16 == 0 && D % 4 == 0, workspace, stream) == hipSuccess ? MAS_OK : MAS_ERR_HIP;
}

}  // extern "C"
