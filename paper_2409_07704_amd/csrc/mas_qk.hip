// Norm of queries and keys for each head, and the rotation to the token's
// position, in one pass; and its backward pass.
//
//   x^ = x / sqrt(mean(x^2) + eps),  y = x^ w,  and the pairs (a, b) of the first R
//   channels turn: (a c - b s, b c + a s).
//   backward: dy = dz turned back, dw = sum of dy x^ over all rows,
//   g = dy w, dx = (g - x^ mean(g x^)) / sqrt(mean(x^2) + eps).
//
// Bound by the vector pipe beside memory (78% busy forward, 80% backward: exchanges of
// partners, conversions and selects): every element is read once and written once, and
// nothing is kept between the passes (the backward pass finds the norm again from x).  A
// group of lanes holds one head of one token, V neighbouring channels a lane;
// sums over a head are exchanges inside the group, and a channel's partner in the
// turn is in the same lane (pairs side by side) or R / 2 / V lanes away.  A group
// walks over heads of its token, so that cosines and sines are fetched once for
// them.  Sums are in fp32; results are rounded once, to the inputs' type.  The
// gradients of the weights are summed in a fixed order: each group over its
// rows, a workgroup over its groups, one more kernel over the workgroups.
//
// Measured, 8 x 4096 tokens of 16 + 4 heads of 128 in bf16: forward 81 us for 336 MB,
// 4.1 TB/s; backward 136 us for 503 MB, 3.7 TB/s (a copy: 5.1); the weights' sum 6 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mas_qk.h"

namespace mas {
namespace {

constexpr int kThreads = 256;
// Workgroups of the backward pass at most (2048: 8 x 4096 tokens of 20 heads 219 us
// with the forward pass, 1024: 214).
constexpr int kMaxBlocks = 1024;
// Heads a group loads at a time, where it has as many (2: 217 us, 4: 214).
constexpr int kInFlight = 4;

template <class T, int V> struct Pack {
  typedef T type __attribute__((ext_vector_type(V)));
};
template <class T, int V> __device__ __forceinline__ void load(const T* at, float (&x)[V]) {
  const auto v = *reinterpret_cast<const typename Pack<T, V>::type*>(at);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)v[i];
}
// PAST: around the caches.
template <bool PAST, class T, int V> __device__ __forceinline__ void store(T* at, const float (&x)[V]) {
  typename Pack<T, V>::type v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (T)x[i];
  auto* to = reinterpret_cast<typename Pack<T, V>::type*>(at);
  if constexpr (PAST)
    __builtin_nontemporal_store(v, to);
  else
    *to = v;
}

// Sum over the GL lanes of a group, in all of them.
template <int GL> __device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int s = 1; s < GL; s *= 2) x += __shfl_xor(x, s);
  return x;
}

// Row of the tables for a token; positions past their end take the last row.
__device__ __forceinline__ size_t angle_row(const QkParams& p, int b, int t) {
  const int at = p.pos ? p.pos[(size_t)b * p.T + t] : t;
  return (size_t)min(max(at, 0), p.P - 1) * (p.R / 2);
}

// The turn of a head that lies V channels a lane, this lane's from c0 on.
template <int V> struct Turn {
  float c[V], s[V];  // of each channel's pair, s with the channel's sign
  int n;             // channels that turn
  int partner;       // lane of the pairs' other halves, or -1: neighbours in this lane
  __device__ __forceinline__ void set(const QkParams& p, int b, int t, int c0) {
    const size_t row = angle_row(p, b, t);
    const int half = p.R / 2, lane = threadIdx.x % 64;
    n = min(max(p.R - c0, 0), V);
    partner = p.interleaved ? -1 : n == 0 ? lane : c0 < half ? lane + half / V : lane - half / V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      c[i] = 1.0f;
      s[i] = 0.0f;
      if (i < n) {
        const int ch = c0 + i, k = p.interleaved ? ch / 2 : ch < half ? ch : ch - half;
        c[i] = p.cos[row + k];
        s[i] = p.sin[row + k] * ((p.interleaved ? ch % 2 == 0 : ch < half) ? -1.0f : 1.0f);
      }
    }
  }
  __device__ __forceinline__ void apply(float (&x)[V], float sign) const {
    float y[V];
    if (partner < 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = x[i ^ 1];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) y[i] = __shfl(x[i], partner);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = i < n ? fmaf(x[i], c[i], sign * s[i] * y[i]) : x[i];
  }
};

// A group's share of the work: one token and every `parts`-th of its heads.
struct Share {
  int b, t, part, heads;
  bool used;  // the token is inside its item
};
__device__ __forceinline__ Share share_of(const QkParams& p, size_t n, int parts) {
  Share s;
  s.part = (int)(n % parts);
  const size_t tok = n / parts;
  s.b = (int)(tok / p.T);
  s.t = (int)(tok % p.T);
  s.heads = p.Hq + p.Hk;
  s.used = s.t < (p.t_x ? min(max(p.t_x[s.b], 0), p.T) : p.T);
  return s;
}

// Head h of the token: queries first, then keys.
template <class T> __device__ __forceinline__ T* head(const QkParams& p, const HeadView& q, const HeadView& k, const Share& s, int h) {
  const HeadView& v = h < p.Hq ? q : k;
  return reinterpret_cast<T*>(v.data) + (int64_t)s.b * v.sb + (int64_t)s.t * v.st + (int64_t)(h < p.Hq ? h : h - p.Hq) * v.sh;
}

template <int V> __device__ __forceinline__ void weights(const float* w, int c0, bool in, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = w && in ? w[c0 + i] : 1.0f;
}

// U: heads a group has in flight.
template <class T, int V, int GL, int U, bool PAST>
__global__ void __launch_bounds__(kThreads) mas_qk_kernel(const QkParams p, int parts) {
  const size_t n = ((size_t)blockIdx.x * kThreads + threadIdx.x) / GL;
  if (n >= (size_t)p.B * p.T * parts) return;  // whole groups
  const int c0 = (int)(threadIdx.x % GL) * V;
  const bool in = c0 < p.D;
  const Share s = share_of(p, n, parts);
  Turn<V> turn;
  float wq[V], wk[V];
  turn.set(p, s.b, s.t, c0);
  weights(p.wq, c0, in, wq);
  weights(p.wk, c0, in, wk);
  for (int h0 = s.part; h0 < s.heads; h0 += U * parts) {
    // Loads without conditions (lanes past the channels and heads past the last one
    // load neighbours, for nothing), so that none waits for another.
    float x[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) load(head<T>(p, p.q, p.k, s, min(h0 + u * parts, s.heads - 1)) + (in ? c0 : 0), x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * parts;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[u][i] = in && s.used ? x[u][i] : 0.0f;
        sum = fmaf(x[u][i], x[u][i], sum);
      }
      const float r = rsqrtf(group_sum<GL>(sum) / (float)p.D + p.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) x[u][i] = s.used ? x[u][i] * (r * (h < p.Hq ? wq[i] : wk[i])) : 0.0f;
      turn.apply(x[u], 1.0f);
      if (in && h < s.heads) store<PAST>(head<T>(p, p.qo, p.ko, s, h) + c0, x[u]);
    }
  }
}

template <class T, int V, int GL, int U, bool PAST>
__global__ void __launch_bounds__(kThreads) mas_qk_backward_kernel(const QkParams p, int parts) {
  constexpr int kGroups = kThreads / GL;
  __shared__ float sums[kGroups][GL * V];
  const int c0 = (int)(threadIdx.x % GL) * V, group = threadIdx.x / GL;
  const bool in = c0 < p.D;
  float wq[V], wk[V], dwq[V], dwk[V];
  weights(p.wq, c0, in, wq);
  weights(p.wk, c0, in, wk);
#pragma unroll
  for (int i = 0; i < V; ++i) dwq[i] = dwk[i] = 0.0f;
  const size_t all = (size_t)p.B * p.T * parts;
  for (size_t n = (size_t)blockIdx.x * kGroups + group; n < all; n += (size_t)gridDim.x * kGroups) {
    const Share s = share_of(p, n, parts);
    Turn<V> turn;
    turn.set(p, s.b, s.t, c0);
    for (int h0 = s.part; h0 < s.heads; h0 += U * parts) {
      float x[U][V], g[U][V];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = min(h0 + u * parts, s.heads - 1), c = in ? c0 : 0;
        load(head<T>(p, p.q, p.k, s, h) + c, x[u]);
        load(head<T>(p, p.qo, p.ko, s, h) + c, g[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * parts;
        const bool counts = in && s.used && h < s.heads;
        float sum = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          x[u][i] = counts ? x[u][i] : 0.0f;
          g[u][i] = counts ? g[u][i] : 0.0f;
          sum = fmaf(x[u][i], x[u][i], sum);
        }
        turn.apply(g[u], -1.0f);
        const float r = rsqrtf(group_sum<GL>(sum) / (float)p.D + p.eps);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          x[u][i] = counts ? x[u][i] * r : 0.0f;  // r is infinite for zeros without eps
          const float d = g[u][i] * x[u][i];
          dwq[i] += h < p.Hq ? d : 0.0f;
          dwk[i] += h < p.Hq ? 0.0f : d;
          g[u][i] *= h < p.Hq ? wq[i] : wk[i];
          dot = fmaf(g[u][i], x[u][i], dot);
        }
        const float mean = group_sum<GL>(dot) / (float)p.D;
#pragma unroll
        for (int i = 0; i < V; ++i) x[u][i] = counts ? r * fmaf(-x[u][i], mean, g[u][i]) : 0.0f;
        if (in && h < s.heads) store<PAST>(head<T>(p, p.dq, p.dk, s, h) + c0, x[u]);
      }
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) sums[group][c0 + i] = which ? dwk[i] : dwq[i];
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += kThreads) {
      float x = 0.0f;
      for (int k = 0; k < kGroups; ++k) x += sums[k][c];
      p.part[((size_t)blockIdx.x * 2 + which) * p.D + c] = x;
    }
  }
}

// Any head size up to 256, any alignment: a wave for a head, channels 64 apart in a
// lane; partners are read from memory once more.
constexpr int kAny = kQkMaxD / 64;
__device__ __forceinline__ int partner(const QkParams& p, int c) {
  return c >= p.R ? c : p.interleaved ? c ^ 1 : c < p.R / 2 ? c + p.R / 2 : c - p.R / 2;
}
__device__ __forceinline__ void angle(const QkParams& p, size_t row, int c, float& cs, float& sn) {
  cs = 1.0f;
  sn = 0.0f;
  if (c >= p.R) return;
  const int k = p.interleaved ? c / 2 : c < p.R / 2 ? c : c - p.R / 2;
  cs = p.cos[row + k];
  sn = p.sin[row + k] * ((p.interleaved ? c % 2 == 0 : c < p.R / 2) ? -1.0f : 1.0f);
}

template <class T>
__global__ void __launch_bounds__(kThreads) mas_qk_any_kernel(const QkParams p, int parts) {
  const size_t n = ((size_t)blockIdx.x * kThreads + threadIdx.x) / 64;
  if (n >= (size_t)p.B * p.T * parts) return;
  const int lane = threadIdx.x % 64;
  const Share s = share_of(p, n, parts);
  const size_t row = angle_row(p, s.b, s.t);
  for (int h = s.part; h < s.heads; h += parts) {
    const T* in = head<T>(p, p.q, p.k, s, h);
    const float* w = h < p.Hq ? p.wq : p.wk;
    float x[kAny], y[kAny], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kAny; ++j) {
      const int c = lane + 64 * j;
      x[j] = y[j] = 0.0f;
      if (c < p.D && s.used) {
        x[j] = (float)in[c];
        y[j] = (float)in[partner(p, c)];
      }
      sum = fmaf(x[j], x[j], sum);
    }
    const float r = rsqrtf(group_sum<64>(sum) / (float)p.D + p.eps);
    T* out = head<T>(p, p.qo, p.ko, s, h);
#pragma unroll
    for (int j = 0; j < kAny; ++j) {
      const int c = lane + 64 * j;
      if (c >= p.D) continue;
      float cs, sn;
      angle(p, row, c, cs, sn);
      float z = x[j] * (r * (w ? w[c] : 1.0f));
      if (c < p.R) z = fmaf(z, cs, sn * (y[j] * (r * (w ? w[partner(p, c)] : 1.0f))));
      out[c] = (T)(s.used ? z : 0.0f);
    }
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads) mas_qk_any_backward_kernel(const QkParams p, int parts) {
  constexpr int kGroups = kThreads / 64;
  __shared__ float sums[kGroups][kQkMaxD];
  const int lane = threadIdx.x % 64, group = threadIdx.x / 64;
  float dwq[kAny], dwk[kAny];
#pragma unroll
  for (int j = 0; j < kAny; ++j) dwq[j] = dwk[j] = 0.0f;
  const size_t all = (size_t)p.B * p.T * parts;
  for (size_t n = (size_t)blockIdx.x * kGroups + group; n < all; n += (size_t)gridDim.x * kGroups) {
    const Share s = share_of(p, n, parts);
    const size_t row = angle_row(p, s.b, s.t);
    for (int h = s.part; h < s.heads; h += parts) {
      const T* in = head<T>(p, p.q, p.k, s, h);
      const T* dz = head<T>(p, p.qo, p.ko, s, h);
      const float* w = h < p.Hq ? p.wq : p.wk;
      float x[kAny], g[kAny], sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int j = 0; j < kAny; ++j) {
        const int c = lane + 64 * j;
        x[j] = g[j] = 0.0f;
        if (c < p.D && s.used) {
          float cs, sn;
          angle(p, row, c, cs, sn);
          x[j] = (float)in[c];
          g[j] = (float)dz[c];
          if (c < p.R) g[j] = fmaf(g[j], cs, -sn * (float)dz[partner(p, c)]);
        }
        sum = fmaf(x[j], x[j], sum);
      }
      const float r = rsqrtf(group_sum<64>(sum) / (float)p.D + p.eps);
#pragma unroll
      for (int j = 0; j < kAny; ++j) {
        const int c = lane + 64 * j;
        x[j] = s.used && c < p.D ? x[j] * r : 0.0f;  // r is infinite for zeros without eps
        if (h < p.Hq)
          dwq[j] += g[j] * x[j];
        else
          dwk[j] += g[j] * x[j];
        if (w && c < p.D) g[j] *= w[c];
        dot = fmaf(g[j], x[j], dot);
      }
      const float mean = group_sum<64>(dot) / (float)p.D;
      T* out = head<T>(p, p.dq, p.dk, s, h);
#pragma unroll
      for (int j = 0; j < kAny; ++j) {
        const int c = lane + 64 * j;
        if (c < p.D) out[c] = (T)(s.used ? r * fmaf(-x[j], mean, g[j]) : 0.0f);
      }
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kAny; ++j) sums[group][lane + 64 * j] = which ? dwk[j] : dwq[j];
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += kThreads) {
      float x = 0.0f;
      for (int k = 0; k < kGroups; ++k) x += sums[k][c];
      p.part[((size_t)blockIdx.x * 2 + which) * p.D + c] = x;
    }
  }
}

// dwq, dwk from the workgroups' sums: 16 columns a workgroup, 16 threads a column.
__global__ void __launch_bounds__(kThreads) mas_qk_weights_kernel(const QkParams p, int blocks) {
  __shared__ float sums[16][17];
  const int col = threadIdx.x % 16, part = threadIdx.x / 16, c = (int)blockIdx.x * 16 + col;
  float x = 0.0f;
  if (c < 2 * p.D)
#pragma unroll 8
    for (int i = part; i < blocks; i += 16) x += p.part[(size_t)i * 2 * p.D + c];
  sums[part][col] = x;
  __syncthreads();
  if (part > 0 || c >= 2 * p.D) return;
  x = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) x += sums[i][col];
  float* dw = c < p.D ? p.dwq : p.dwk;
  if (dw) dw[c < p.D ? c : c - p.D] = x;
}

// Groups that share a token's heads: several while tokens are few, so that there are
// groups for the whole chip; more heads a group save fetches of the angles.  Measured
// with at least 8192 / 32768 / 131072 groups, 20 heads, bf16: 4 x 1024 tokens of 128
// channels 14.9 / 18.2 / 28.3 us, backward 27.2 / 27.8 / 34.5; 32 x 1024 of 64 32.4 /
// 32.5 / 39.5 and 64.8 / 64.6 / 92.8.
int parts_of(const QkParams& p) {
  const int heads = p.Hq + p.Hk;
  const int64_t tokens = (int64_t)p.B * p.T;
  int parts = 1;
  while (parts < heads && tokens * parts < 8192) parts *= 2;
  return parts < heads ? parts : heads;
}

template <class T, int V, int GL, int U, bool PAST> hipError_t launch_u(const QkParams& p, int parts, bool back, hipStream_t stream) {
  if (back) {
    hipLaunchKernelGGL((mas_qk_backward_kernel<T, V, GL, U, PAST>), dim3(qk_backward_blocks(p.B, p.T, p.Hq + p.Hk)), dim3(kThreads), 0, stream, p, parts);
  } else {
    const uint64_t groups = (uint64_t)p.B * p.T * parts;
    hipLaunchKernelGGL((mas_qk_kernel<T, V, GL, U, PAST>), dim3((uint32_t)((groups * GL + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p, parts);
  }
  return hipGetLastError();
}

template <class T, int V, int GL> hipError_t launch(const QkParams& p, bool back, hipStream_t stream) {
  const int parts = parts_of(p);
  if ((p.Hq + p.Hk) / parts < kInFlight) return launch_u<T, V, GL, 1, false>(p, parts, back, stream);
  const bool past = (double)p.B * p.T * (p.Hq + p.Hk) * p.D * sizeof(T) > kPastBytes;
  return past ? launch_u<T, V, GL, kInFlight, true>(p, parts, back, stream) : launch_u<T, V, GL, kInFlight, false>(p, parts, back, stream);
}

template <class T> hipError_t launch_any(const QkParams& p, bool back, hipStream_t stream) {
  const int parts = parts_of(p);
  if (back) {
    hipLaunchKernelGGL((mas_qk_any_backward_kernel<T>), dim3(qk_backward_blocks(p.B, p.T, p.Hq + p.Hk)), dim3(kThreads), 0, stream, p, parts);
  } else {
    const uint64_t groups = (uint64_t)p.B * p.T * parts;
    hipLaunchKernelGGL((mas_qk_any_kernel<T>), dim3((uint32_t)((groups * 64 + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, p, parts);
  }
  return hipGetLastError();
}

// Whether a lane can hold V channels: heads are whole such pieces, and a piece's
// partners are one piece.
bool fits(const QkParams& p, int V) {
  return p.D % V == 0 && p.align % V == 0 && (p.interleaved || p.R / 2 % V == 0);
}

template <class T, int V> hipError_t by_width(const QkParams& p, bool back, hipStream_t stream) {
  const int lanes = p.D / V;
  if (lanes <= 8) return launch<T, V, 8>(p, back, stream);
  if (lanes <= 16) return launch<T, V, 16>(p, back, stream);
  if (lanes <= 32) return launch<T, V, 32>(p, back, stream);
  return launch<T, V, 64>(p, back, stream);
}

template <class T> hipError_t dispatch(const QkParams& p, bool back, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (fits(p, 8)) return by_width<T, 8>(p, back, stream);
  }
  if (fits(p, 4)) return by_width<T, 4>(p, back, stream);
  return launch_any<T>(p, back, stream);
}

hipError_t by_type(const QkParams& p, int dtype, bool back, hipStream_t stream) {
  if (dtype == kF32) return dispatch<float>(p, back, stream);
  if (dtype == kF16) return dispatch<_Float16>(p, back, stream);
  return dispatch<__bf16>(p, back, stream);
}

}  // namespace

int32_t qk_backward_blocks(int32_t B, int32_t T, int32_t heads) {
  const int64_t rows = (int64_t)B * T * heads;
  const int64_t blocks = (rows + 3) / 4;  // a wave each for every row, at most
  return (int32_t)(blocks < kMaxBlocks ? blocks : kMaxBlocks);
}

hipError_t launch_qk(const QkParams& p, int dtype, hipStream_t stream) { return by_type(p, dtype, false, stream); }

hipError_t launch_qk_backward(const QkParams& p, int dtype, hipStream_t stream) {
  const hipError_t e = by_type(p, dtype, true, stream);
  if (e != hipSuccess || (!p.dwq && !p.dwk)) return e;
  hipLaunchKernelGGL(mas_qk_weights_kernel, dim3((2 * p.D + 15) / 16), dim3(kThreads), 0, stream, p,
                     qk_backward_blocks(p.B, p.T, p.Hq + p.Hk));
  return hipGetLastError();
}

}  // namespace mas
