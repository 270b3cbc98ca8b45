// Aligned loss: the negative log-likelihood of every frame under the Gaussian of
// its text row, summed over an item, and its gradients, in one pass over the frames.
//
//   r = z - mu, w = exp(-2 log_sigma)
//   loss = sum over frames and channels of ln(2 pi)/2 + log_sigma + r^2 w / 2
//   dz = r w,  dmu = -sum over the row's frames of r w,
//   dlog_sigma = sum over the row's frames of 1 - r^2 w, each times the item's weight.
//
// Bound by memory: frames are read once and their gradients written once; a text
// row is read by the frames of its segment, neighbours in the same workgroup.
//
// The work is cut along the frames, not the text rows, whose shares of the frames
// differ by orders of magnitude.  A workgroup takes a chunk of frames, each of its
// groups of lanes a run of them, V channels a lane, and sums a row until the next
// one begins.  Rows inside a run are written at once; rows that the ends of a run
// cut are summed over the runs in LDS; rows that the ends of a chunk cut leave
// their sums in the workspace, where a second kernel adds them, in order, with the
// item's loss.  So sums do not depend on the order in which workgroups run.  All
// in fp32.
//
// Measured, 64 items of up to 1024 text rows and 4096 frames of 192 channels with
// log-sigmas: 138 us for 600 MB moved (294 read, 306 written), 4.3 TB/s (a copy: 5.1),
// and 5 us to join.  50 MB of the reads are frames past the items' ends, loaded for
// nothing beside their neighbours.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mas_heads.h"
#include "mas_loss.h"

namespace mas {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // frames a group has in flight
constexpr float kHalfLog2Pi = 0.9189385332046727f;

template <int V> __device__ __forceinline__ void load(const float* at, float (&x)[V]) {
  typedef float vec __attribute__((ext_vector_type(V)));
  const vec v = *reinterpret_cast<const vec*>(at);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = v[i];
}
// PAST: around the caches.
template <bool PAST, int V> __device__ __forceinline__ void store(float* at, const float (&x)[V]) {
  typedef float vec __attribute__((ext_vector_type(V)));
  vec v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = x[i];
  if constexpr (PAST)
    __builtin_nontemporal_store(v, reinterpret_cast<vec*>(at));
  else
    *reinterpret_cast<vec*>(at) = v;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x += __shfl_xor(x, s);
  return x;
}

template <int V, int GL, bool PAST>
__global__ void __launch_bounds__(kThreads) mas_loss_kernel(const LossParams p) {
  constexpr int kGroups = kThreads / GL, kCols = GL * V;
  constexpr int kMaxFrames = kGroups * 16;
  __shared__ int32_t src[kMaxFrames];
  __shared__ int32_t cut_row[2 * kGroups];
  __shared__ float cut[2 * kGroups][2][kCols];
  __shared__ float sums[kThreads / 64];
  const int slab = blockIdx.x % p.slabs, n = blockIdx.x / p.slabs;
  const int b = n / p.chunks, chunk = n % p.chunks;
  const int j0 = chunk * p.frames, count = min(p.frames, p.S - j0);
  const int32_t* rs = p.row_start + (size_t)b * (p.T + 1);
  const int tid = threadIdx.x, group = tid / GL;
  const int c0 = slab * kCols + tid % GL * V;
  const bool in = c0 < p.D;

  for (int k = tid; k < p.frames; k += kThreads) src[k] = -1;
  if (tid < 2 * kGroups) cut_row[tid] = -1;
  __syncthreads();
  // The text row of every frame of the chunk, clamped to it whatever the table holds.
  for (int i = tid; i < p.T; i += kThreads) {
    const int lo = max(rs[i], j0), hi = min(rs[i + 1], j0 + count);
    for (int j = lo; j < hi; ++j) src[j - j0] = i;
  }
  __syncthreads();

  const float weight = p.item_weight ? p.item_weight[b] : 1.0f;
  const bool rows = p.dmu || p.dlog_sigma;
  const int run = p.frames / kGroups, k0 = group * run, k1 = min(k0 + run, count);
  const float* z = p.z + ((size_t)b * p.S + j0) * p.D + c0;
  float* dz = p.dz ? p.dz + ((size_t)b * p.S + j0) * p.D + c0 : nullptr;
  float am[V], al[V], loss = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i) am[i] = al[i] = 0.0f;
  int row = -1, slot = 2 * group;

  // The sums of `row`, whose last frame in this run has been added.
  const auto flush = [&]() {
    if (row < 0 || !rows) return;
    if (rs[row] >= j0 + k0 && rs[row + 1] <= j0 + k1) {
      if (in) {
        const size_t at = ((size_t)b * p.T + row) * p.D + c0;
        float x[V];
        if (p.dmu) {
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] = -weight * am[i];
          store<PAST>(p.dmu + at, x);
        }
        if (p.dlog_sigma) {
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] = weight * al[i];
          store<PAST>(p.dlog_sigma + at, x);
        }
      }
    } else if (slot < 2 * group + 2) {  // two at most: the first and the last row of the run
#pragma unroll
      for (int i = 0; i < V; ++i) {
        cut[slot][0][tid % GL * V + i] = am[i];
        cut[slot][1][tid % GL * V + i] = al[i];
      }
      if (tid % GL == 0) cut_row[slot] = row;
      ++slot;
    }
  };

  for (int k = k0; k < k1; k += kUnroll) {
    float zv[kUnroll][V], mv[kUnroll][V], lv[kUnroll][V];
    int at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      // Without conditions, so that none waits for another: frames past the end and
      // without a row load neighbours, for nothing.
      const int f = min(k + u, k1 - 1);
      at[u] = k + u < k1 ? src[f] : -2;
      const size_t m = ((size_t)b * p.T + max(src[f], 0)) * p.D + (in ? c0 : 0);
      load(z + (size_t)f * p.D - (in ? 0 : c0), zv[u]);
      load(p.mu + m, mv[u]);
      if (p.log_sigma) load(p.log_sigma + m, lv[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (at[u] == -2) continue;
      if (at[u] != row) {
        flush();
        row = at[u];
#pragma unroll
        for (int i = 0; i < V; ++i) am[i] = al[i] = 0.0f;
      }
      float g[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        g[i] = 0.0f;
        if (at[u] >= 0 && in) {
          const float r = zv[u][i] - mv[u][i];
          const float ls = p.log_sigma ? lv[u][i] : 0.0f, y = p.log_sigma ? r * expf(-2.0f * ls) : r;
          loss += fmaf(0.5f * r, y, kHalfLog2Pi + ls);
          am[i] += y;
          al[i] += fmaf(-r, y, 1.0f);
          g[i] = weight * y;
        }
      }
      if (dz && in) store<PAST>(dz + (size_t)(k + u) * p.D, g);
    }
  }
  flush();

  loss = wave_sum(loss);
  if (tid % 64 == 0) sums[tid / 64] = loss;
  __syncthreads();
  if (tid == 0) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) x += sums[w];
    p.part_loss[((size_t)b * p.chunks + chunk) * p.slabs + slab] = x;
  }
  if (!rows) return;
  // Rows without a frame: zeros, this chunk's share of the text.
  const int i0 = (int)((int64_t)p.T * chunk / p.chunks), i1 = (int)((int64_t)p.T * (chunk + 1) / p.chunks);
  for (int i = i0 + group; i < i1; i += kGroups)
    if (in && rs[i + 1] <= rs[i]) {
      const size_t at = ((size_t)b * p.T + i) * p.D + c0;
      float zero[V];
#pragma unroll
      for (int v = 0; v < V; ++v) zero[v] = 0.0f;
      if (p.dmu) store<PAST>(p.dmu + at, zero);
      if (p.dlog_sigma) store<PAST>(p.dlog_sigma + at, zero);
    }
  if (tid >= kCols || slab * kCols + tid >= p.D) return;
  // Rows cut by the ends of runs, a channel a thread.
  const int c = slab * kCols + tid;
  float sm = 0.0f, sl = 0.0f;
  int open = -1, goes_on = -1;
  for (int s = 0; s <= 2 * kGroups; ++s) {
    const int i = s < 2 * kGroups ? cut_row[s] : -2;
    if (i == -1) continue;
    if (i != open && open >= 0) {
      if (rs[open] >= j0 && rs[open + 1] <= j0 + count) {
        const size_t at = ((size_t)b * p.T + open) * p.D + c;
        if (p.dmu) p.dmu[at] = -weight * sm;
        if (p.dlog_sigma) p.dlog_sigma[at] = weight * sl;
      } else {
        float* at = p.part + (((size_t)b * p.chunks + chunk) * 2 + (rs[open] < j0 ? 0 : 1)) * 2 * p.D + c;
        at[0] = sm;
        at[p.D] = sl;
        if (rs[open] >= j0) goes_on = open;
      }
      sm = sl = 0.0f;
    }
    open = i;
    if (i >= 0) {
      sm += cut[s][0][tid];
      sl += cut[s][1][tid];
    }
  }
  if (c == 0) p.part_row[(size_t)b * p.chunks + chunk] = goes_on;
}

// Rows cut by the ends of chunks: a wave for each chunk, which adds up the row that
// begins there and goes on.  Then a wave for each item's loss.
__global__ void __launch_bounds__(kThreads) mas_loss_join_kernel(const LossParams p) {
  const size_t n = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  const size_t cuts = p.dmu || p.dlog_sigma ? (size_t)p.B * p.chunks : 0;
  if (n >= cuts) {
    const size_t b = n - cuts;
    if (b >= (size_t)p.B) return;
    const size_t parts = (size_t)p.chunks * p.slabs;
    float x = 0.0f;
    for (size_t i = lane; i < parts; i += 64) x += p.part_loss[b * parts + i];
    x = wave_sum(x);
    if (lane == 0) p.loss[b] = x;
    return;
  }
  const int i = p.part_row[n];
  if (i < 0) return;
  const int b = (int)(n / p.chunks), first = (int)(n % p.chunks);
  const int end = min(max(p.row_start[(size_t)b * (p.T + 1) + i + 1], 1), p.S), last = (end - 1) / p.frames;
  const float weight = p.item_weight ? p.item_weight[b] : 1.0f;
  for (int c = lane; c < p.D; c += 64) {
    float sm = 0.0f, sl = 0.0f;
    for (int k = first; k <= last; ++k) {
      const float* at = p.part + (((size_t)b * p.chunks + k) * 2 + (k == first ? 1 : 0)) * 2 * p.D + c;
      sm += at[0];
      sl += at[p.D];
    }
    const size_t at = ((size_t)b * p.T + i) * p.D + c;
    if (p.dmu) p.dmu[at] = -weight * sm;
    if (p.dlog_sigma) p.dlog_sigma[at] = weight * sl;
  }
}

// Lanes a frame and workgroups of a launch, for channels in pieces of V.
int lanes_of(int D, int V) {
  if (V == 1) return 64;
  return D <= 64 ? 16 : D <= 128 ? 32 : 64;
}
void plan(LossParams& p, int V) {
  const int lanes = lanes_of(p.D, V), groups = kThreads / lanes;
  p.slabs = (p.D + lanes * V - 1) / (lanes * V);
  // Runs of 16 frames; of 4 where those would leave compute units without work
  // (measured, 16 / 4: 16 x 512 frames of 80 channels 16.3 / 13.7 us, 32 x 1024 of 192
  // 20.0 / 20.0, 64 x 2048 of 192 49.3 / 57.1).
  const int64_t blocks = (int64_t)p.B * p.slabs * ((p.S + 16 * groups - 1) / (16 * groups));
  p.frames = groups * (blocks >= 1024 ? 16 : 4);
  p.chunks = (p.S + p.frames - 1) / p.frames;
}
size_t bytes_of(const LossParams& p) {
  return (size_t)p.B * p.chunks * ((p.slabs + 4 * (size_t)p.D) * sizeof(float) + sizeof(int32_t));
}

template <int V, int GL> hipError_t launch(const LossParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)p.B * p.chunks * p.slabs);
  if (4.0 * p.B * ((double)p.S + 2.0 * p.T) * p.D > kPastBytes)
    hipLaunchKernelGGL((mas_loss_kernel<V, GL, true>), grid, dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL((mas_loss_kernel<V, GL, false>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

size_t loss_workspace_bytes(int32_t B, int32_t T, int32_t S, int32_t D) {
  LossParams p = {};
  p.B = B;
  p.T = T;
  p.S = S;
  p.D = D;
  plan(p, 1);
  size_t n = bytes_of(p);
  plan(p, 4);
  return bytes_of(p) > n ? bytes_of(p) : n;
}

hipError_t launch_loss(LossParams p, bool vec, void* workspace, hipStream_t stream) {
  plan(p, vec ? 4 : 1);
  p.part = static_cast<float*>(workspace);
  p.part_loss = p.part + (size_t)p.B * p.chunks * 4 * p.D;
  p.part_row = reinterpret_cast<int32_t*>(p.part_loss + (size_t)p.B * p.chunks * p.slabs);
  const int lanes = lanes_of(p.D, vec ? 4 : 1);
  const hipError_t e = !vec          ? launch<1, 64>(p, stream)
                       : lanes == 16 ? launch<4, 16>(p, stream)
                       : lanes == 32 ? launch<4, 32>(p, stream)
                                     : launch<4, 64>(p, stream);
  if (e != hipSuccess) return e;
  const uint64_t waves = (p.dmu || p.dlog_sigma ? (uint64_t)p.B * p.chunks : 0) + p.B;
  hipLaunchKernelGGL(mas_loss_join_kernel, dim3((uint32_t)((waves + kThreads / 64 - 1) / (kThreads / 64))), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace mas
