// Attention over text tokens and speech frames, forward and backward.
//
//   s = scale q.k;  s = cap tanh(s / cap) (with a cap);  s -= slope |place_q - place_k|
//   p = exp(s - lse) over the keys a query sees, out = sum p v
//   delta = sum dout out;  dp = dout.v;  ds = p (dp - delta) (1 - tanh^2) scale
//   dq = sum ds k;  dk = sum ds q;  dv = sum p dout
//
// What a query sees is one interval [lo, hi) of keys: its document (or the whole
// item), cut after its own place where the mask is causal, but never before the
// end of the document's prefix.  Each lane holds its row's interval in two
// registers, and a ballot tells whether a block of keys is seen by every row of
// the wave (no mask), by none (skipped) or by some.
//
// The G query heads of a key head form one row axis, row = token * G + head:
// keys and values are read once for the group, a step of one token still fills
// a matrix tile with its heads, and dk, dv of shared heads are one sum.
//
// Products are 32 x 32 matrix-core tiles, computed transposed: s^T = k q^T, so
// that a row's scores lie in one lane (and its partner 32 lanes on), and maxima
// and sums need one exchange.  p^T in that layout is the right-hand operand of
// out^T = v^T p^T as it stands, if the contraction runs over the keys in the order
// in which the lanes hold them: lane half h holds keys 8 (r/4) + 4 h + r % 4.
// v^T is read in that order too, with the transposing LDS reads for 16-bit types.
// fp32 uses the fp32 matrix cores in the same layout (eight products of depth 2
// for one of depth 16), so results are at fp32 level in fp32.
//
// Bound by, and measured (8192^3 products reach 1157 TFLOP/s in bf16 on this card, 153
// in fp32; a copy 5.1 TB/s):
//   long forward passes: matrix and vector pipes in turn, each wave its own scores,
//     exponents and sums, two waves a SIMD (8 items of 4096 causal frames, 16 heads of
//     128 over 4, bf16: 643 us, 855 TFLOP/s);
//   gradients: no pipe alone (vector 62% and 51% busy in dq and in dk, dv, matrix 39% and
//     30%), but the steps from scores to exponents to products in each wave and the
//     barrier of every 64 rows or keys (4 items, 8 heads over 2, capped, sloped: dq 325 us
//     for 3 products of 34 GFLOP and their recomputed exponents, dk and dv 527 us for 4;
//     forward 251);
//   short passes and documents: the chain of dependent steps from lengths to tables to
//     tiles, about 1 us each, and few tiles behind it (64 items of up to 1001 tokens, 3
//     heads of 64, 5 documents: 43 + 55 + 87 us for 173 MB);
//   steps over caches: memory (64 caches of up to 4096 keys, 203 MB: 43 us, 4.7 TB/s,
//     and 5 us to join the parts).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "mas_attention.h"

namespace mas {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;  // four waves
constexpr int kWaves = kThreads / 64;
constexpr int kMaxWaves = 8;
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.0f;  // powers of two
constexpr float kHalfCap = 256.0f;

// Eight elements of an operand: one lane's share of 16 steps of a contraction.
template <class T> struct Frag;
template <> struct Frag<float> { using type = f32x8; using four = f32x4; };
template <> struct Frag<_Float16> { using type = half8; using four = half4; };
template <> struct Frag<__bf16> { using type = bf8; using four = bf4; };
template <class T> using frag = typename Frag<T>::type;
template <class T> using four = typename Frag<T>::four;

__device__ __forceinline__ f32x16 mma(half8 a, half8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(bf8 a, bf8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Row (of the first operand) that register r of an accumulator holds.
__device__ __forceinline__ int acc_row(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

// x and its partner's 32 lanes on, in both lanes.
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  lo = __uint_as_float(r[0]);
  hi = __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_halves(float x) {
  float a, b;
  both_halves(x, a, b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float add_halves(float x) {
  float a, b;
  both_halves(x, a, b);
  return a + b;
}

// LDS written by lanes of the wave is read by others of the same wave.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A capped score by way of r = -1 / (e^2x + 1): tanh(x) = 1 + 2 r, whose last step the
// next factor takes along, and tanh'(x) = -4 (r + r r).  x is a product times `pre`;
// twice_pre: 2 pre in powers of two.  tanh so has an absolute error of up to 2.5 units
// of 2^-23, and a score, cap times it, an error that grows with the cap however small
// the score is.  Up to kHalfCap in 16-bit types that is a sixth at most of the rounding
// of p.  Larger caps, and fp32, take tanh itself (EXACT): for |x| < 1/4 the Taylor sum up
// to x^9, whose next term is below 2^-26 of x, so that a score has a relative error.  In
// the kernels of the ordinary caps that way spilled registers (dq of 128 channels 5 of
// them, of 64 channels 33), so large caps in 16 bits have kernels of their own, those of
// few rows and keys (4 x 4096 causal frames of 8 heads of 128, bf16, cap 50 / 257: 247 /
// 661 us, gradients 861 / 1587).
template <bool EXACT> __device__ __forceinline__ float bent(float product, float pre, float twice_pre) {
  const float e = __builtin_amdgcn_exp2f(product * twice_pre);
  const float r = __builtin_amdgcn_rcpf(-1.0f - e);
  if constexpr (EXACT) {
    const float t = fmaf(2.0f, r, 1.0f);
    const float x = product * pre, y = x * x;
    float s = fmaf(y, 62.0f / 2835.0f, -17.0f / 315.0f);
    s = fmaf(y, s, 2.0f / 15.0f);
    s = fmaf(y, s, -1.0f / 3.0f);
    s = fmaf(y * s, x, x);
    return fabsf(x) < 0.25f ? s : t;
  }
  return r;
}
// The way of ordinary caps.
template <class T> constexpr bool kExact = sizeof(T) == 4;
// tanh', without its factor 4 where r stands for tanh.
template <bool EXACT> __device__ __forceinline__ float bend_of(float x) { return fmaf(-x, x, EXACT ? 1.0f : -x); }

// 1 / l, and 0 where nothing was summed; NaN stays.
__device__ __forceinline__ float inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

struct Interval {
  int lo, hi;
};

// Keys that the query at `place` of item b sees; tk is the item's key length.
__device__ __forceinline__ Interval interval(const AttnParams& p, int b, int place, int tk) {
  int lo = 0, hi = tk;
  int pre = 0;
  if (p.doc_start) {
    const int32_t* t = p.doc_start + (size_t)b * (p.N + 1);
    int first = 0, n = p.N + 1;  // starts up to `place`: the first n of them are candidates
    while (n > 0) {
      const int step = n / 2;
      if (t[first + step] <= place) {
        first += step + 1;
        n -= step + 1;
      } else {
        n = step;
      }
    }
    if (first == 0 || first > p.N) return {0, 0};
    lo = max(t[first - 1], 0);
    hi = min(t[first], tk);
    if (p.prefix) pre = p.prefix[(size_t)b * p.N + first - 1];
  } else if (p.prefix) {
    pre = p.prefix[b];
  }
  if (p.causal) hi = min(hi, max(place + 1, lo + min(max(pre, 0), tk)));
  return hi > lo ? Interval{lo, hi} : Interval{0, 0};
}

__device__ __forceinline__ int clamp_len(const int32_t* t, int b, int n) { return t ? min(max(t[b], 0), n) : n; }

__device__ __forceinline__ int token_of(const AttnParams& p, int row) {
  return p.g_mul ? (int)__umulhi((uint32_t)row, p.g_mul) : row >> p.g_shift;
}

// Which (item, key head), tile and part a workgroup works on.  Workgroups go to
// the eight dies in turn; where there are pairs for all of them, the workgroups of
// one pair, which read the same keys, are eight apart.
struct Place {
  int pair, tile, split;
  bool idle;
};
__device__ __forceinline__ Place place_of(const AttnParams& p, uint32_t block, int tiles) {
  const uint32_t per = (uint32_t)tiles * (uint32_t)p.splits;
  uint32_t pair = block / per, rest = block % per;
  if (p.spread) {
    const uint32_t n = block / 8;
    pair = n / per * 8 + block % 8;
    rest = n % per;
  }
  return {(int)pair, (int)(rest % (uint32_t)tiles), (int)(rest / (uint32_t)tiles), pair >= (uint32_t)p.pairs};
}
__device__ __forceinline__ Place place_of(const AttnParams& p) { return place_of(p, blockIdx.x, p.tiles); }

template <class T> __device__ __forceinline__ const T* head(const HeadView& v, int b, int h) {
  return reinterpret_cast<const T*>(v.data) + (int64_t)b * v.sb + (int64_t)h * v.sh;
}
template <class T> __device__ __forceinline__ T* head_out(const HeadView& v, int b, int h) {
  return reinterpret_cast<T*>(v.data) + (int64_t)b * v.sb + (int64_t)h * v.sh;
}

// n elements from c on of a row of D, zeros past its end.
template <class T> __device__ __forceinline__ u32x4 load16(const T* row, int c, int D, bool vec) {
  if (vec) return c < D ? *reinterpret_cast<const u32x4*>(row + c) : u32x4(0);
  constexpr int E = 16 / sizeof(T);
  union {
    T e[E];
    u32x4 v;
  } u;
#pragma unroll
  for (int i = 0; i < E; ++i) u.e[i] = c + i < D ? row[c + i] : T(0);
  return u.v;
}

template <class T> __device__ __forceinline__ frag<T> load_frag(const T* row, int c, int D, bool vec) {
  union {
    u32x4 v[sizeof(frag<T>) / 16];
    frag<T> f;
  } u;
  constexpr int E = 16 / sizeof(T);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(frag<T>) / 16); ++i) u.v[i] = load16(row, c + i * E, D, vec);
  return u.f;
}

// A tile in LDS.  16-bit types: rows of DP elements whose 16-byte pieces are dealt out
// anew in every row, piece c of row r at c ^ turned(r).  The LDS gives 256 bytes a
// cycle, 64 banks: 16 lanes of a read of rows, a piece of 16 rows each, or 32 lanes of
// a transposing read, 64 bytes of 4 rows each.  So of 16 rows each has another turn
// (as far as rows share banks), and of 4 neighbours each another one in units of 64
// bytes.  (Rows 16 bytes longer instead suit only the reads of rows: the transposing
// ones took four times as long.)  fp32: rows 16 bytes longer, or not where only columns
// are read.
template <class T, int DP> constexpr int kLd = DP + (sizeof(T) == 4 ? 4 : 0);
template <class T, int DP> constexpr int kLdCols = DP;
template <class T> __device__ __forceinline__ int turned(int row, int ld) {
  if (sizeof(T) == 4) return 0;
  return row / 4 % 4 ^ (ld % 128 == 0 ? row % 4 * 4 : ld % 64 == 0 ? row / 2 % 2 * 4 : 0);
}

// Tiles of ROWS rows of DP channels on their way from memory to LDS, spread over
// TEAM threads in 16-byte pieces: rows k of one head, st apart, or (BY_ROWS) rows of
// the group's row axis.  Where a tile is inside the tensor, rows are whole aligned
// pieces and the tile's extent fits 32 bits, a piece's place in the tile is found
// once, and a tile costs one unconditional load each, which nothing waits for
// before `store`.  Other tiles are fetched by `store`, element by element if need be.
template <class T, int DP, int ROWS, int TEAM, bool BY_ROWS> struct Stage {
  static constexpr int E = 16 / sizeof(T), CPR = DP / E, N = ROWS * CPR / TEAM;
  static_assert(ROWS * CPR % TEAM == 0, "whole pieces for every thread");
  const AttnParams& p;
  const HeadView& v;
  const T* base;  // of the head, or of the group's first
  int tid, limit; // zeros from row `limit` on
  bool fast, whole;
  int at;
  // A head's pieces of one thread lie evenly apart where threads are whole rows.
  static constexpr bool kEven = !BY_ROWS && TEAM % CPR == 0;
  u32x4 r[N];
  uint32_t off[kEven ? 1 : N];
  __device__ __forceinline__ int row(int n) const { return (tid + n * TEAM) / CPR; }
  __device__ __forceinline__ int col(int n) const { return (tid + n * TEAM) % CPR * E; }
  __device__ __forceinline__ Stage(const AttnParams& p, const HeadView& v, int b, int hk, int limit, int tid)
      : p(p), v(v), base(head<T>(v, b, BY_ROWS ? hk * p.G : hk)), tid(tid), limit(limit), whole(false), at(0) {
    const int most = (1 << 29) / (ROWS * (int)sizeof(T));
    // Offsets inside a tile are unsigned 32-bit numbers: strides that go backwards, which
    // they do not hold, take the element-by-element way.
    fast = p.vec && v.st >= 0 && v.st < most && (!BY_ROWS || (32 % p.G == 0 && v.sh >= 0 && v.sh < most));
#pragma unroll
    for (int n = 0; n < (kEven ? 1 : N); ++n) {
      const int i = row(n), c = col(n) < p.D ? col(n) : 0;
      const int o = BY_ROWS ? (i >> p.g_shift) * (int)v.st + (i & (p.G - 1)) * (int)v.sh : i * (int)v.st;
      off[n] = (uint32_t)(o + c) * (uint32_t)sizeof(T);
    }
  }
  // Rows from `k0` on (a multiple of 32) are wanted next.
  __device__ __forceinline__ void load(int k0) {
    at = k0;
    whole = fast && k0 + ROWS <= limit;
    if (!whole) return;
    const char* tile = reinterpret_cast<const char*>(base + (int64_t)(BY_ROWS ? k0 >> p.g_shift : k0) * v.st);
#pragma unroll
    for (int n = 0; n < N; ++n)
      r[n] = *reinterpret_cast<const u32x4*>(kEven ? tile + (int64_t)(n * (TEAM / CPR)) * v.st * (int)sizeof(T) + off[0] : tile + off[n]);
  }
  __device__ __forceinline__ u32x4 slow(int i, int c) const {
    if (i >= limit) return u32x4(0);
    if (!BY_ROWS) return load16(base + (int64_t)i * v.st, c, p.D, p.vec);
    const int tok = token_of(p, i);
    return load16(base + (int64_t)(i - tok * p.G) * v.sh + (int64_t)tok * v.st, c, p.D, p.vec);
  }
  __device__ __forceinline__ u32x4* place(T* lds, int ld, int n) const {
    return reinterpret_cast<u32x4*>(lds + row(n) * ld + ((col(n) / E) ^ turned<T>(row(n), ld)) * E);
  }
  __device__ __forceinline__ void store(T* lds, int ld) const {
    if (whole) {
      const bool all = p.D == DP;
#pragma unroll
      for (int n = 0; n < N; ++n) *place(lds, ld, n) = all || col(n) < p.D ? r[n] : u32x4(0);
    } else {
#pragma unroll 1
      for (int n = 0; n < N; ++n) *place(lds, ld, n) = slow(at + row(n), col(n));
    }
  }
};

// Operand from rows of a tile: lane l holds row l % 32, channels c + 8 (l / 32) ...
template <class T> __device__ __forceinline__ frag<T> rows_frag(const T* tile, int ld, int c, int lane) {
  union {
    u32x4 v[sizeof(frag<T>) / 16];
    frag<T> f;
  } u;
  constexpr int E = 16 / sizeof(T);
  const int row = lane % 32, piece = c / E + 8 / E * (lane / 32);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(frag<T>) / 16); ++i)
    u.v[i] = *reinterpret_cast<const u32x4*>(tile + row * ld + ((piece + i) ^ turned<T>(row, ld)) * E);
  return u.f;
}

// Operand from columns of a tile: lane l holds channel c + l % 32 of the rows
// 16 m + 4 (l / 32) + {0..3, 8..11}.
template <class T> __device__ __forceinline__ frag<T> cols_frag(const T* tile, int ld, int m, int c, int lane) {
  const int h = lane / 32;
  if constexpr (sizeof(T) == 4) {
    frag<T> f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = tile[(16 * m + 8 * (e / 4) + 4 * h + e % 4) * ld + c + lane % 32];
    return f;
  } else {
    // Sixteen lanes read a block of 4 rows and 16 channels, four channels each, and
    // get it transposed: a channel each, of the four rows.
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int j = lane % 16;
    const int row = 4 * h + j / 4, piece = c / 8 + 2 * (lane / 16 % 2) + j % 4 / 2;
    const T* at = tile + (16 * m + row) * ld + 4 * (j % 2);
    union {
      s16x4 q[2];
      frag<T> f;
    } u;
    u.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + (piece ^ turned<T>(row, ld)) * 8));
    u.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * ld + (piece ^ turned<T>(row + 8, ld)) * 8));
    return u.f;
  }
}

// Registers 8 m ... 8 m + 7 of an accumulator as an operand.
template <class T> __device__ __forceinline__ frag<T> acc_frag(const f32x16& x, int m) {
  frag<T> f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (T)x[8 * m + e];
  return f;
}

// ds as an operand: rounded to the type, and in 16 bits what that leaves out, rounded
// again, as a second one.  The gradients then are as exact as their own rounding and
// the rounded output in delta let them be (4096 causal frames in bf16: error of dq over
// its size 0.0027 with one part, 0.0021 with two; its own rounding alone 0.0017).  It
// costs 8% of a training pass, 1054 -> 1143 us; the matrix cores are busy for a third of
// the kernels' run.
template <class T> struct Parts {
  static constexpr bool kTwo = sizeof(T) == 2;
  frag<T> hi, lo;
  __device__ __forceinline__ Parts(const f32x16& x, int m) : hi(acc_frag<T>(x, m)) {
    if constexpr (kTwo) {
#pragma unroll
      for (int e = 0; e < 8; ++e) lo[e] = (T)(x[8 * m + e] - (float)hi[e]);
    }
  }
  __device__ __forceinline__ f32x16 mma_to(frag<T> a, f32x16 c) const {
    c = mma(a, hi, c);
    if constexpr (kTwo) c = mma(a, lo, c);
    return c;
  }
};

// A row of one head from the transposed accumulators o[DP / 32], times mul: a lane
// holds four neighbours at a time.  A factor of 0 stands for a row without a
// result: zeros, whatever the accumulators hold.
template <class T, int DP> __device__ __forceinline__ void store_row(T* row, const f32x16* o, float mul, int half, int D, bool vec) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int c = 32 * d + acc_row(r, half);
      four<T> x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (T)(mul != 0.0f ? o[d][r + e] * mul : 0.0f);
      if (vec) {
        if (c < D) *reinterpret_cast<four<T>*>(row + c) = x;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < D) row[c + e] = x[e];
      }
    }
}

// A wave's 32 rows: lane l and l + 32 hold row l % 32.
struct Rows {
  int row, tok, h;      // of the row axis; its token, its query head
  int lo, hi, at;       // keys it sees, and its place among the keys
  bool in, used;        // the row is one of the tensor's; its token is inside the item
  float slope;          // in powers of two
};
__device__ __forceinline__ Rows rows_of(const AttnParams& p, int row, int b, int hk, int tq, int tk) {
  Rows r;
  r.row = row;
  r.in = row < p.rows;
  r.tok = token_of(p, r.in ? row : 0);
  r.h = hk * p.G + (r.in ? row - r.tok * p.G : 0);
  r.used = r.in && r.tok < tq;
  r.at = r.tok + tk - tq;
  const Interval s = r.used ? interval(p, b, r.at, tk) : Interval{0, 0};
  r.lo = s.lo;
  r.hi = s.hi;
  r.slope = p.slope ? p.slope[r.h] * kLog2E : 0.0f;
  return r;
}

// First and last number of the intervals that the workgroup's threads hold.
__device__ __forceinline__ Interval key_range(int lo, int hi, int (&lds)[2 * kMaxWaves]) {
  int a = hi > lo ? lo : 0x7fffffff, z = hi > lo ? hi : 0;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    a = min(a, __shfl_xor(a, s));
    z = max(z, __shfl_xor(z, s));
  }
  if (threadIdx.x % 64 == 0) {
    lds[threadIdx.x / 64] = a;
    lds[kMaxWaves + threadIdx.x / 64] = z;
  }
  __syncthreads();
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    a = min(a, lds[w]);
    z = max(z, lds[kMaxWaves + w]);
  }
  a = __builtin_amdgcn_readfirstlane(a);
  z = __builtin_amdgcn_readfirstlane(z);
  return a < z ? Interval{a, z} : Interval{0, 0};
}

enum class Seen { none, some, all };
// How the wave's rows see the n keys from k on.
__device__ __forceinline__ Seen seen(int lo, int hi, int k, int n) {
  if (__ballot(lo < k + n && hi > k) == 0) return Seen::none;
  return __ballot((lo <= k && hi >= k + n) || hi <= lo) == ~0ull ? Seen::all : Seen::some;
}

// From products to scores, in powers of two: x mul - slope distance, with x the
// product, or tanh(product pre) with a cap.
// That is mul x + add of the product, or of what `bent` makes of it, and the forward
// pass brings `add` in with the log-sum-exp.  lift: added to the exponent where tanh'
// lacks its factor 4, so that ds has it (and p, until dv is stored).
template <bool EXACT> struct ScoreRule {
  static constexpr bool kExactly = EXACT;
  float pre, twice_pre, mul, add, lift;
  bool capped, sloped;
};
template <bool EXACT> __device__ __forceinline__ float score_add(const AttnParams& p) { return !EXACT && p.cap > 0.0f ? p.cap * kLog2E : 0.0f; }
template <bool EXACT> __device__ __forceinline__ ScoreRule<EXACT> score_rule(const AttnParams& p) {
  ScoreRule<EXACT> s;
  s.capped = p.cap > 0.0f;
  s.sloped = p.slope != nullptr;
  s.pre = s.capped ? p.scale / p.cap : 1.0f;
  s.twice_pre = s.pre * (2.0f * kLog2E);
  s.mul = (s.capped ? p.cap : p.scale) * kLog2E;
  s.add = score_add<EXACT>(p);
  s.lift = 0.0f;
  if (!EXACT && s.capped) {
    s.mul *= 2.0f;
    s.lift = 2.0f;
  }
  return s;
}

// What undoes `lift`.
template <bool EXACT> __device__ __forceinline__ float p_unit(const AttnParams& p) { return !EXACT && p.cap > 0.0f ? 0.25f : 1.0f; }

// ------------------------------------------------------------------ forward
// Keys of a tile: 64, or 32 in fp32, whose rows are twice as long.
template <class T> constexpr int kTile = sizeof(T) == 4 ? 32 : 64;

// One wave's state: out^T of 32 rows, the reference of the exponents (a running
// maximum, at most kSlack behind) and each lane's part of the total.
template <class T, int DP> struct Forward {
  frag<T> q[DP / 16];
  f32x16 o[DP / 32];
  float m, l;
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = f32x16(0.0f);
    clear();
  }
  // No total: also of a row that sees nothing, which takes part in unmasked blocks.
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.0f;
  }
  // NB blocks of 32 keys from k0 on, in LDS.
  template <int NB, class Rule> __device__ __forceinline__ void step(const T* kt, const T* vt, int ld, int ldv, int k0, const Rows& w, const Rule& rule, int lane) {
    const Seen how = seen(w.lo, w.hi, k0, 32 * NB);
    if (how == Seen::none) return;
    const int half = lane / 32;
    // Scores stay short of their last factor, which the exponent's argument brings in,
    // unless a distance comes between or the factor turns their order round.
    const bool general = rule.sloped || rule.mul < 0.0f;
    const float mul = general ? 1.0f : rule.mul;
    f32x16 s[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      s[n] = f32x16(0.0f);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) s[n] = mma(rows_frag(kt + 32 * n * ld, ld, 16 * c, lane), q[c], s[n]);
    }
    if (rule.capped) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = bent<Rule::kExactly>(s[n][r], rule.pre, rule.twice_pre);
    }
    if (general) {
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float d = (float)(w.at - k0 - 32 * n - 4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] = fmaf(-w.slope, fabsf(d - acc_row(r, 0)), s[n][r] * rule.mul);
      }
    }
    if (how == Seen::some) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + 32 * n + acc_row(r, half);
          const bool sees = (key >= w.lo) & (key < w.hi);
          s[n][r] = sees ? s[n][r] : -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
    top = max_halves(top) * mul;
    // The reference of the exponents moves only when a score passes it by more than
    // kSlack: p is at most 2^kSlack then, which all types hold, and the sums are
    // seldom rescaled.
    if (__ballot(top > m + kSlack) != 0) {
      const float to = top > m + kSlack ? top : m;  // each row by itself: its result is the same in any company
      const float shrink = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.0f : to));
      l *= shrink;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) o[d] *= shrink;
      m = to;
    }
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], mul, -base));
        l += s[n][r];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const frag<T> pf = acc_frag<T>(s[n], h);  // rounded to T for the product; the total is not
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) o[d] = mma(cols_frag(vt, ldv, 2 * n + h, 32 * d, lane), pf, o[d]);
      }
    }
  }
};

template <class T, int DP> __device__ __forceinline__ void load_q(const AttnParams& p, const HeadView& v, const Rows& w, int b, int lane, frag<T> (&q)[DP / 16]) {
  const T* row = head<T>(v, b, w.h) + (int64_t)w.tok * v.st;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) q[c] = w.used ? load_frag(row, 16 * c + 8 * (lane / 32), p.D, p.vec) : frag<T>(0);
}

// A hidden value must not count whatever it holds, but its p, a 0, does not silence
// an infinity or a NaN in the product.  So a wave whose sums are not all finite
// makes them again here: without such elements, and next to that counts which
// results they do reach, by products with ones for the keys seen: `up` counts
// infinities and NaN, which become +inf, `down` negative infinities and NaN, which
// become -inf, both together NaN.  In a cold branch: 32 channels at a time, operands
// straight from memory, so that it takes fewer registers than the loop before it.

// The rows of one wave over the keys [from, to); with `part` sums, maximum and
// total go there, at this lane's row.
template <class T, bool EXACT>
__device__ __forceinline__ void forward_carefully(const AttnParams& p, int row, int b, int hk, int from, int to, float* part) {
  const int lane = threadIdx.x % 64, half = lane / 32;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const Rows w = rows_of(p, row, b, hk, tq, tk);
  const ScoreRule<EXACT> rule = score_rule<EXACT>(p);
  const T* qr = head<T>(p.q, b, w.h) + (int64_t)w.tok * p.q.st;
  const T* kb = head<T>(p.k, b, hk);
  const T* vb = head<T>(p.v, b, hk);
  T* out = head_out<T>(p.out, b, w.h) + (int64_t)w.tok * p.out.st;
  float m = -INFINITY, l = 0.0f;
#pragma unroll 1
  for (int c0 = 0; c0 < p.D; c0 += 32) {
    f32x16 o(0.0f), up(0.0f), down(0.0f);
    m = -INFINITY;
    l = 0.0f;
#pragma unroll 1
    for (int k0 = from / 32 * 32; k0 < to; k0 += 32) {
      if (seen(w.lo, w.hi, k0, 32) == Seen::none) continue;
      const int key = k0 + lane % 32;
      f32x16 s(0.0f);
#pragma unroll 1
      for (int c = 0; c < p.D; c += 16) {
        const frag<T> kf = key < tk ? load_frag(kb + (int64_t)key * p.k.st, c + 8 * half, p.D, p.vec) : frag<T>(0);
        const frag<T> qf = w.used ? load_frag(qr, c + 8 * half, p.D, p.vec) : frag<T>(0);
        s = mma(kf, qf, s);
      }
      float top = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = k0 + acc_row(r, half);
        const bool sees = (at >= w.lo) & (at < w.hi);
        float x = rule.capped ? bent<EXACT>(s[r], rule.pre, rule.twice_pre) : s[r];
        x = fmaf(-w.slope, fabsf((float)(w.at - at)), x * rule.mul);
        s[r] = sees ? x : -INFINITY;
        top = fmaxf(top, s[r]);
      }
      top = max_halves(top);
      const float high = top > m + kSlack ? top : m, base = high == -INFINITY ? 0.0f : high;
      const float shrink = __builtin_amdgcn_exp2f(m - base);
      l *= shrink;
      o *= shrink;
      m = high;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(s[r] - base);
        l += s[r];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        frag<T> v, vu, vd, see;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int at = k0 + 16 * h + acc_row(e, half), c = c0 + lane % 32;
          const T x = at < tk && c < p.D ? vb[(int64_t)at * p.v.st + c] : (T)0.0f;
          const bool fin = fabsf((float)x) < INFINITY, sees = (at >= w.lo) & (at < w.hi);
          v[e] = fin ? x : (T)0.0f;
          vu[e] = fin || (float)x == -INFINITY ? (T)0.0f : (T)1.0f;
          vd[e] = fin || (float)x == INFINITY ? (T)0.0f : (T)1.0f;
          see[e] = sees ? (T)1.0f : (T)0.0f;
        }
        o = mma(v, acc_frag<T>(s, h), o);
        up = mma(vu, see, up);
        down = mma(vd, see, down);
      }
    }
    const float total = add_halves(l), mul = part ? 1.0f : inverse(total);
    if (!w.in) continue;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int c = c0 + acc_row(r, half);
      const float mark = (up[r] > 0.0f ? INFINITY : 0.0f) + (down[r] > 0.0f ? -INFINITY : 0.0f);
      const float x = w.hi > w.lo ? o[r] * mul + mark : 0.0f;
      if (c >= p.D) continue;
      if (part)
        part[c] = x;
      else
        out[c] = (T)x;
    }
  }
  if (w.hi <= w.lo) {
    m = -INFINITY;
    l = 0.0f;
  }
  l = add_halves(l);
  if (!w.in || lane >= 32) return;
  if (part) {
    part[p.D] = m;
    part[p.D + 1] = l;
  } else if (p.lse) {
    p.lse[((size_t)b * p.Hq + w.h) * p.Tq + w.tok] = (m + __builtin_amdgcn_logf(l) + score_add<EXACT>(p)) * kLn2;
  }
}

// Whether a lane's accumulators are finite numbers.
template <int N> __device__ __forceinline__ bool finite(const f32x16 (&x)[N]) {
  float t = 0.0f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(x[n][r], 0.0f, t);
  return t == 0.0f;
}

// W waves a workgroup, 32 rows a wave; the workgroup shares each tile of keys and
// values, of which the next is on its way while one is used.
template <class T, int DP, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 2 && DP <= 64 ? 3 : 2) mas_attention_rows(const AttnParams p) {
  constexpr int KT = kTile<T>, LD = kLd<T, DP>, LDV = kLdCols<T, DP>;
  __shared__ __align__(16) T kt[2][KT * LD];
  __shared__ __align__(16) T vt[2][KT * LDV];
  __shared__ int range[2 * kMaxWaves];
  const Place at = place_of(p);
  if (at.idle) return;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  // The last rows see most where the mask is causal: they start first.
  const int tile = p.causal ? p.tiles - 1 - at.tile : at.tile;
  const Rows w = rows_of(p, 32 * W * tile + 32 * wave + lane % 32, b, hk, tq, tk);
  const Interval keys = key_range(w.lo, w.hi, range);
  const auto rule = score_rule<kExact<T>>(p);

  Forward<T, DP> f;
  load_q<T, DP>(p, p.q, w, b, lane, f.q);
  f.start();

  Stage<T, DP, KT, 64 * W, false> ks(p, p.k, b, hk, tk, tid), vs(p, p.v, b, hk, tk, tid);
  const int first = keys.lo / KT * KT;
  if (first < keys.hi) {
    ks.load(first);
    vs.load(first);
    ks.store(kt[0], LD);
    vs.store(vt[0], LDV);
  }
  __syncthreads();
  int cur = 0;
  for (int k0 = first; k0 < keys.hi; k0 += KT, cur ^= 1) {
    const bool more = k0 + KT < keys.hi;
    if (more) {
      ks.load(k0 + KT);
      vs.load(k0 + KT);
    }
    f.template step<KT / 32>(kt[cur], vt[cur], LD, LDV, k0, w, rule, lane);
    if (more) {
      ks.store(kt[cur ^ 1], LD);
      vs.store(vt[cur ^ 1], LDV);
    }
    __syncthreads();
  }
  if (__ballot(w.hi > w.lo && !finite(f.o)) != 0)
    return forward_carefully<T, kExact<T>>(p, 32 * W * tile + 32 * wave + lane % 32, b, hk, keys.lo, keys.hi, nullptr);
  if (!w.in) return;
  if (w.hi <= w.lo) f.clear();
  const float l = add_halves(f.l);
  store_row<T, DP>(head_out<T>(p.out, b, w.h) + (int64_t)w.tok * p.out.st, f.o, inverse(l), lane / 32, p.D, p.vec);
  if (p.lse && lane < 32) p.lse[((size_t)b * p.Hq + w.h) * p.Tq + w.tok] = (f.m + __builtin_amdgcn_logf(l) + score_add<kExact<T>>(p)) * kLn2;
}

// Few rows: 32 a workgroup, whose four waves take the blocks of 32 keys in turn,
// each with its own maximum, total and sums, joined at the end; with `splits` > 1
// a workgroup takes a part of the keys and a second kernel joins the parts.
template <class T, int DP, bool EXACT>
__global__ void __launch_bounds__(kThreads, 1) mas_attention_keys(const AttnParams p) {
  constexpr int LD = kLd<T, DP>, LDV = kLdCols<T, DP>;
  struct Tiles {
    T k[32 * LD], v[32 * LDV];
  };
  struct Join {
    float o[kWaves - 1][DP / 32 * 16][64], m[kWaves - 1][64], l[kWaves - 1][64];
  };
  __shared__ __align__(16) union {
    Tiles t[kWaves];
    Join j;
  } lds;
  __shared__ int range[2 * kMaxWaves];
  const Place at = place_of(p);
  if (at.idle) return;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int tile = p.causal ? p.tiles - 1 - at.tile : at.tile;
  const Rows w = rows_of(p, 32 * tile + lane % 32, b, hk, tq, tk);
  Interval keys = key_range(w.lo, w.hi, range);
  const auto rule = score_rule<EXACT>(p);
  keys.lo = max(keys.lo / 32 * 32, at.split * p.span);
  keys.hi = min(keys.hi, (at.split + 1) * p.span);

  Forward<T, DP> f;
  load_q<T, DP>(p, p.q, w, b, lane, f.q);
  f.start();

  Stage<T, DP, 32, 64, false> ks(p, p.k, b, hk, tk, lane), vs(p, p.v, b, hk, tk, lane);
  Tiles& mine = lds.t[wave];
  int k0 = keys.lo + 32 * wave;
  if (k0 < keys.hi) {
    ks.load(k0);
    vs.load(k0);
  }
  for (; k0 < keys.hi; k0 += 32 * kWaves) {
    ks.store(mine.k, LD);
    vs.store(mine.v, LDV);
    wave_sync();
    if (k0 + 32 * kWaves < keys.hi) {
      ks.load(k0 + 32 * kWaves);
      vs.load(k0 + 32 * kWaves);
    }
    f.template step<1>(mine.k, mine.v, LD, LDV, k0, w, rule, lane);
    wave_sync();
  }
  if (w.hi <= w.lo) f.clear();
  float* part = p.part + (((size_t)at.split * p.pairs + at.pair) * (32 * (size_t)p.tiles) + w.row) * (p.D + 2);
  // Also the barrier between the tiles and the sums, which share LDS.
  if (__syncthreads_or(w.hi > w.lo && !finite(f.o))) {
    if (wave == 0) forward_carefully<T, EXACT>(p, 32 * tile + lane % 32, b, hk, keys.lo, keys.hi, p.splits > 1 ? part : nullptr);
    return;
  }
  if (wave > 0) {
    lds.j.m[wave - 1][lane] = f.m;
    lds.j.l[wave - 1][lane] = f.l;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) lds.j.o[wave - 1][16 * d + r][lane] = f.o[d][r];
  }
  __syncthreads();
  if (wave > 0 || !w.in) return;
  float top = f.m;
#pragma unroll
  for (int i = 0; i < kWaves - 1; ++i) top = fmaxf(top, lds.j.m[i][lane]);
  const float base = top == -INFINITY ? 0.0f : top;
  float a = __builtin_amdgcn_exp2f(f.m - base), l = f.l * a;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) f.o[d] *= a;
#pragma unroll
  for (int i = 0; i < kWaves - 1; ++i) {
    a = __builtin_amdgcn_exp2f(lds.j.m[i][lane] - base);
    l = fmaf(a, lds.j.l[i][lane], l);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) f.o[d][r] = fmaf(a, lds.j.o[i][16 * d + r][lane], f.o[d][r]);
  }
  l = add_halves(l);
  if (p.splits > 1) {
    if (lane < 32) {
      part[p.D] = top;
      part[p.D + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 32 * d + acc_row(r, lane / 32);
        if (c < p.D) part[c] = f.o[d][r];
      }
    return;
  }
  store_row<T, DP>(head_out<T>(p.out, b, w.h) + (int64_t)w.tok * p.out.st, f.o, inverse(l), lane / 32, p.D, p.vec);
  if (p.lse && lane < 32) p.lse[((size_t)b * p.Hq + w.h) * p.Tq + w.tok] = (top + __builtin_amdgcn_logf(l) + score_add<EXACT>(p)) * kLn2;
}

// The parts of a row, joined: a wave for each row, two channels a lane.
template <class T, bool EXACT>
__global__ void __launch_bounds__(kThreads) mas_attention_join(const AttnParams p) {
  const size_t n = (size_t)blockIdx.x * kWaves + threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  const int pair = (int)(n / p.rows), row = (int)(n % p.rows);
  if (pair >= p.pairs) return;
  const size_t stride = (size_t)p.pairs * 32 * p.tiles * (p.D + 2);
  const float* o = p.part + ((size_t)pair * 32 * p.tiles + row) * (p.D + 2);
  // Maxima and totals of 64 parts at a time, one a lane; then the sums, whose loads
  // do not wait for each other.
  float top = -INFINITY, l = 0.0f, x[2] = {0.0f, 0.0f};
  for (int s0 = 0; s0 < p.splits; s0 += 64) {
    const bool in = s0 + lane < p.splits;
    const float m = in ? o[(s0 + lane) * stride + p.D] : -INFINITY;
    float to = m;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) to = fmaxf(to, __shfl_xor(to, i));
    to = fmaxf(top, to);
    const float base = to == -INFINITY ? 0.0f : to, shrink = __builtin_amdgcn_exp2f(top - base);
    const float a = __builtin_amdgcn_exp2f(m - base);
    float part = in ? a * o[(s0 + lane) * stride + p.D + 1] : 0.0f;
#pragma unroll
    for (int i = 1; i < 64; i *= 2) part += __shfl_xor(part, i);
    l = fmaf(l, shrink, part);
    x[0] *= shrink;
    x[1] *= shrink;
    const int n = min(64, p.splits - s0);
    for (int s = 0; s < n; s += 8) {
      // Lanes past the channels and parts past the end load a neighbour's, for nothing.
      float v[8][2];
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) v[u][e] = o[(s0 + min(s + u, n - 1)) * stride + min(lane + 64 * e, p.D - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float w = s + u < n ? __shfl(a, s + u) : 0.0f;
#pragma unroll
        for (int e = 0; e < 2; ++e) x[e] = w != 0.0f ? fmaf(w, v[u][e], x[e]) : x[e];
      }
    }
    top = to;
  }
  const int tok = token_of(p, row), b = pair / p.Hk, h = pair % p.Hk * p.G + row - tok * p.G;
  T* out = head_out<T>(p.out, b, h) + (int64_t)tok * p.out.st;
  const float mul = inverse(l);
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (lane + 64 * e < p.D) out[lane + 64 * e] = (T)(mul != 0.0f ? x[e] * mul : 0.0f);
  if (p.lse && lane == 0) p.lse[((size_t)b * p.Hq + h) * p.Tq + tok] = (top + __builtin_amdgcn_logf(l) + score_add<EXACT>(p)) * kLn2;
}

// ----------------------------------------------------------------- backward
// Sums of W waves, number `wave` among them, in the first of them: rounds through
// LDS (W / 2 times a wave's accumulators), which all waves of the workgroup make.
template <int W, int N> __device__ __forceinline__ void add_waves(f32x16 (&x)[N], float* lds, int wave, int lane) {
#pragma unroll
  for (int from = W / 2; from > 0; from /= 2) {
    __syncthreads();
    if (wave >= from && wave < 2 * from) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) lds[((wave - from) * N * 16 + n * 16 + r) * 64 + lane] = x[n][r];
    }
    __syncthreads();
    if (wave < from) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[n][r] += lds[(wave * N * 16 + n * 16 + r) * 64 + lane];
    }
  }
}

// dq of a wave's 32 rows; also delta, which the second kernel needs.
template <class T, int DP> struct BackwardQ {
  frag<T> q[DP / 16], g[DP / 16];  // queries and gradients of the output
  f32x16 dq[DP / 32];
  float base, delta;  // base: what the exponent has besides the score's factor
  template <int NB, class Rule> __device__ __forceinline__ void step(const T* kt, const T* vt, int ld, int k0, const Rows& w, const Rule& rule, int lane) {
    const int half = lane / 32;
#pragma unroll
    for (int n = 0; n < NB; ++n, kt += 32 * ld, vt += 32 * ld, k0 += 32) {
      const Seen how = seen(w.lo, w.hi, k0, 32);
      if (how == Seen::none) continue;
      f32x16 s(0.0f), dp(0.0f);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) s = mma(rows_frag(kt, ld, 16 * c, lane), q[c], s);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) dp = mma(rows_frag(vt, ld, 16 * c, lane), g[c], dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] -= delta;
      if (rule.capped) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = bent<Rule::kExactly>(s[r], rule.pre, rule.twice_pre);
          dp[r] *= bend_of<Rule::kExactly>(s[r]);
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], rule.mul, base);
      if (rule.sloped) {
        const float d = (float)(w.at - k0 - 4 * half);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(-w.slope, fabsf(d - acc_row(r, 0)), s[r]);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r]) * dp[r];
      if (how == Seen::some) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + acc_row(r, half);
          const bool sees = (key >= w.lo) & (key < w.hi);
          s[r] = sees ? s[r] : 0.0f;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Parts<T> sf(s, h);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) dq[d] = sf.mma_to(cols_frag(kt, ld, h, 32 * d, lane), dq[d]);
      }
    }
  }
};

// What a wave's rows need before their keys: queries, gradients, statistics.  KEEP:
// the kernel of dk and dv will want them.
template <class T, int DP, bool KEEP, class Rule>
__device__ __forceinline__ void start_dq(const AttnParams& p, BackwardQ<T, DP>& f, const Rows& w, const Rule& rule, int pair, int b, int hk, int lane, bool first) {
  load_q<T, DP>(p, p.q, w, b, lane, f.q);
  load_q<T, DP>(p, p.dout, w, b, lane, f.g);
  f.delta = 0.0f;
  const T* row = head<T>(p.out, b, w.h) + (int64_t)w.tok * p.out.st;
#pragma unroll
  for (int c = 0; c < DP / 16; ++c) {
    const frag<T> o = w.used ? load_frag(row, 16 * c + 8 * (lane / 32), p.D, p.vec) : frag<T>(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) f.delta = fmaf((float)o[e], (float)f.g[c][e], f.delta);
  }
  f.delta = add_halves(f.delta);
  const float lse = w.hi > w.lo ? p.lse[((size_t)b * p.Hq + w.h) * p.Tq + w.tok] * kLog2E : 0.0f;
  f.base = rule.add + rule.lift - lse;
  if (KEEP && w.in && lane < 32 && first) {
    p.stat[(size_t)pair * p.rows + w.row] = float2{lse, f.delta};
    if (hk == 0 && w.row == w.tok * p.G) p.see[(size_t)b * p.Tq + w.tok] = int2{w.lo, w.hi};
  }
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) f.dq[d] = f32x16(0.0f);
}
template <class T, int DP> __device__ __forceinline__ void store_dq(const AttnParams& p, const BackwardQ<T, DP>& f, const Rows& w, int b, int lane) {
  if (w.in) store_row<T, DP>(head_out<T>(p.dq, b, w.h) + (int64_t)w.tok * p.dq.st, f.dq, w.hi > w.lo ? p.scale : 0.0f, lane / 32, p.D, p.vec);
}

// W waves of 32 rows with shared tiles, as in the forward pass.
template <class T, int DP, int W>
__global__ void __launch_bounds__(64 * W, sizeof(T) == 4 ? 1 : DP <= 64 ? 3 : 2) mas_attention_dq(const AttnParams p) {
  constexpr int KT = kTile<T>, LD = kLd<T, DP>;
  __shared__ __align__(16) T kt[2][KT * LD];
  __shared__ __align__(16) T vt[2][KT * LD];
  __shared__ int range[2 * kMaxWaves];
  const Place at = place_of(p);
  if (at.idle) return;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int tile = p.causal ? p.tiles - 1 - at.tile : at.tile;
  const Rows w = rows_of(p, 32 * W * tile + 32 * wave + lane % 32, b, hk, tq, tk);
  const Interval keys = key_range(w.lo, w.hi, range);
  const auto rule = score_rule<kExact<T>>(p);
  BackwardQ<T, DP> f;
  start_dq<T, DP, true>(p, f, w, rule, at.pair, b, hk, lane, true);
  const int first = keys.lo / KT * KT;
  Stage<T, DP, KT, 64 * W, false> ks(p, p.k, b, hk, tk, tid), vs(p, p.v, b, hk, tk, tid);
  if (first < keys.hi) {
    ks.load(first);
    vs.load(first);
    ks.store(kt[0], LD);
    vs.store(vt[0], LD);
  }
  __syncthreads();
  int cur = 0;
  for (int k0 = first; k0 < keys.hi; k0 += KT, cur ^= 1) {
    const bool more = k0 + KT < keys.hi;
    if (more) {
      ks.load(k0 + KT);
      vs.load(k0 + KT);
    }
    f.template step<KT / 32>(kt[cur], vt[cur], LD, k0, w, rule, lane);
    if (more) {
      ks.store(kt[cur ^ 1], LD);
      vs.store(vt[cur ^ 1], LD);
    }
    __syncthreads();
  }
  store_dq(p, f, w, b, lane);
}

// What a row brings along: its statistics and the keys it sees.  Loaded without
// conditions (rows past the end load the last one's), put to use by `put`.
struct RowInfo {
  float2 stat;
  int2 see;
  float slope;
  int row, tok;
  __device__ __forceinline__ void load(const AttnParams& p, int b, int hk, int r) {
    row = r;
    const int i = min(r, p.rows - 1);
    tok = token_of(p, i);
    stat = p.stat[((size_t)b * p.Hk + hk) * p.rows + i];
    see = p.see[(size_t)b * p.Tq + tok];
    slope = p.slope ? p.slope[hk * p.G + i - tok * p.G] : 0.0f;
  }
  // The same from the tensors themselves: rows r and, in the lanes 32 on, r again.
  template <class T> __device__ __forceinline__ void make(const AttnParams& p, int b, int hk, int r, int tq, int tk, int lane) {
    const Rows w = rows_of(p, r, b, hk, tq, tk);
    row = r;
    tok = w.tok;
    see = int2{w.lo, w.hi};
    slope = p.slope ? p.slope[w.h] : 0.0f;
    float delta = 0.0f;
    const T* o = head<T>(p.out, b, w.h) + (int64_t)w.tok * p.out.st;
    const T* g = head<T>(p.dout, b, w.h) + (int64_t)w.tok * p.dout.st;
    for (int c = 8 * (lane / 32); c < p.D; c += 16) {
      const frag<T> x = w.used ? load_frag(o, c, p.D, p.vec) : frag<T>(0), y = w.used ? load_frag(g, c, p.D, p.vec) : frag<T>(0);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)x[e], (float)y[e], delta);
    }
    stat = float2{w.hi > w.lo ? p.lse[((size_t)b * p.Hq + w.h) * p.Tq + w.tok] * kLog2E : 0.0f, add_halves(delta)};
  }
};
// As a table for the workgroup's `keys` keys from kb0 on.  The exponent of a row and
// a key is mul x + base + slope (key - kb0): distances are linear on one side of the
// row's place; where the row sees keys on both sides here, those behind `at` take
// 2 slope (key - at) more off.
template <int ROWS> struct RowTable {
  float base[ROWS], less[ROWS], slope[ROWS], at[ROWS];  // less: -delta
  int lo[ROWS], hi[ROWS];
  // shift: from a token to its place; rows from `limit` on see nothing.
  template <class Rule> __device__ __forceinline__ void put(int i, const RowInfo& x, int shift, int limit, const Rule& rule, int kb0, int keys) {
    const int place = x.tok + shift, e = place - kb0;
    const float k = (e > 0 ? x.slope : -x.slope) * kLog2E;
    base[i] = fmaf(-k, (float)e, rule.add + rule.lift - x.stat.x);
    less[i] = -x.stat.y;
    slope[i] = k;
    at[i] = e > 0 && e < keys - 1 && x.see.y > place + 1 ? (float)e : INFINITY;
    lo[i] = x.row < limit ? x.see.x : 0;
    hi[i] = x.row < limit ? x.see.y : 0;
  }
  // Scores of rows i + 8 n + 0 ... 3 down the registers and the key kb0 + k, complete.
  template <class Rule> __device__ __forceinline__ void add_to(f32x16& s, int i, int k, bool both_sides, const Rule& rule) const;
};
template <class V> __device__ __forceinline__ V four_at(const void* at) { return *reinterpret_cast<const V*>(at); }
template <int ROWS> template <class Rule> __device__ __forceinline__ void RowTable<ROWS>::add_to(f32x16& s, int i, int k, bool both_sides, const Rule& rule) const {
  if (!rule.sloped) {
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const f32x4 b = four_at<f32x4>(&base[i + 2 * r]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[r + e] = fmaf(s[r + e], rule.mul, b[e]);
    }
    return;
  }
  const float place = (float)k;
#pragma unroll
  for (int r = 0; r < 16; r += 4) {
    const f32x4 b = four_at<f32x4>(&base[i + 2 * r]), m = four_at<f32x4>(&slope[i + 2 * r]);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[r + e] = fmaf(s[r + e], rule.mul, fmaf(m[e], place, b[e]));
  }
  if (!both_sides) return;
#pragma unroll
  for (int r = 0; r < 16; r += 4) {
    const f32x4 m = four_at<f32x4>(&slope[i + 2 * r]), where = four_at<f32x4>(&at[i + 2 * r]);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[r + e] = fmaf(-2.0f * m[e], fmaxf(place - where[e], 0.0f), s[r + e]);
  }
}

// dk, dv of a wave's 32 keys (lane l and l + 32 hold key l % 32): s = q k^T with
// the rows down the registers, so that p and ds are operands of dv^T = dout^T p
// and dk^T = q^T ds as they stand.
template <class T, int DP> struct BackwardK {
  frag<T> k[DP / 16], v[DP / 16];
  f32x16 dk[DP / 32], dv[DP / 32];
  __device__ __forceinline__ void start(const AttnParams& p, int b, int hk, int key, int tk, int lane) {
    const T* kr = head<T>(p.k, b, hk) + (int64_t)key * p.k.st;
    const T* vr = head<T>(p.v, b, hk) + (int64_t)key * p.v.st;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) {
      k[c] = key < tk ? load_frag(kr, 16 * c + 8 * (lane / 32), p.D, p.vec) : frag<T>(0);
      v[c] = key < tk ? load_frag(vr, 16 * c + 8 * (lane / 32), p.D, p.vec) : frag<T>(0);
    }
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = f32x16(0.0f);
  }
  // Rows i0 ... i0 + 31 of a tile in LDS against the keys from k0 on.
  template <int ROWS, class Rule> __device__ __forceinline__ void step(const T* qt, const T* gt, int ld, const RowTable<ROWS>& t, int i0, int kb0, int k0, const Rule& rule, int lane) {
    const int half = lane / 32, key = k0 + lane % 32, i = i0 + 4 * half;
    const int lo = t.lo[i0 + lane % 32], hi = t.hi[i0 + lane % 32];
    if (__ballot(lo < k0 + 32 && hi > k0) == 0) return;
    // Rows that see nothing have no statistics: they are masked, not taken for full.
    const bool mask = __ballot(lo <= k0 && hi >= k0 + 32) != ~0ull;
    const bool both_sides = rule.sloped && __ballot(t.at[i0 + lane % 32] != INFINITY) != 0;
    qt += i0 * ld;
    gt += i0 * ld;
    f32x16 s(0.0f), dp;  // dp: the products less delta
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const f32x4 less = four_at<f32x4>(&t.less[i + 2 * r]);
#pragma unroll
      for (int e = 0; e < 4; ++e) dp[r + e] = less[e];
    }
    {
      frag<T> x[DP / 16];
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) x[c] = rows_frag(qt, ld, 16 * c, lane);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) s = mma(x[c], k[c], s);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) x[c] = rows_frag(gt, ld, 16 * c, lane);
#pragma unroll
      for (int c = 0; c < DP / 16; ++c) dp = mma(x[c], v[c], dp);
    }
    if (rule.capped) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = bent<Rule::kExactly>(s[r], rule.pre, rule.twice_pre);
        dp[r] *= bend_of<Rule::kExactly>(s[r]);
      }
    }
    t.add_to(s, i, key - kb0, both_sides, rule);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(s[r]);
      dp[r] *= s[r];
    }
    if (mask) {
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const i32x4 from = four_at<i32x4>(&t.lo[i + 2 * r]), to = four_at<i32x4>(&t.hi[i + 2 * r]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool sees = (key >= from[e]) & (key < to[e]);
          s[r + e] = sees ? s[r + e] : 0.0f;
          dp[r + e] = sees ? dp[r + e] : 0.0f;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const frag<T> pf = acc_frag<T>(s, h);
      const Parts<T> sf(dp, h);
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        dv[d] = mma(cols_frag(gt, ld, h, 32 * d, lane), pf, dv[d]);
        dk[d] = sf.mma_to(cols_frag(qt, ld, h, 32 * d, lane), dk[d]);
      }
    }
  }
};

// The rows that see any of the n keys from kb0 on.
template <bool OWN = false>
__device__ __forceinline__ Interval rows_seeing(const AttnParams& p, int b, int tq, int kb0, int n, int tk, int (&range)[2 * kMaxWaves]) {
  int lo = 0x7fffffff, hi = 0;
  if (kb0 < tk) {
    for (int t = threadIdx.x; t < tq; t += blockDim.x) {
      int2 s;
      if (OWN) {
        const Interval v = interval(p, b, t + tk - tq, tk);
        s = int2{v.lo, v.hi};
      } else {
        s = p.see[(size_t)b * p.Tq + t];
      }
      if (s.x < kb0 + n && s.y > kb0) {
        lo = min(lo, t);
        hi = t + 1;
      }
    }
  }
  Interval rows = key_range(lo, hi, range);
  rows.lo *= p.G;
  rows.hi *= p.G;
  return rows;
}

template <class T, int DP, bool EXACT> __device__ __forceinline__ void store_keys(const AttnParams& p, int b, int hk, int key, const f32x16* dk, const f32x16* dv, int lane) {
  if (key >= p.Tk) return;
  store_row<T, DP>(head_out<T>(p.dk, b, hk) + (int64_t)key * p.dk.st, dk, p.scale, lane / 32, p.D, p.vec);
  store_row<T, DP>(head_out<T>(p.dv, b, hk) + (int64_t)key * p.dv.st, dv, p_unit<EXACT>(p), lane / 32, p.D, p.vec);
}

// Few rows or keys, and all keys in fp32: 32 of them a workgroup, whose four waves take
// the blocks of 32 of the others in turn; their sums are added at the end.
template <class T, int DP> struct FewLds {
  static constexpr int LD = kLd<T, DP>;
  T a[kWaves][32 * LD], b[kWaves][32 * LD];
  RowTable<32> table[kWaves];
  int range[2 * kMaxWaves];
  static_assert(sizeof(T) * 32 * LD * kWaves >= kWaves / 2 * (DP / 32) * 16 * 64 * sizeof(float), "the waves' sums fit");
};

template <class T, int DP, bool KEEP, bool EXACT> __device__ __forceinline__ void few_rows(const AttnParams& p, const Place& at, int tiles, FewLds<T, DP>& lds) {
  constexpr int LD = kLd<T, DP>;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int tile = p.causal ? tiles - 1 - at.tile : at.tile;
  const Rows w = rows_of(p, 32 * tile + lane % 32, b, hk, tq, tk);
  const Interval keys = key_range(w.lo, w.hi, lds.range);
  const auto rule = score_rule<EXACT>(p);
  BackwardQ<T, DP> f;
  start_dq<T, DP, KEEP>(p, f, w, rule, at.pair, b, hk, lane, wave == 0);
  Stage<T, DP, 32, 64, false> ks(p, p.k, b, hk, tk, lane), vs(p, p.v, b, hk, tk, lane);
  int k0 = keys.lo / 32 * 32 + 32 * wave;
  if (k0 < keys.hi) {
    ks.load(k0);
    vs.load(k0);
  }
  for (; k0 < keys.hi; k0 += 32 * kWaves) {
    ks.store(lds.a[wave], LD);
    vs.store(lds.b[wave], LD);
    wave_sync();
    if (k0 + 32 * kWaves < keys.hi) {
      ks.load(k0 + 32 * kWaves);
      vs.load(k0 + 32 * kWaves);
    }
    f.template step<1>(lds.a[wave], lds.b[wave], LD, k0, w, rule, lane);
    wave_sync();
  }
  add_waves<kWaves>(f.dq, reinterpret_cast<float*>(lds.a), wave, lane);
  if (wave == 0) store_dq(p, f, w, b, lane);
}

// OWN: without the statistics and intervals of another kernel.
template <class T, int DP, bool OWN, bool EXACT> __device__ __forceinline__ void few_keys(const AttnParams& p, const Place& at, FewLds<T, DP>& lds) {
  constexpr int LD = kLd<T, DP>;
  // fp32 fetches no tile ahead: with 128 channels, where the kernel spills as it is,
  // there are no registers for one.  (Up to 96 channels it holds 244 and spills none.)
  constexpr bool kAhead = sizeof(T) == 2;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int k0 = 32 * at.tile, key = k0 + lane % 32;
  const Interval rows = rows_seeing<OWN>(p, b, tq, k0, 32, tk, lds.range);
  const auto rule = score_rule<EXACT>(p);
  BackwardK<T, DP> f;
  f.start(p, b, hk, key, tk, lane);
  Stage<T, DP, 32, 64, true> qs(p, p.q, b, hk, tq * p.G, lane), gs(p, p.dout, b, hk, tq * p.G, lane);
  RowInfo info;
  const auto learn = [&](int r) {
    if (OWN)
      info.make<T>(p, b, hk, r + lane % 32, tq, tk, lane);
    else
      info.load(p, b, hk, r + lane % 32);
  };
  int r0 = rows.lo / 32 * 32 + 32 * wave;
  if (kAhead && r0 < rows.hi) {
    qs.load(r0);
    gs.load(r0);
    learn(r0);
  }
  for (; r0 < rows.hi; r0 += 32 * kWaves) {
    if (kAhead) {
      qs.store(lds.a[wave], LD);
      gs.store(lds.b[wave], LD);
    } else {
      qs.load(r0);
      qs.store(lds.a[wave], LD);
      gs.load(r0);
      gs.store(lds.b[wave], LD);
      learn(r0);
    }
    if (lane < 32) lds.table[wave].put(lane, info, tk - tq, rows.hi, rule, k0, 32);
    wave_sync();
    const int next = r0 + 32 * kWaves;
    if (kAhead && next < rows.hi) {
      qs.load(next);
      gs.load(next);
      learn(next);
    }
    f.step(lds.a[wave], lds.b[wave], LD, lds.table[wave], 0, k0, k0, rule, lane);
    wave_sync();
  }
  add_waves<kWaves>(f.dk, reinterpret_cast<float*>(lds.a), wave, lane);
  add_waves<kWaves>(f.dv, reinterpret_cast<float*>(lds.a), wave, lane);
  if (wave == 0) store_keys<T, DP, EXACT>(p, b, hk, key, f.dk, f.dv, lane);
}

template <class T, int DP, bool EXACT> __global__ void __launch_bounds__(kThreads, 1) mas_attention_dq_few(const AttnParams p) {
  __shared__ __align__(16) FewLds<T, DP> lds;
  const Place at = place_of(p);
  if (!at.idle) few_rows<T, DP, true, EXACT>(p, at, p.tiles, lds);
}

template <class T, int DP, bool EXACT> __global__ void __launch_bounds__(kThreads, 1) mas_attention_dkv(const AttnParams p) {
  __shared__ __align__(16) FewLds<T, DP> lds;
  const Place at = place_of(p);
  if (!at.idle) few_keys<T, DP, false, EXACT>(p, at, lds);
}

// Both at once, the first `split` workgroups for dq, where neither fills the chip.
template <class T, int DP> __global__ void __launch_bounds__(kThreads, 1) mas_attention_few_backward(const AttnParams p, uint32_t split, int row_tiles, int key_tiles) {
  __shared__ __align__(16) FewLds<T, DP> lds;
  const bool by_rows = blockIdx.x < split;
  const Place at = place_of(p, by_rows ? blockIdx.x : blockIdx.x - split, by_rows ? row_tiles : key_tiles);
  if (at.idle) return;
  if (by_rows)
    few_rows<T, DP, false, kExact<T>>(p, at, row_tiles, lds);
  else
    few_keys<T, DP, true, kExact<T>>(p, at, lds);
}

// 16-bit types: 64 keys a workgroup, two waves by keys and two by rows, which
// share tiles of 64 rows; the next tile is on its way while one is used.  Up to 64
// channels two waves fit a SIMD, so that one multiplies while the other takes
// exponents.
template <class T, int DP>
__global__ void __launch_bounds__(kThreads, DP <= 64 ? 2 : 1) mas_attention_dkv_tiles(const AttnParams p) {
  constexpr int LD = kLd<T, DP>, RT = 64;
  __shared__ __align__(16) T tiles[2][2][RT * LD];
  __shared__ __align__(16) RowTable<RT> table[2];
  __shared__ int range[2 * kMaxWaves];
  static_assert(sizeof(tiles) >= 2 * (DP / 32) * 16 * 64 * sizeof(float), "the waves' sums fit");
  const Place at = place_of(p);
  if (at.idle) return;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int by_key = wave % 2, by_row = wave / 2;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int kb0 = 64 * at.tile, k0 = kb0 + 32 * by_key, key = k0 + lane % 32;
  BackwardK<T, DP> f;
  f.start(p, b, hk, key, tk, lane);
  const Interval rows = rows_seeing(p, b, tq, kb0, 64, tk, range);
  const auto rule = score_rule<kExact<T>>(p);
  Stage<T, DP, RT, kThreads, true> qs(p, p.q, b, hk, tq * p.G, tid), gs(p, p.dout, b, hk, tq * p.G, tid);
  RowInfo info;
  const int first = rows.lo / 32 * 32;
  const auto fetch = [&](int r) {
    info.load(p, b, hk, r + tid % RT);
    qs.load(r);
    gs.load(r);
  };
  const auto put = [&](int to) {
    qs.store(tiles[to][0], LD);
    gs.store(tiles[to][1], LD);
    if (tid < RT) table[to].put(tid, info, tk - tq, rows.hi, rule, kb0, 64);
  };
  if (first < rows.hi) {
    fetch(first);
    put(0);
  }
  __syncthreads();
  int cur = 0;
  for (int r0 = first; r0 < rows.hi; r0 += RT, cur ^= 1) {
    const bool more = r0 + RT < rows.hi;
    if (more) fetch(r0 + RT);
    f.step(tiles[cur][0], tiles[cur][1], LD, table[cur], 32 * by_row, kb0, k0, rule, lane);
    if (more) put(cur ^ 1);
    __syncthreads();
  }
  float* sums = reinterpret_cast<float*>(tiles) + by_key * ((DP / 32) * 16 * 64);
  add_waves<2>(f.dk, sums, by_row, lane);
  add_waves<2>(f.dv, sums, by_row, lane);
  if (by_row == 0) store_keys<T, DP, kExact<T>>(p, b, hk, key, f.dk, f.dv, lane);
}

// The same for more than 64 channels, whose two sums do not fit the registers of
// one wave next to another's: two waves share a block of 32 keys by 32 rows.  One
// makes the scores, p and dv; the other, a tile later, takes p (1 - tanh^2) from
// LDS, where it lies lane by lane, makes ds and dk.  So each holds one operand and
// one sum, and while one takes exponents the other, on the same SIMD, multiplies.
// Eight waves: both kinds, two blocks of keys, two of rows; three tiles of 64
// rows: in use by the first kind, by the second, on its way.
template <class T, int DP>
__global__ void __launch_bounds__(2 * kThreads, 2) mas_attention_dkv_pairs(const AttnParams p) {
  constexpr int LD = kLd<T, DP>, RT = 64;
  __shared__ __align__(16) T tiles[3][2][RT * LD];
  __shared__ __align__(16) f32x4 probs[2][4][4][64];
  __shared__ __align__(16) RowTable<RT> table[3];
  __shared__ int range[2 * kMaxWaves];
  static_assert(sizeof(tiles) >= 4 * (DP / 32) * 16 * 64 * sizeof(float), "the waves' sums fit");
  const Place at = place_of(p);
  if (at.idle) return;
  const int b = at.pair / p.Hk, hk = at.pair % p.Hk;
  const int tid = threadIdx.x, lane = tid % 64, half = lane / 32, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int by_key = wave % 2, by_row = wave / 2 % 2, block = wave % 4;
  const bool scores = wave < 4;
  const int tq = clamp_len(p.t_q, b, p.Tq), tk = clamp_len(p.t_k, b, p.Tk);
  const int kb0 = 64 * at.tile, k0 = kb0 + 32 * by_key, key = k0 + lane % 32;
  // The block's keys, or its values.
  frag<T> own[DP / 16];
  {
    const HeadView& v = scores ? p.k : p.v;
    const T* row = head<T>(v, b, hk) + (int64_t)key * v.st;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) own[c] = key < tk ? load_frag(row, 16 * c + 8 * half, p.D, p.vec) : frag<T>(0);
  }
  const Interval rows = rows_seeing(p, b, tq, kb0, 64, tk, range);
  const auto rule = score_rule<kExact<T>>(p);
  // The first kind brings the queries, the second the gradients.
  const HeadView brings = scores ? p.q : p.dout;
  Stage<T, DP, RT, kThreads, true> st(p, brings, b, hk, tq * p.G, tid % kThreads);
  RowInfo info;
  f32x16 sum[DP / 32];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) sum[d] = f32x16(0.0f);
  const int first = rows.lo / 32 * 32, n = (rows.hi - first + RT - 1) / RT;
  const auto fetch = [&](int t) {
    info.load(p, b, hk, first + RT * t + tid % RT);
    st.load(first + RT * t);
  };
  const auto put = [&](int to) {
    st.store(tiles[to][scores ? 0 : 1], LD);
    if (tid < RT) table[to].put(tid, info, tk - tq, rows.hi, rule, kb0, 64);
  };
  if (n > 0) {
    fetch(0);
    put(0);
  }
  __syncthreads();
  int cur = 0;  // the tile of the first kind, modulo 3
  for (int t = 0; t <= n && n > 0; ++t) {
    const int next = cur == 2 ? 0 : cur + 1, last = cur == 0 ? 2 : cur - 1;
    if (t + 1 < n) fetch(t + 1);
    const int mine = scores ? cur : last;
    const RowTable<RT>& tab = table[mine];
    const int i0 = 32 * by_row, i = i0 + 4 * half;
    const bool turn = scores ? t < n : t > 0;
    const int lo = tab.lo[i0 + lane % 32], hi = tab.hi[i0 + lane % 32];
    if (turn && __ballot(lo < k0 + 32 && hi > k0) != 0) {
      f32x4(&pr)[4][64] = probs[(scores ? t : t - 1) & 1][block];
      const T* rt = tiles[mine][scores ? 0 : 1] + i0 * LD;
      f32x16 s(0.0f);
      if (!scores) {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 less = four_at<f32x4>(&tab.less[i + 2 * r]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r + e] = less[e];
        }
      }
      {
        frag<T> x[DP / 16];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) x[c] = rows_frag(rt, LD, 16 * c, lane);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) s = mma(x[c], own[c], s);
      }
      if (scores) {
        f32x16 bend(1.0f);
        if (rule.capped) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] = bent<kExact<T>>(s[r], rule.pre, rule.twice_pre);
            bend[r] = bend_of<kExact<T>>(s[r]);
          }
        }
        tab.add_to(s, i, key - kb0, rule.sloped && __ballot(tab.at[i0 + lane % 32] != INFINITY) != 0, rule);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r]);
        // Rows that see nothing have no statistics: they are masked, not taken for full.
        if (__ballot(lo <= k0 && hi >= k0 + 32) != ~0ull) {
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const i32x4 from = four_at<i32x4>(&tab.lo[i + 2 * r]), to = four_at<i32x4>(&tab.hi[i + 2 * r]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool sees = (key >= from[e]) & (key < to[e]);
              s[r + e] = sees ? s[r + e] : 0.0f;
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 16; r += 4) pr[r / 4][lane] = f32x4{s[r] * bend[r], s[r + 1] * bend[r + 1], s[r + 2] * bend[r + 2], s[r + 3] * bend[r + 3]};
      } else {
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 x = pr[r / 4][lane];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r + e] *= x[e];
        }
      }
      // p in one part, ds in two.
      frag<T> hi[2], lo[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) hi[h] = lo[h] = acc_frag<T>(s, h);
      if (!scores) {
#pragma unroll
        for (int h = 0; h < 2; ++h) lo[h] = Parts<T>(s, h).lo;
      }
      const T* ct = tiles[mine][scores ? 1 : 0] + i0 * LD;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        frag<T> x[DP / 32];
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) x[d] = cols_frag(ct, LD, h, 32 * d, lane);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) sum[d] = mma(x[d], hi[h], sum[d]);
        if (!scores) {
#pragma unroll
          for (int d = 0; d < DP / 32; ++d) sum[d] = mma(x[d], lo[h], sum[d]);
        }
      }
    }
    if (t + 1 < n) put(next);
    __syncthreads();
    cur = next;
  }
  add_waves<2>(sum, reinterpret_cast<float*>(tiles) + (wave / 4 * 2 + by_key) * ((DP / 32) * 16 * 64), by_row, lane);
  if (by_row != 0 || key >= p.Tk) return;
  if (scores)
    store_row<T, DP>(head_out<T>(p.dv, b, hk) + (int64_t)key * p.dv.st, sum, p_unit<kExact<T>>(p), half, p.D, p.vec);
  else
    store_row<T, DP>(head_out<T>(p.dk, b, hk) + (int64_t)key * p.dk.st, sum, p.scale, half, p.D, p.vec);
}

// Workgroups, and how place_of deals them out: over the dies if the last, partly
// used round of eight pairs is a small part.
uint32_t grid_of(AttnParams& p) {
  p.spread = p.pairs % 8 == 0 || p.pairs >= 64;
  return (uint32_t)(p.spread ? (p.pairs + 7) / 8 * 8 : p.pairs) * (uint32_t)p.tiles * (uint32_t)p.splits;
}

// Workgroups of eight waves, 256 rows, with 128 channels of 16 bits, where they fill
// the compute units: tiles are fetched half as often, and a thread holds half as much
// of the next one (4096 causal frames of 8 items and 16 heads 669 -> 655 us, a training
// pass over 4 items and 8 heads 1144 -> 1106; with 64 channels 5 short documents an
// item 177 -> 224).
template <class T, int DP> constexpr bool kWide = sizeof(T) == 2 && DP == 128;
bool wide_rows(int32_t pairs, int32_t rows) { return (int64_t)((rows + 255) / 256) * pairs >= 256; }

// Caps for which 16-bit types have kernels of their own (see bent).
template <class T> bool exact_caps(const AttnParams& p) { return sizeof(T) == 2 && p.cap > kHalfCap; }

template <class T, int DP, bool EXACT> hipError_t forward_keys(const AttnParams& p, uint32_t grid, hipStream_t stream) {
  hipLaunchKernelGGL((mas_attention_keys<T, DP, EXACT>), dim3(grid), dim3(kThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const uint64_t rows = (uint64_t)p.pairs * p.rows;
  hipLaunchKernelGGL((mas_attention_join<T, EXACT>), dim3((uint32_t)((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <class T, int DP> hipError_t forward(AttnParams p, const AttnPlan& plan, hipStream_t stream) {
  const uint32_t grid = grid_of(p);
  if (!plan.small) {
    if constexpr (kWide<T, DP>) {
      if (plan.waves == 8) {
        hipLaunchKernelGGL((mas_attention_rows<T, DP, 8>), dim3(grid), dim3(512), 0, stream, p);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((mas_attention_rows<T, DP, 4>), dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
  }
  return exact_caps<T>(p) ? forward_keys<T, DP, true>(p, grid, stream) : forward_keys<T, DP, kExact<T>>(p, grid, stream);
}

template <class T, int DP, bool EXACT> hipError_t backward_few(AttnParams p, hipStream_t stream) {
  p.tiles = (p.rows + 31) / 32;
  hipLaunchKernelGGL((mas_attention_dq_few<T, DP, EXACT>), dim3(grid_of(p)), dim3(kThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  p.tiles = (p.Tk + 31) / 32;
  hipLaunchKernelGGL((mas_attention_dkv<T, DP, EXACT>), dim3(grid_of(p)), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <class T, int DP> hipError_t backward(AttnParams p, hipStream_t stream) {
  p.splits = 1;
  if (exact_caps<T>(p)) return backward_few<T, DP, true>(p, stream);
  // 128 rows a workgroup where those fill the 256 compute units, else 32 (1024 keys of
  // 64 channels, bf16, with dk, dv: 128 workgroups 53.4 / 44.4 us, 256 60.5 / 62.8).
  p.tiles = (p.rows + 127) / 128;
  const bool few_rows = (int64_t)p.tiles * p.pairs < 256;
  const bool wide = kWide<T, DP> && wide_rows(p.pairs, p.rows);
  // 64 keys a workgroup where those fill the compute units, else 32 (512 keys of 64
  // channels, bf16, with dq: 128 workgroups of 64 keys 28.3 / 25.4 us, 256 30.9 / 38.4).
  const int key_tiles = (p.Tk + 63) / 64;
  const bool few_keys = sizeof(T) == 4 || (int64_t)key_tiles * p.pairs < 256;
  // One launch where the workgroups of both find a compute unit of their own, else one
  // after the other (256 workgroups against two launches of 128: 64 channels bf16 18.6 /
  // 22.4 us, 96 channels fp32 26.8 / 36.0; 512 against 256 and 256: 27.2 / 22.7, 42.5 / 36.8).
  if (few_rows && few_keys) {
    const int rows = (p.rows + 31) / 32, keys = (p.Tk + 31) / 32;
    p.tiles = rows;
    const uint32_t split = grid_of(p);
    p.tiles = keys;
    const uint32_t both = split + grid_of(p);
    if (both <= 256) {
      hipLaunchKernelGGL((mas_attention_few_backward<T, DP>), dim3(both), dim3(kThreads), 0, stream, p, split, rows, keys);
      return hipGetLastError();
    }
    p.tiles = (p.rows + 127) / 128;
  }
  if (few_rows) p.tiles = (p.rows + 31) / 32;
  if (wide) p.tiles = (p.rows + 255) / 256;
  uint32_t grid = grid_of(p);
  if (few_rows) {
    hipLaunchKernelGGL((mas_attention_dq_few<T, DP, kExact<T>>), dim3(grid), dim3(kThreads), 0, stream, p);
  } else if (!wide) {
    hipLaunchKernelGGL((mas_attention_dq<T, DP, 4>), dim3(grid), dim3(256), 0, stream, p);
  } else {
    if constexpr (kWide<T, DP>) hipLaunchKernelGGL((mas_attention_dq<T, DP, 8>), dim3(grid), dim3(512), 0, stream, p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if constexpr (sizeof(T) == 2) {
    if (!few_keys) {
      p.tiles = key_tiles;
      grid = grid_of(p);
      if constexpr (DP > 64)
        hipLaunchKernelGGL((mas_attention_dkv_pairs<T, DP>), dim3(grid), dim3(2 * kThreads), 0, stream, p);
      else
        hipLaunchKernelGGL((mas_attention_dkv_tiles<T, DP>), dim3(grid), dim3(kThreads), 0, stream, p);
      return hipGetLastError();
    }
  }
  p.tiles = (p.Tk + 31) / 32;
  grid = grid_of(p);
  hipLaunchKernelGGL((mas_attention_dkv<T, DP, kExact<T>>), dim3(grid), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

template <class T, class F> hipError_t by_width(int D, F&& f) {
  if (D <= 32) return f(std::integral_constant<int, 32>());
  if (D <= 64) return f(std::integral_constant<int, 64>());
  if (D <= 96) return f(std::integral_constant<int, 96>());
  return f(std::integral_constant<int, 128>());
}

}  // namespace

AttnPlan attention_plan(int32_t pairs, int32_t rows, int32_t Tk, int32_t D, bool fp32, float cap) {
  AttnPlan a;
  a.waves = 4;
  a.splits = 1;
  a.span = Tk;
  a.tiles = (rows + 127) / 128;
  // Workgroups of 128 rows where they fill the compute units (256; from half of them
  // on with more than 64 channels in 16 bits, where those of 32 rows fit a unit only
  // once), else of 32 rows whose waves share the keys.  Measured, 128 / 32 rows, causal,
  // 512 keys of 64 channels, bf16: 128 workgroups 16.0 / 13.0 us, 256 16.3 / 21.6; 1024
  // keys 24.9 / 17.9 and 25.2 / 26.6; 128 channels, 512 keys, 128 workgroups 23.1 / 29.2,
  // 1024 keys, 32 workgroups 35.7 / 23.1; fp32, 512 keys of 64 channels, 128 workgroups
  // 45.2 / 29.2, 256 49.4 / 49.1.  Up to 32 rows always the latter (64 caches of 4096
  // keys, 4 heads: 128 / 43; 512 of 1024 keys 25.7 / 26.1; 2048 of 256 keys 32.3 / 37.6).
  a.small = rows <= 32 || (int64_t)a.tiles * pairs < (fp32 || D <= 64 ? 256 : 128);
  if (!a.small && !fp32 && cap > kHalfCap) {  // keys in one part: the workspace does not depend on the cap
    a.small = true;
    a.tiles = (rows + 31) / 32;
    return a;
  }
  if (!a.small) {
    if (!fp32 && D > 96 && wide_rows(pairs, rows)) {
      a.waves = 8;
      a.tiles = (rows + 255) / 256;
    }
    return a;
  }
  a.tiles = (rows + 31) / 32;
  // The keys are split until two workgroups a compute unit are there, into parts of at
  // least 512, four blocks a wave; steps over more than 1024 keys into parts of 128.
  // Measured with 128 / 512 at least: a step over 2048 keys 16.3 / 20.7 us, over 1024
  // keys 15.0 / 15.9; 64 workgroups of 32 rows by 512 keys 13.6 / 10.9 (the second
  // kernel, which joins the parts, takes 5).
  const int least = rows <= 32 && Tk > 1024 ? 128 : 512;
  const int64_t groups = (int64_t)a.tiles * pairs;
  int64_t want = (512 + groups - 1) / groups;
  const int64_t most = (Tk + least - 1) / least;
  if (want > most) want = most;
  a.span = (int32_t)(((Tk + want - 1) / want + 127) / 128 * 128);
  a.splits = (Tk + a.span - 1) / a.span;
  return a;
}

size_t attention_part_bytes(const AttnPlan& a, int32_t pairs, int32_t D) {
  return a.splits > 1 ? (size_t)a.splits * pairs * 32 * a.tiles * (D + 2) * sizeof(float) : 0;
}

hipError_t launch_attention(AttnParams p, int dtype, const AttnPlan& plan, hipStream_t stream) {
  p.tiles = plan.tiles;
  p.splits = plan.splits;
  p.span = plan.span;
  const auto go = [&](auto t) {
    using T = decltype(t);
    return by_width<T>(p.D, [&](auto dp) { return forward<T, decltype(dp)::value>(p, plan, stream); });
  };
  if (dtype == kF32) return go(0.0f);
  if (dtype == kF16) return go((_Float16)0.0f);
  return go((__bf16)0.0f);
}

hipError_t launch_attention_backward(AttnParams p, int dtype, hipStream_t stream) {
  const auto go = [&](auto t) {
    using T = decltype(t);
    return by_width<T>(p.D, [&](auto dp) { return backward<T, decltype(dp)::value>(p, stream); });
  };
  if (dtype == kF32) return go(0.0f);
  if (dtype == kF16) return go((_Float16)0.0f);
  return go((__bf16)0.0f);
}

}  // namespace mas
