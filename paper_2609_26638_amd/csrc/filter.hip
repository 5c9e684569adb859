// sample_filtered and accept_sampled: tokens drawn from softmax(z / T) cut by
// top-k, top-p and min-p, and acceptance-rejection of drafted tokens over such
// distributions (Preliminaries, "Speculative Decoding").  Every random number
// is an input.
//
// The tokens of a row are ordered by (logit descending, index ascending); each
// filter keeps a prefix of that order, so the kept set is
//   z > cut.z, or z == cut.z and index <= cut.idx,   and weight >= min_p,
// with weight w = exp((z - max z) / T) in 64 bits: the running sums of a
// vocabulary of 65536 are compared with u * total at every token, and sums of
// 32-bit weights (1e-7 relative) would draw a neighbour for one row in a few
// hundred.  (A 64-bit FMA takes 4.3 cycles per wave, a 32-bit one 2.7.)
//
// One workgroup per row (RowFilter).  Wave w owns one contiguous range of
// the row, so the ranges' sums are in index order.
//   1. one pass: the maximum; where the whole weight is needed, it too, each
//      thread's sum relative to its own running maximum; and each thread's
//      maxima over PARTS parts of its logits;
//   2. a logit that no kept token lies below (parts_bound).  The parts' maxima
//      are tokens: where their count reaches k, the row's does.  For top-p
//      they are a sample: one of s tokens that a share q of the parts exceeds
//      stands for (1 - q)^(1/s - 1) tokens (a share x of all tokens exceeds it,
//      (1 - x)^s = 1 - q, and (1 - x)^(s - 1) of its like are maxima), and
//      where the weights so counted reach a little more than the share p, the
//      cut is likely above, which step 3 checks;
//   3. a second pass: the tokens from there up, as a list in LDS, and whether
//      they do weigh the share p (otherwise, and where the list overflows,
//      again from a bound that is sure: tokens of less than (1 - p) / V of the
//      weight each, or row_bound);
//   4. up to SMALL of them (a longer list is first cut short by a histogram)
//      are ranked against each other, which gives the cut, the kept weight and
//      the draw at once (filter_small).
// Longer lists (filter_list) take histograms with a count and a weight sum per
// bin, narrowed to the tokens of one wave (select_cut), and draw by the kept
// weight per index.  Rows whose candidates do not fit a list: flat ones of top-p
// add up what lies above a window around the cut (filter_flat); a large k and
// many equal logits take the histograms over the row (filter_row_again).
//
// A pass is a rolled loop that reads the row again, from L2 mostly: code that is
// run once per launch is bound by fetching its instructions (16 KB of unrolled
// passes over a row held in registers took 16,000 cycles for what the loop does
// in 10,000), so the rest is kept small, and out of line where it is rare.
// Weights that atomics or an unordered list add up are fixed-point integers,
// whose sums do not depend on the order; the other sums have a fixed order.
// Results do not depend on timing, nor on the other rows of the call (the
// number of rows may choose another order of the 64-bit sums).
//
// What bounds it, at V = 65536 f32, in cycles of 65,000 (n of 80) to 105,000
// (n of 7500): the first pass 31,000 where it sums weights (21,000 of them the
// 64-bit exponentials), 10,000 where it does not; the bound 9,000; the second
// pass 12,000 to 19,000 (the rows of an XCD's CUs together exceed its L2); then
// 12,000 for a short list, which is barriers and LDS latency, up to 45,000 for a
// long one.  136 such rows: 49 us, 0.73 TB/s of logits read once; 1024 rows of
// bf16 with top-k, two to a CU: 67 us, 2.0 TB/s.
#include <float.h>
#include <math.h>

#include "dvs_common.h"

namespace dvs {

#define NOINLINE __attribute__((noinline))

constexpr int RANK = 64;          // tokens that one wave ranks
constexpr int SMALL = 256;        // tokens that the workgroup ranks
constexpr int PARTS = 8;          // parts of a thread's logits
constexpr int BATCH = 16;         // logits that a thread has in flight
constexpr double LIST_SCALE = 281474976710656.0;   // 2^48: a list's weights stay below 2^63

// What a row's filters keep: weight >= min_w of the tokens with z > cut.z, or
// z == cut.z and index <= cut.idx.
struct RowCut {
  float zmax, z;     // largest logit; the cut's
  int idx;           // the cut's index among equal logits
  float min_w;       // min_p
  double log2e_t;    // log2(e) / T
  double total;      // kept weight
  double inv_total;  // 1 / total (accept_sampled)
  int single;        // 1: only token idx is kept (weight 1); -1: no token
};

// What a histogram over all the tokens has found: the bin of the cut, its
// tokens, and the count and weight above it.  bin < 0: nothing yet.
struct Found {
  int bin, n;
  uint32_t above_c;
  unsigned long long above_m;
};

// 2^(d c) for -1021 < d c <= 0: 2^n (1 + f P(f)), d c = n + f, |f| <= 1/2.  P
// interpolates (2^f - 1) / f at Chebyshev nodes: 3.7e-14 relative.
__device__ __forceinline__ double exp2_normal(double d, double c) {
  const double shift = 6755399441055744.0;     // 1.5 * 2^52: n in the low word
  const double s = fma(d, c, shift);
  const double f = fma(d, c, shift - s);
  double q = 1.02031210633917290e-07;
  q = fma(q, f, 1.32552248786688168e-06);
  q = fma(q, f, 1.52526868462677196e-05);
  q = fma(q, f, 1.54034558524538382e-04);
  q = fma(q, f, 1.33335581790431116e-03);
  q = fma(q, f, 9.61812915940255843e-03);
  q = fma(q, f, 5.55041086647604237e-02);
  q = fma(q, f, 2.40226506958129887e-01);
  q = fma(q, f, 6.93147180559945286e-01);
  q = fma(q, f, 1.0);
  return __hiloint2double(__double2hiint(q) + (__double2loint(s) << 20), __double2loint(q));
}

// The same for every d <= 0, 0 for d c below -1021, -inf and NaN (a masked
// logit, or one that is not a number).
__device__ __forceinline__ double exp2_neg(double d, double c) {
  const double w = exp2_normal(d, c);
  return d * c > -1021.0 ? w : 0.0;
}

// exp((z - zmax) / T), zmax finite.
__device__ __forceinline__ double weight(float z, const RowCut& c) {
  return exp2_neg((double)z - (double)c.zmax, c.log2e_t);
}

__device__ __forceinline__ bool before_cut(float z, int idx, const RowCut& c) {
  return z > c.z || (z == c.z && idx <= c.idx);
}

// Weight of a token, 0 if it is not kept.
__device__ __forceinline__ double kept_weight(float z, int idx, const RowCut& c) {
  if (!before_cut(z, idx, c)) return 0.0;
  const double w = weight(z, c);
  return w >= (double)c.min_w ? w : 0.0;
}

__device__ __forceinline__ float load_logit(const float* p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t* p) { return bf16_bits_to_f32(*p); }

// Order-preserving key of a number (-0 as +0).
__device__ __forceinline__ uint32_t order_key(float z) {
  uint32_t u = __float_as_uint(z);
  if ((u & 0x7fffffffu) == 0) u = 0;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// 16 bytes at the alignment of an element (a row may start on any).
typedef uint32_t u32x4_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_b16 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ u32x4 load_vec(const float* p) { return *(const u32x4_f32*)p; }
__device__ __forceinline__ u32x4 load_vec(const uint16_t* p) { return *(const u32x4_b16*)p; }

template <typename E>
__device__ __forceinline__ float vec_elem(const u32x4& x, int e);
template <typename E>
__device__ __forceinline__ float vec_max(const u32x4& x) {
  float m = vec_elem<E>(x, 0);
#pragma unroll
  for (int e = 1; e < 16 / (int)sizeof(E); ++e) m = fmaxf(m, vec_elem<E>(x, e));
  return m;
}
template <typename E>
__device__ __forceinline__ float vec_elem(const u32x4& x, int e) {
  if constexpr (sizeof(E) == 2)
    return __uint_as_float((e & 1) ? (x[e >> 1] & 0xffff0000u) : (x[e >> 1] << 16));
  else
    return __uint_as_float(x[e]);
}

typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));

// A value that every thread of the workgroup has, in scalar registers: what
// branches on it is then no divergent branch, whose both sides would keep
// their registers.
__device__ __forceinline__ float uniform(float v) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ double uniform(double v) {
  return __hiloint2double(uniform(__double2hiint(v)), uniform(__double2loint(v)));
}

// v of the lane that CTRL names in this lane's row of 16 (or a row's last lane
// for the broadcasts), `old` where there is none: one vector move, where a
// general shuffle takes a round trip through LDS.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T dpp(T old, T v) {
  if constexpr (sizeof(T) == 4) {
    const int r = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old),
                                              __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, r);
  } else {
    const unsigned long long o = __builtin_bit_cast(unsigned long long, old);
    const unsigned long long x = __builtin_bit_cast(unsigned long long, v);
    const uint32_t lo = dpp<CTRL, ROWS>((uint32_t)o, (uint32_t)x);
    const uint32_t hi = dpp<CTRL, ROWS>((uint32_t)(o >> 32), (uint32_t)(x >> 32));
    return __builtin_bit_cast(T, ((unsigned long long)hi << 32) | lo);
  }
}
template <typename T>
__device__ __forceinline__ T at_lane(T v, int lane) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const unsigned long long x = __builtin_bit_cast(unsigned long long, v);
    const uint32_t lo = at_lane((uint32_t)x, lane), hi = at_lane((uint32_t)(x >> 32), lane);
    return __builtin_bit_cast(T, ((unsigned long long)hi << 32) | lo);
  }
}
struct Add {
  template <typename T>
  __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
  __device__ __forceinline__ int operator()(int a, int b) const { return max(a, b); }
};
struct Min {
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
  __device__ __forceinline__ int operator()(int a, int b) const { return min(a, b); }
};
// Inclusive scan over each row of 16 lanes, and over the wave.  none: op's
// neutral value.
template <typename T, typename Op>
__device__ __forceinline__ T row_scan(T v, T none, Op op) {
  v = op(dpp<0x111, 0xf>(none, v), v);         // row_shr:1, 2, 4, 8
  v = op(dpp<0x112, 0xf>(none, v), v);
  v = op(dpp<0x114, 0xf>(none, v), v);
  v = op(dpp<0x118, 0xf>(none, v), v);
  return v;
}
template <typename T, typename Op>
__device__ __forceinline__ T wave_scan(T v, T none, Op op) {
  v = row_scan(v, none, op);
  v = op(dpp<0x142, 0xa>(none, v), v);         // row_bcast:15 into rows 1 and 3
  v = op(dpp<0x143, 0xc>(none, v), v);         // row_bcast:31 into rows 2 and 3
  return v;
}

struct Cut {
  float z;
  int idx;
  unsigned long long mass;   // fixed-point weight through the cut
};

__device__ __forceinline__ unsigned long long fixed_weight(float z, const RowCut& c, double scale) {
  return (unsigned long long)(weight(z, c) * scale + 0.5);
}

// Scale of weights that integers add up: base, whose sums stay below 2^63 by the
// number of the tokens, or more where these weigh `whole` at most (< 0: not
// known).  Each weight is rounded by half a unit, so a sum over 2^22 of them is
// off by 2^-40 of the whole at most; by 2^-18 of the largest weight with the
// base alone, where 4 million tokens of 2^-40 each would count as nothing.
__device__ __forceinline__ double mass_scale(double base, double whole) {
  return whole > 0.0 ? fmax(base, ldexp(1.0, 61 - ilogb(whole))) : base;
}

// A logit such that exp((z - hi) / T) is below w for every smaller one,
// whatever the roundings on the way.
__device__ __forceinline__ float weight_bound(float hi, double T, double w) {
  // (the largest: also for T infinite, whose products may be no number)
  return fmaxf((float)((double)hi + T * (log(w) * (1.0 + 1e-6) - 1e-9)) - fabsf(hi) * 1e-6f,
               -FLT_MAX);
}

// A row by a workgroup of FT threads: 1024 (one workgroup per CU) or 512 (two
// per CU, so that the latencies of one row run under the passes of the other).
template <int FT>
struct RowFilter {

static constexpr int FW = FT / 64;
static constexpr int BINS = FT, BIN_BITS = FT == 1024 ? 10 : 9;   // one bin per thread
static constexpr int LIST = 16 * FT;   // candidates held in LDS (128 KB or 64 KB)

struct FilterShared {
  uint32_t cnt[BINS];
  unsigned long long mass[BINS > 3 * SMALL ? BINS : 3 * SMALL];
  float lz[LIST];
  int li[LIST];
  double d[FW];
  unsigned long long u[FW];
  uint32_t c[FW];
  float f[FW], g[FW];
  int i[FW];
  int found, n, token;
  uint32_t fc;
  unsigned long long fm;
  double w;
  RowCut rc;
  Found so_far;
  float lo, hi;
  int inside;
};

// The workgroup's LDS, for the functions that are kept out of line too.
static __device__ __forceinline__ FilterShared& shared() {
  __shared__ FilterShared sh;
  return sh;
}

// A row of V logits: 16-byte vectors, wave w with the nit * 64 vectors of its
// range lane by lane, and the V % EPV last logits with the last wave.  A pass
// has BATCH logits in flight; absent ones are -inf.
template <typename E>
struct Row {
  static constexpr int EPV = 16 / sizeof(E), AHEAD = BATCH / EPV;
  const E* p;
  int V, nit, base;

  __device__ __forceinline__ Row(const E* p_, int V_, int nit_) : p(p_), V(V_), nit(nit_) {
    base = ((threadIdx.x >> 6) * nit * 64 + (threadIdx.x & 63)) * EPV;
  }
  __device__ __forceinline__ int at(int it) const { return base + it * 64 * EPV; }
  // A batch of AHEAD vectors.  No branches: a wait for each load would stand in
  // them.  (The first vector stands in for absent ones; a pass begins a batch
  // only if there is one.)
  __device__ __forceinline__ u32x16 batch(int it) const {
    const uint32_t none = sizeof(E) == 2 ? 0xff80ff80u : 0xff800000u;
    u32x4 x[AHEAD];
    bool there[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = at(it + k);
      there[k] = it + k < nit && i + EPV <= V;
      x[k] = load_vec(p + (there[k] ? i : 0));
    }
    u32x16 b;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
#pragma unroll
      for (int d = 0; d < 4; ++d) b[4 * k + d] = there[k] ? x[k][d] : none;
    return b;
  }
  // vector k of a batch (k uniform: indexed registers)
  static __device__ __forceinline__ u32x4 vec(const u32x16& b, int k) {
    return u32x4{b[4 * k], b[4 * k + 1], b[4 * k + 2], b[4 * k + 3]};
  }
  // logit e of a batch (e constant)
  static __device__ __forceinline__ float logit(const u32x16& b, int e) {
    return vec_elem<E>(vec(b, e / EPV), e % EPV);
  }
  // The logit behind the last vector that this thread has, or -1.
  __device__ __forceinline__ int rest_index() const {
    const int i = V / EPV * EPV + (int)threadIdx.x - (FT - 64);
    return (int)threadIdx.x >= FT - 64 && i < V ? i : -1;
  }
  // f(batch, number of its first vector)
  template <typename F>
  __device__ __forceinline__ void batches(F f) const {
#pragma unroll 1
    for (int it = 0; it < nit; it += AHEAD) f(batch(it), it);
  }
  // f(z, index) for every token.  A vector that is absent has an index past the
  // whole ones, which the tokens behind them have too.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    batches([&](const u32x16& b, int it) {
#pragma unroll 1
      for (int k = 0; k < min(AHEAD, nit - it); ++k) {
        const u32x4 x = vec(b, k);
        const int first = at(it + k);
        if (first + EPV <= V) {
#pragma unroll
          for (int e = 0; e < EPV; ++e) f(vec_elem<E>(x, e), first + e);
        }
      }
    });
    const int i = rest_index();
    if (i >= 0) f(load_logit(p + i), i);
  }
  // f(z, index) where some lane's vector reaches zlo; f decides by itself.  Absent
  // tokens come as -inf with index V (a branch around them: 136 rows of 65536
  // with min-p 25.1 -> 27.0 us).
  template <typename F>
  __device__ __forceinline__ void each_from(float zlo, F f) const {
    batches([&](const u32x16& b, int it) {
      float m = -INFINITY;
#pragma unroll
      for (int e = 0; e < BATCH; ++e) m = fmaxf(m, logit(b, e));
      if (!__ballot(m >= zlo)) return;
#pragma unroll 1
      for (int k = 0; k < min(AHEAD, nit - it); ++k) {
        const u32x4 x = vec(b, k);
        if (__ballot(vec_max<E>(x) >= zlo)) {
          const int first = at(it + k) + EPV <= V ? at(it + k) : V;
#pragma unroll
          for (int e = 0; e < EPV; ++e) f(vec_elem<E>(x, e), first + e);
        }
      }
    });
    const int i = rest_index();
    if (i >= 0) f(load_logit(p + i), i);
  }
};

// The n candidates in LDS.
struct List {
  int n;
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    const FilterShared& sh = shared();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += FT) f(sh.lz[i], sh.li[i]);
  }
};

  // -- over the workgroup

// v over the workgroup, in scalar registers; buf: FW values in LDS.
template <typename T, typename Op>
static __device__ __forceinline__ T block_reduce(T v, T none, Op op, T* buf) {
  const int lane = threadIdx.x & 63, wv = uniform((int)threadIdx.x >> 6);
  v = wave_scan(v, none, op);
  if (lane == 63) buf[wv] = v;
  __syncthreads();
  v = row_scan(lane < FW ? buf[lane] : none, none, op);
  __syncthreads();
  return at_lane(v, FW - 1);
}

static __device__ __forceinline__ void block_max_min(float& hi, float& lo) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, wv = uniform((int)threadIdx.x >> 6);
  hi = wave_scan(hi, -INFINITY, Max());
  lo = wave_scan(lo, INFINITY, Min());
  if (lane == 63) { sh.f[wv] = hi; sh.g[wv] = lo; }
  __syncthreads();
  hi = at_lane(row_scan(lane < FW ? sh.f[lane] : -INFINITY, -INFINITY, Max()), FW - 1);
  lo = at_lane(row_scan(lane < FW ? sh.g[lane] : INFINITY, INFINITY, Min()), FW - 1);
  __syncthreads();
}

// Inclusive scan over the workgroup of (count, mass), in thread order.
static __device__ __forceinline__ void scan_bins(uint32_t& c, unsigned long long& m) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, wv = uniform((int)threadIdx.x >> 6);
  c = wave_scan(c, 0u, Add());
  m = wave_scan(m, 0ull, Add());
  if (lane == 63) { sh.c[wv] = c; sh.u[wv] = m; }
  __syncthreads();
  const uint32_t bc = row_scan(lane < FW ? sh.c[lane] : 0u, 0u, Add());
  const unsigned long long bm = row_scan(lane < FW ? sh.u[lane] : 0ull, 0ull, Add());
  if (wv) {
    c += at_lane(bc, wv - 1);
    m += at_lane(bm, wv - 1);
  }
  __syncthreads();
}

// Smallest index of a thread for which `yes` holds, `none` without one.
static __device__ __forceinline__ int first_index(bool yes, int i, int none) {
  const int got = block_reduce(yes ? i : 0x7fffffff, 0x7fffffff, Min(), shared().i);
  return got == 0x7fffffff ? none : got;
}

// Smallest index whose running weight (index order) exceeds t, given each
// wave's range sum in sh.d; the last index of positive weight when rounding
// (or u = 1) puts t past the sum; -1 when every weight is zero.  fn(z, i) is
// the weight of token i.
template <typename E, typename F>
static __device__ __forceinline__ int pick_index(const Row<E>& row, F fn, double t) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const double own = lane < FW ? sh.d[lane] : 0.0;
  const double runs = row_scan(own, 0.0, Add());
  const unsigned long long some = __ballot(own > 0.0);
  if (!some) return -1;
  const unsigned long long over = __ballot(own > 0.0 && runs > t);
  const int w = over ? __ffsll((long long)over) - 1 : 63 - __clzll((long long)some);
  const double excl = w ? at_lane(runs, w - 1) : 0.0;
  if (!over) t = INFINITY;
  // the range's tokens in whole vectors per thread
  constexpr int EPV = Row<E>::EPV;
  const int span = row.nit * 64 * EPV, lo = min(w * span, row.V / EPV * EPV);
  const int hi = w == FW - 1 ? row.V : min(row.V / EPV * EPV, lo + span);
  const int per = ((hi - lo + FT - 1) / FT + EPV - 1) / EPV * EPV;
  const int first = lo + tid * per;
  double part = 0.0;
  int lastpos = -1;
  auto walk = [&](auto&& f) {            // this thread's tokens, in index order
#pragma unroll 4
    for (int i = first; i < min(hi, first + per); ++i) f(fn(load_logit(row.p + i), i), i);
  };
  walk([&](double x, int i) {
    part += x;
    if (x > 0.0) lastpos = i;
  });
  const double incl = wave_scan(part, 0.0, Add());
  const double before = dpp<0x138, 0xf>(0.0, incl);   // the lane before's
  __syncthreads();                       // sh.d has been read by every thread
  if (lane == 63) sh.d[wv] = incl;
  __syncthreads();
  const double waves = row_scan(lane < FW ? sh.d[lane] : 0.0, 0.0, Add());
  double base = excl;
  if (wv) base += at_lane(waves, wv - 1);
  int at = 0x7fffffff;
  if (part > 0.0 && base + incl > t) {   // the first such thread holds the token
    double acc = base + before;
    at = lastpos;
    walk([&](double x, int i) {
      acc += x;
      if (acc > t) at = min(at, i);
    });
  }
  at = first_index(at != 0x7fffffff, at, -1);
  return at >= 0 ? at : block_reduce(lastpos, -1, Max(), sh.i);
}

// The tokens for which in(z) holds (not for -inf), as a list in LDS if at most
// LIST; returns how many they are.  each(z): called for all of the row (-inf for
// absent ones).
template <typename E, typename I, typename F>
static __device__ __forceinline__ int gather(const Row<E>& row, I in, F each) {
  FilterShared& sh = shared();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  row.batches([&](const u32x16& b, int it) {
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < BATCH; ++e) {
      const float z = Row<E>::logit(b, e);
      each(z);
      c += in(z);
    }
    if (!__ballot(c)) return;
    const uint32_t incl = wave_scan(c, 0u, Add());   // a place for each, one count-in per wave
    int at = 0;
    if ((threadIdx.x & 63) == 63) at = atomicAdd(&sh.n, (int)incl);
    at = at_lane(at, 63) + (int)(incl - c);
    constexpr int EPV = Row<E>::EPV;
#pragma unroll
    for (int e = 0; e < BATCH; ++e) {
      const float z = Row<E>::logit(b, e);
      if (in(z)) {
        if (at < LIST) { sh.lz[at] = z; sh.li[at] = row.at(it + e / EPV) + e % EPV; }
        ++at;
      }
    }
  });
  const int ri = row.rest_index();
  if (ri >= 0) {
    const float z = load_logit(row.p + ri);
    each(z);
    if (in(z)) {
      const int at = atomicAdd(&sh.n, 1);
      if (at < LIST) { sh.lz[at] = z; sh.li[at] = ri; }
    }
  }
  __syncthreads();
  const int n = uniform(sh.n);
  __syncthreads();
  return n;
}
// The tokens from `lo` up.
template <typename E>
static __device__ __forceinline__ int gather(const Row<E>& row, float lo) {
  return gather(row, [=](float z) { return z >= lo; }, [](float) {});
}

// Every wave's range sum to sh.d; returns their sum, in order.
static __device__ __forceinline__ double range_sums(double part) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, wv = uniform((int)threadIdx.x >> 6);
  part = wave_scan(part, 0.0, Add());
  __syncthreads();
  if (lane == 63) sh.d[wv] = part;
  __syncthreads();
  return at_lane(row_scan(lane < FW ? sh.d[lane] : 0.0, 0.0, Add()), FW - 1);
}

  // -- the cut

// Bins over [zlo, zhi], the largest logits first: linear ones, which spread a
// row's logits well, or ones of the numbers' ordered keys, which end at single
// values whatever the spread.
struct Binning {
  float half, sc, width;   // half the largest logit, bins per half a unit, half a bin
  uint32_t khi;
  int shift;
  bool linear;
  __device__ __forceinline__ Binning(float zhi, float zlo, bool lin) : linear(lin) {
    half = zhi * 0.5f;
    width = fmaxf((half - zlo * 0.5f) * (1.0f / BINS), 1e-36f);
    sc = __builtin_amdgcn_rcpf(width);
    khi = order_key(zhi);
    shift = max(0, 32 - BIN_BITS - __clz(khi - order_key(zlo)));
  }
  __device__ __forceinline__ int operator()(float z) const {
    if (linear) return (int)fminf((half - z * 0.5f) * sc, (float)(BINS - 1));
    return (int)((khi - order_key(z)) >> shift);
  }
  // a logit that none of the bins up to b lies below
  __device__ __forceinline__ float lower_edge(int b) const {
    if (linear) {
      const double edge = 2.0 * ((double)half - (b + 1) * (double)width);
      return (float)fmax(edge - 1e-6 * (fabs(edge) + 2.0 * fabs((double)half)), -(double)FLT_MAX);
    }
    const unsigned long long down = ((unsigned long long)(b + 1) << shift) - 1;
    const uint32_t key = down < khi ? khi - (uint32_t)down : 0u;
    return fmaxf(__uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key), -FLT_MAX);
  }
};

// The r-th lowest index (r >= 1) whose logit equals z.
template <typename E>
static __device__ NOINLINE int nth_equal(const E* p, int V, int nit, float z, int r) {
  const Row<E> row(p, V, nit);
  auto one = [&](float x, int) { return x == z ? 1.0 : 0.0; };
  double part = 0.0;
  row.each([&](float x, int i) { part += one(x, i); });
  range_sums(part);
  return pick_index(row, one, (double)r - 0.5);
}

// The last token kept when the tokens of `src` with zlo <= z <= zhi (n of
// them, in order) are kept up to the k-th (by_mass false), or up to the first
// at which the weight reaches `target` (by_mass true; the last one if none
// does).  Weights are summed only when `masses` is set.  `row`: where equal
// logits are counted in index order.
template <typename Src, typename E>
static __device__ __forceinline__ Cut select_cut(const Src& src, const Row<E>& row, const RowCut& rc,
                                          double scale, int n, float zhi, float zlo, bool by_mass,
                                          bool masses, uint32_t k, double target, Found so_far) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x;
  uint32_t above_c = so_far.above_c;
  unsigned long long above_m = so_far.above_m;
  int at_bin = so_far.bin;               // the bin looked at; -1: all of [zlo, zhi]
  if (at_bin >= 0) n = so_far.n;
  Binning bin(zhi, zlo, true);
  auto in = [&](float z) { return z <= zhi && z >= zlo && (at_bin < 0 || bin(z) == at_bin); };
  for (int level = at_bin >= 0; n > RANK; ++level) {
    if (at_bin >= 0) {
      float lo = INFINITY, hi = -INFINITY;
      src.each([&](float z, int) {
        if (in(z)) { lo = fminf(lo, z); hi = fmaxf(hi, z); }
      });
      zlo = block_reduce(lo, INFINITY, Min(), sh.f);
      zhi = block_reduce(hi, -INFINITY, Max(), sh.f);
      at_bin = -1;
    }
    if (zlo == zhi) break;
    bin = Binning(zhi, zlo, level == 0);
    sh.cnt[tid] = 0;
    sh.mass[tid] = 0;
    __syncthreads();
    src.each([&](float z, int) {
      if (z <= zhi && z >= zlo) {
        const int b = bin(z);
        atomicAdd(&sh.cnt[b], 1u);
        if (masses) atomicAdd(&sh.mass[b], fixed_weight(z, rc, scale));
      }
    });
    __syncthreads();
    const uint32_t own_c = sh.cnt[tid];
    uint32_t c = own_c;
    unsigned long long m = sh.mass[tid];
    const unsigned long long own_m = m;
    scan_bins(c, m);
    const bool here = by_mass ? (double)(above_m + m) >= target : above_c + c >= k;
    int b = first_index(own_c && here, tid, -1);
    if (b < 0) b = BINS - 1 - first_index(own_c > 0, BINS - 1 - tid, 0);   // the last bin
    if (tid == b) { sh.n = (int)own_c; sh.fc = c - own_c; sh.fm = m - own_m; }
    __syncthreads();
    n = uniform(sh.n);
    above_c += sh.fc;
    above_m += sh.fm;
    at_bin = b;
  }
  Cut cut;
  if (n > RANK) {                        // equal logits: in index order
    const unsigned long long w = masses ? fixed_weight(zhi, rc, scale) : 0;
    int keep = by_mass ? n : (int)(k - above_c);
    if (by_mass && w > 0) {
      const double more = ceil((target - (double)above_m) / (double)w);
      keep = more < 1.0 ? 1 : more < (double)n ? (int)more : n;
    }
    keep = min(max(keep, 1), n);
    cut.z = zhi;
    cut.idx = nth_equal(row.p, row.V, row.nit, zhi, keep);
    cut.mass = above_m + w * (unsigned long long)keep;
    return cut;
  }
  // what is left, gathered in the histogram's memory and ranked by one wave
  float* lz = (float*)sh.cnt;
  int* li = (int*)sh.cnt + RANK;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  src.each([&](float z, int i) {
    if (in(z)) {
      const int at = atomicAdd(&sh.n, 1);
      if (at < RANK) { lz[at] = z; li[at] = i; }
    }
  });
  __syncthreads();
  if (tid < 64) {
    const bool any = tid < n;
    const float z = any ? lz[tid] : 0.0f;
    const int idx = any ? li[tid] : 0;
    const unsigned long long own = any && masses ? fixed_weight(z, rc, scale) : 0;
    const unsigned long long key =
        any ? ((unsigned long long)order_key(z) << 32) | (uint32_t)~idx : 0ull;
    int rank = 0;
    unsigned long long m = above_m + own;
    for (int j = 0; j < n; ++j) {
      const bool ahead = at_lane(key, j) > key;
      rank += ahead;
      if (masses) m += ahead ? at_lane(own, j) : 0ull;
    }
    bool here = by_mass ? (double)m >= target : above_c + rank + 1 >= k;
    // the lowest rank that fulfils it, the last one if none does
    const int at = at_lane(wave_scan(any && here ? rank : RANK, RANK, Min()), 63);
    if (any && rank == min(at, n - 1)) { sh.f[0] = z; sh.n = idx; sh.fm = m; }
  }
  __syncthreads();
  cut.z = uniform(sh.f[0]);
  cut.idx = uniform(sh.n);
  cut.mass = sh.fm;
  __syncthreads();
  return cut;
}

// The draw among the kept tokens, given each wave's kept weight in sh.d;
// sh.token and sh.w (its weight).
template <typename E>
static __device__ NOINLINE void draw_kept(const E* p, int V, int nit, float u) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const Row<E> row(p, V, nit);
  const int t = pick_index(row, [&](float z, int i) { return kept_weight(z, i, rc); },
                           (double)u * rc.total);
  if (threadIdx.x == 0) {
    sh.token = t;
    sh.w = t < 0 ? 0.0 : kept_weight(load_logit(p + t), t, rc);
  }
  __syncthreads();
}

// Both cuts of the tokens of `src` that reach `bound` (n of them): rc.z, rc.idx.
// whole: the weight that top-p is a share of, < 0: that of the k tokens.  scale:
// the weights', raised where these tokens' weight has to be found first.
template <typename Src, typename E>
static __device__ __forceinline__ void both_cuts(const Src& src, const Row<E>& row, RowCut& rc, int n,
                                          float bound, int k, double top_p, double whole,
                                          double& scale, Found so_far) {
  FilterShared& sh = shared();
  const bool need_p = top_p < 1.0;
  auto sum = [&] {                                  // (a list has no order)
    unsigned long long part = 0;
    src.each([&](float z, int) { part += z >= bound ? fixed_weight(z, rc, scale) : 0ull; });
    return (double)block_reduce(part, 0ull, Add(), sh.u);
  };
  if (need_p && whole < 0.0) scale = mass_scale(scale, sum() / scale);
  whole *= scale;
  for (int step = k < n ? 0 : 1; step < (need_p ? 2 : 1); ++step) {   // top-k, top-p
    if (step && whole < 0.0) whole = sum();         // top-k keeps all
    const Cut c = select_cut(src, row, rc, scale, n, rc.zmax, bound, step == 1, need_p,
                             (uint32_t)k, fmax(top_p, 0.0) * whole,
                             step == 1 ? so_far : Found{-1, 0, 0u, 0ull});
    if (c.z > rc.z || (c.z == rc.z && c.idx < rc.idx)) { rc.z = c.z; rc.idx = c.idx; }
    if (!step) whole = (double)c.mass;
  }
  rc.z = fmaxf(rc.z, bound);                        // without a cut: the candidates
}

// Cut, kept weight and draw over the row; n tokens reach `bound`.  u < 0: no
// draw.
template <typename E>
static __device__ NOINLINE void filter_row_again(const E* p, int V, int nit, int n, float bound, int k,
                                            double top_p, double whole, float u) {
  FilterShared& sh = shared();
  RowCut rc = sh.rc;
  const Row<E> row(p, V, nit);
  float lo = INFINITY;                              // the smallest candidate
  row.each([&](float z, int) { lo = z >= bound ? fminf(lo, z) : lo; });
  lo = block_reduce(lo, INFINITY, Min(), sh.f);
  // V weights of at most 2^(clz(V) + 30) stay below 2^62
  double scale = mass_scale(ldexp(1.0, __clz(V) + 30), whole);
  both_cuts(row, row, rc, n, lo, k, top_p, whole, scale, Found{-1, 0, 0u, 0ull});
  double part = 0.0;
  row.each_from(rc.z, [&](float z, int i) { part += kept_weight(z, i, rc); });
  rc.total = range_sums(part);
  if (threadIdx.x == 0) sh.rc = rc;
  __syncthreads();
  if (u >= 0.0f) draw_kept(p, V, nit, u);
}

// The draw among the n tokens of the list, -1 if they weigh nothing or u < 0.
// fixed(z, i): a token's weight, integers; 0 for tokens that are not in the
// list.  They are added up in bins of the index, and the drawn bin's tokens
// walked by one wave.
template <typename E, typename F>
static __device__ __forceinline__ int draw_list(const E* p, int V, int n, F fixed, float u,
                                                unsigned long long& total) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x;
  const int shift = max(0, 32 - BIN_BITS - __clz(V - 1));      // BINS bins over [0, V)
  __syncthreads();
  sh.mass[tid] = 0;
  __syncthreads();
  List{n}.each([&](float z, int i) {
    const unsigned long long w = fixed(z, i);
    if (w) atomicAdd(&sh.mass[i >> shift], w);
  });
  __syncthreads();
  uint32_t none = 0;
  unsigned long long m = sh.mass[tid];
  const unsigned long long own = m;
  scan_bins(none, m);
  if (tid == BINS - 1) sh.fm = m;
  __syncthreads();
  total = sh.fm;
  if (u < 0.0f || !total) return -1;
  const double t = (double)u * (double)total;
  int b = first_index(own && (double)m > t, tid, -1);
  const bool past = b < 0;                          // u = 1, or by rounding: the last token
  if (past) b = BINS - 1 - first_index(own > 0, BINS - 1 - tid, 0);
  if (tid == b) sh.fm = m - own;
  __syncthreads();
  if (tid < 64) {                                   // the bin's tokens, a run per lane
    const unsigned long long base = sh.fm;
    const int run = max(1, (1 << shift) / 64), first = (b << shift) + tid * run;
    const int end = min(min(V, first + run), (b + 1) << shift);
    unsigned long long part = 0;
    int last = -1;
    for (int i = first; i < end; ++i) {
      const unsigned long long w = fixed(load_logit(p + i), i);
      part += w;
      if (w) last = i;
    }
    const unsigned long long incl = wave_scan(part, 0ull, Add());
    unsigned long long acc = base + incl - part;
    const unsigned long long hit = __ballot(part && !past && (double)(base + incl) > t);
    const unsigned long long any = __ballot(part > 0);
    const int lane = hit ? __ffsll((long long)hit) - 1 : 63 - __clzll((long long)any);
    if (tid == lane) {
      int at = last;
      if (hit)
        for (int i = first; i < end; ++i) {
          acc += fixed(load_logit(p + i), i);
          if ((double)acc > t) { at = i; break; }
        }
      sh.i[0] = at;
    }
  }
  __syncthreads();
  return uniform(sh.i[0]);
}

// The same over the n <= LIST candidates in LDS.  found: shorten_list has left
// its histogram's bin of the weight.
template <typename E>
static __device__ NOINLINE void filter_list(const E* p, int V, int nit, int n, float bound, int k,
                                         double top_p, double whole, float u, bool found) {
  FilterShared& sh = shared();
  RowCut rc = sh.rc;
  const Row<E> row(p, V, nit);
  const List list{n};
  const Found so_far = found ? sh.so_far : Found{-1, 0, 0u, 0ull};
  double scale = mass_scale(LIST_SCALE, whole);
  both_cuts(list, row, rc, n, bound, k, top_p, whole, scale, so_far);
  // a positive weight counts for 1 at least
  auto fixed = [&](float z, int i) -> unsigned long long {
    const double w = kept_weight(z, i, rc);
    return w > 0.0 ? max((unsigned long long)(w * scale + 0.5), 1ull) : 0ull;
  };
  unsigned long long total;
  const int t = draw_list(p, V, n, fixed, u, total);
  if (threadIdx.x == 0) {
    rc.total = (double)total / scale;
    sh.rc = rc;
    if (u >= 0.0f) {
      sh.token = t;
      sh.w = t < 0 ? 0.0 : kept_weight(load_logit(p + t), t, rc);
    }
  }
  __syncthreads();
}

// Shortens a list of SMALL < n <= LIST candidates to those in the histogram
// bins up to the one that holds the k-th token, or (by_mass) in which the
// weight reaches `target` of `whole`.  Returns how many they are; n, and the list as it
// was, if more than SMALL; -1 if the list does not weigh `target`.
static __device__ NOINLINE int shorten_list(int n, float bound, bool by_mass, int k, double target,
                                            double whole) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const int tid = threadIdx.x;
  const double scale = mass_scale(LIST_SCALE, whole);   // filter_list's
  const Binning bin(rc.zmax, bound, true);
  const List list{n};
  sh.cnt[tid] = 0;
  sh.mass[tid] = 0;
  __syncthreads();
  list.each([&](float z, int) {
    const int b = bin(z);
    atomicAdd(&sh.cnt[b], 1u);
    if (by_mass) atomicAdd(&sh.mass[b], fixed_weight(z, rc, scale));
  });
  __syncthreads();
  uint32_t c = sh.cnt[tid];
  unsigned long long m = sh.mass[tid];
  scan_bins(c, m);
  const int b = first_index(by_mass ? (double)m >= target * scale : c >= (uint32_t)k, tid, -1);
  if (b < 0) return -1;
  if (tid == b) {
    const uint32_t own_c = sh.cnt[tid];
    sh.found = (int)c;
    sh.so_far = Found{b, (int)own_c, c - own_c, m - sh.mass[tid]};
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  const int left = uniform(sh.found);
  if (left > SMALL) return n;
  // gathered behind the histogram, then put in front
  float* gz = (float*)sh.mass;
  int* gi = (int*)sh.mass + SMALL;
  __syncthreads();
  list.each([&](float z, int i) {
    if (bin(z) <= b) {
      const int at = atomicAdd(&sh.n, 1);
      gz[at] = z;
      gi[at] = i;
    }
  });
  __syncthreads();
  if (tid < left) { sh.lz[tid] = gz[tid]; sh.li[tid] = gi[tid]; }
  __syncthreads();
  return left;
}

// Both cuts and the draw over the n <= SMALL candidates in LDS.  Every pair is
// compared, by logit and by index (the waves share the candidates out as 64 of
// them and a part of the others), which gives the tokens' places in both
// orders.  In the first, scanned weights give the cuts: kept by top-k are the
// first k, by top-p those whose weight ahead is below the target.  In the
// second, the lowest kept token whose running weight exceeds u * total is
// drawn.  (Adding up weights in the comparisons in place of the two scans: 32000
// cycles for 219 candidates, two rows to a CU.)  whole: the weight that top-p is
// a share of, < 0: that of the k tokens.  u < 0: no draw.  check: false if the
// candidates do not weigh that share.
static __device__ NOINLINE bool filter_small(int n, int k, double top_p, double whole, float u,
                                            bool check) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const double scale = 18014398509481984.0;    // 2^54: SMALL weights stay below 2^63
  unsigned long long* key = sh.mass;           // larger logit, then lower index, first
  unsigned long long* w = sh.mass + SMALL;
  float* zi = (float*)(sh.mass + 2 * SMALL);
  uint32_t *places = sh.cnt, *after = sh.cnt + SMALL;
  float z = 0.f;
  int idx = 0;
  unsigned long long own = 0;
  uint32_t heavy = 0;                          // not below min_p
  if (tid < n) {
    z = sh.lz[tid];
    idx = sh.li[tid];
    const double x = weight(z, rc);
    own = x > 0.0 ? max((unsigned long long)(x * scale + 0.5), 1ull) : 0ull;
    heavy = x >= (double)rc.min_w;
    key[tid] = ((unsigned long long)order_key(z) << 32) | (uint32_t)~idx;
  }
  if (tid < SMALL) places[tid] = 0;
  __syncthreads();
  const int groups = (n + 63) >> 6, parts = FW / groups;   // waves: part * groups + group
  const int part = wv / groups, cand = (wv - part * groups) * 64 + lane;
  if (part < parts && cand < n) {
    const unsigned long long mine = key[cand];
    uint32_t ahead = 0, lower = 0;
#pragma unroll 4
    for (int j = part; j < n; j += parts) {
      const unsigned long long other = key[j];
      ahead += other > mine;
      lower += (uint32_t)other > (uint32_t)mine;           // ~index
    }
    atomicAdd(&places[cand], ahead | lower << 16);
  }
  __syncthreads();
  if (tid < n) {
    const uint32_t both = places[tid], r = both & 0xffffu;
    sh.lz[r] = z;
    sh.li[r] = idx;
    w[r] = own;
    after[r] = both >> 16 | heavy << 31;
  }
  __syncthreads();
  // thread t: the t-th token by logit
  const int first_k = min(k, n);
  uint32_t at = 0, none = 0;
  own = 0;
  if (tid < n) {
    z = sh.lz[tid];
    idx = sh.li[tid];
    own = w[tid];
    at = after[tid];
  }
  bool kept = tid < first_k, next = tid + 1 < first_k;
  if (top_p < 1.0) {
    unsigned long long run = own;
    scan_bins(none, run);
    if (tid == first_k - 1) sh.fm = run;
    __syncthreads();
    const double sum_k = (double)sh.fm;
    const double target = fmax(top_p, 0.0) * (whole < 0.0 ? sum_k : whole * scale);
    if (check && sum_k < target) return false;
    next = next && (double)run < target;
    kept = kept && (tid == 0 || (double)(run - own) < target);
  }
  if (kept && !next) { sh.rc.z = z; sh.rc.idx = idx; }     // the last one
  if (!(kept && (at >> 31 || tid == 0))) own = 0;
  if (u < 0.0f) {
    const unsigned long long total = block_reduce(own, 0ull, Add(), sh.u);
    if (tid == 0) sh.rc.total = (double)total / scale;
    __syncthreads();
    return true;
  }
  at &= 0xffffu;
  if (tid < n) { key[at] = own; places[at] = idx; zi[at] = z; }
  __syncthreads();
  // thread t: the t-th by index
  own = tid < n ? key[tid] : 0;
  idx = tid < n ? (int)places[tid] : 0;
  unsigned long long run = own;
  scan_bins(none, run);
  if (tid == n - 1) sh.fm = run;
  __syncthreads();
  const unsigned long long total = sh.fm;
  if (tid == 0) sh.rc.total = (double)total / scale;
  int token = first_index(own > 0 && (double)run > (double)u * (double)total, idx, -1);
  if (token < 0) token = block_reduce(own > 0 ? idx : -1, -1, Max(), sh.i);
  if (own > 0 && idx == token) { sh.token = token; sh.w = weight(zi[tid], rc); }
  __syncthreads();
  return true;
}

// A logit that every token before the cut reaches (k > 0), or is likely to
// (top-p).  part[]: maxima over parts of this thread's logits, lo the smallest
// of them.  The lower edge of the histogram bin where their count reaches k,
// or their weight, each taken for the tokens that it stands for, `target`;
// -FLT_MAX if it does not, or where a part stands for too many.
static __device__ __forceinline__ float parts_bound(const float (&part)[PARTS], const RowCut& rc,
                                                    int V, float lo, int k, float target) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x;
  if (!(lo < rc.zmax)) return -FLT_MAX;
  // (linear bins would be one bin where tokens are masked by a lowest number)
  const Binning bin(rc.zmax, lo, rc.zmax * 0.5f - lo * 0.5f <= 32.0f * (fabsf(rc.zmax) + 1.0f));
  // a bin: its count above 40 bits of weight, in 2^-26 (at most 2^13 parts)
  const float scale = 67108864.0f, log2e_t = (float)rc.log2e_t;
  sh.mass[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PARTS; ++j) {
    if (part[j] > -INFINITY) {
      const float w = __builtin_amdgcn_exp2f((part[j] - rc.zmax) * log2e_t) * scale;
      atomicAdd(&sh.mass[bin(part[j])], (1ull << 40) | (uint32_t)w);
    }
  }
  __syncthreads();
  const unsigned long long got = sh.mass[tid];
  uint32_t c = (uint32_t)(got >> 40);
  unsigned long long m = 0;
  scan_bins(c, m);
  bool there = c >= (uint32_t)k;
  if (!k) {
    if (tid == FT - 1) sh.fc = c;
    const float own = (float)(got & ((1ull << 40) - 1));
    __syncthreads();
    const float parts = (float)sh.fc;
    const float left = 1.0f - (float)c * __builtin_amdgcn_rcpf(parts);
    // parts that more than nine tenths exceed say little
    uint32_t few = left < 0.1f;
    const float others = 1.0f - parts / (float)V;
    m = few ? 0ull : (unsigned long long)(own * __builtin_amdgcn_exp2f(-others * __builtin_amdgcn_logf(left)));
    scan_bins(few, m);
    there = !few && (float)m >= target * scale;
  }
  const int at = first_index(there, tid, -1);
  return at < 0 ? -FLT_MAX : bin.lower_edge(at);
}

// A bound as parts_bound's, by a histogram over the row, where the parts do
// not hold enough.  No weights: a bin adds up its tokens' count and, in 2^-16
// of the bin's width, how far they lie below its upper edge, rounded up.  As
// exp is convex, the count times the weight at their mean is no more than they
// weigh, and less by (width / T)^2 / 8 at most.  sh.lo: the bound; sh.found: how
// many tokens reach it (about; V + 1: the row ends before the target).  For
// top-p also sh.hi, a logit from which the tokens up weigh less than the target,
// and sh.inside, how many lie between the two.
template <typename E>
static __device__ __forceinline__ void row_bound(const E* p, int V, int nit, float bound, int k,
                                                 double target, double scale) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const int tid = threadIdx.x;
  const Row<E> row(p, V, nit);
  const Binning bin(rc.zmax, bound, rc.zmax * 0.5f - bound * 0.5f <= 32.0f * (fabsf(rc.zmax) + 1.0f));
  sh.mass[tid] = 0;
  __syncthreads();
  auto add = [&](float z) {
    if (z >= bound) {
      const float x = (bin.half - z * 0.5f) * bin.sc;
      const int b = bin(z);
      const uint32_t below = bin.linear ? (uint32_t)((x - (float)b) * 65536.0f) + 1u : 0u;
      atomicAdd(&sh.mass[b], (1ull << 40) | below);   // V <= 2^22
    }
  };
  row.batches([&](const u32x16& b, int) {
#pragma unroll
    for (int e = 0; e < BATCH; ++e) add(Row<E>::logit(b, e));
  });
  const int ri = row.rest_index();
  if (ri >= 0) add(load_logit(p + ri));
  __syncthreads();
  const unsigned long long got = sh.mass[tid];
  const double count = (double)(got >> 40);
  unsigned long long m = got >> 40;
  if (!k && m) {
    double w;
    if (bin.linear) {
      // below the largest logit, not as a logit: those far from zero are
      // further apart than this may be off
      const double mean = tid + (double)(got & ((1ull << 40) - 1)) / (65536.0 * count);
      w = exp2_neg(-2.0 * mean * (double)bin.width, rc.log2e_t);
    } else {
      w = weight(bin.lower_edge(tid), rc);
    }
    // (1e-5 less: the roundings of x and sc move a mean by less at any T whose
    // weights reach this far)
    m = (unsigned long long)(count * w * (1.0 - 1e-5) * scale);
  }
  uint32_t c = (uint32_t)(got >> 40);
  scan_bins(c, m);
  const bool there = k ? m >= (unsigned long long)k : (double)m >= target * scale;
  const int at = first_index(there, tid, -1);
  int over = 0;                                     // the bins before may be above
  if (!k && bin.linear) {
    const double h = 1.3863 * (double)bin.width * rc.log2e_t;
    over = first_index((double)m * (1.0 + 0.125 * h * h + 1e-4) >= target * scale, tid, 0);
  }
  if (tid == 0) {
    sh.inside = sh.found = V + 1;
    sh.hi = over ? bin.lower_edge(over - 1) : INFINITY;
  }
  __syncthreads();
  if (tid == at) sh.found = (int)c;
  if (tid == over - 1) sh.fc = c;
  __syncthreads();
  if (tid == 0) {
    if (at >= 0) sh.inside = sh.found - (over ? (int)sh.fc : 0);
    sh.lo = at < 0 ? bound : fmaxf(bound, bin.lower_edge(at));
  }
  __syncthreads();
}

// The weight of min-p's tokens, none of them below `bound`.
template <typename E>
static __device__ __forceinline__ double min_p_sum(const Row<E>& row, const RowCut& rc,
                                                   float bound) {
  double kept = 0.0;
  row.each_from(bound, [&](float z, int) {
    const double w = weight(z, rc);
    kept += w >= (double)rc.min_w ? w : 0.0;
  });
  return range_sums(kept);
}

// Bound (sh.lo) and, for a flat row of top-p, the cut and the draw: the tokens
// from sh.hi up, too many for a list, are added up, those of [sh.lo, sh.hi) are
// the list.  Where min-p's tokens weigh less than the target, they are kept.
// false if there is no cut yet.  65536 normal logits of sigma / T about 0.6, one
// row: 56 us, 124 by filter_row_again (26 where a list holds the cut).
template <typename E>
static __device__ NOINLINE bool filter_flat(const E* p, int V, int nit, float sure, int k,
                                            double target, double whole_w, float u) {
  FilterShared& sh = shared();
  RowCut rc = sh.rc;
  const int tid = threadIdx.x, lane = tid & 63;
  const Row<E> row(p, V, nit);
  const double scale = mass_scale(ldexp(1.0, __clz(V) + 30), whole_w);   // as filter_row_again
  row_bound(p, V, nit, sure, k, target * (1.0 + 1e-9), scale);
  const float lo = uniform(sh.lo), hi = uniform(sh.hi);
  if (k || uniform(sh.found) <= LIST) return false;
  if (rc.min_w > 0.0f && uniform(sh.found) > V) {
    const double kept = min_p_sum(row, rc, lo);
    if (!(kept < target)) return false;
    rc.z = lo;
    rc.total = kept;
    if (tid == 0) sh.rc = rc;
    __syncthreads();
    if (u >= 0.0f) draw_kept(p, V, nit, u);
    return true;
  }
  if (uniform(sh.inside) > LIST) return false;
  const double floor = -1000.0 / rc.log2e_t;        // 2^-1000 stands for less
  double part = 0.0;
  const double top = (double)rc.zmax;
  const int n = gather(
      row, [=](float z) { return z >= lo && z < hi; },
      [&](float z) {
        const double w = exp2_normal(fmax((double)z - top, floor), rc.log2e_t);
        part += z >= hi ? w : 0.0;
      });
  const double above = range_sums(part);
  if (n < 1 || n > LIST || !(above < target)) return false;
  const double range = lane < FW ? sh.d[lane] : 0.0;
  const List list{n};
  const Cut cut = select_cut(list, row, rc, scale, n, fminf(hi, rc.zmax), lo, true, true, 0u,
                             target * scale,
                             Found{-1, 0, 0u, (unsigned long long)(above * scale + 0.5)});
  if ((double)cut.mass < target * scale || weight(cut.z, rc) < (double)rc.min_w) return false;
  rc.z = cut.z;
  rc.idx = cut.idx;
  // the kept weight of each wave's range
  if (tid < FW) sh.mass[tid] = 0;
  __syncthreads();
  const int span = nit * 64 * Row<E>::EPV, whole = V / Row<E>::EPV * Row<E>::EPV;
  list.each([&](float z, int i) {
    if (before_cut(z, i, rc))
      atomicAdd(&sh.mass[i < whole ? i / span : FW - 1], fixed_weight(z, rc, scale));
  });
  __syncthreads();
  const double kept = lane < FW ? range + (double)sh.mass[lane] / scale : 0.0;
  if (tid < FW) sh.d[tid] = kept;
  rc.total = at_lane(row_scan(kept, 0.0, Add()), FW - 1);
  if (tid == 0) sh.rc = rc;
  __syncthreads();
  if (u >= 0.0f) draw_kept(p, V, nit, u);
  return true;
}

// Reads a row, finds what its filters keep (sh.rc) and, for u >= 0, draws a
// token (sh.token, sh.w: its weight).
template <typename E>
static __device__ __forceinline__ void filter_row(const Row<E>& row, const RowParams& par, int pi,
                                           float u, int32_t* err) {
  FilterShared& sh = shared();
  constexpr int EPV = Row<E>::EPV;
  const int tid = threadIdx.x, V = row.V;
  const float T = uniform(par.temperature ? par.temperature[pi] : 1.0f);
  const int k = uniform(par.top_k ? par.top_k[pi] : 0);
  const double top_p = (double)uniform(par.top_p ? par.top_p[pi] : 1.0f);
  RowCut rc;
  rc.z = -INFINITY;
  rc.idx = 0x7fffffff;
  rc.min_w = uniform(par.min_p ? par.min_p[pi] : 0.0f);
  if (!(rc.min_w > 0.0f)) rc.min_w = 0.0f;
  rc.log2e_t = 1.4426950408889634 / (double)T;
  rc.total = 0.0;
  rc.single = 0;
  const bool greedy = !(T > 0.0f) || k == 1 || rc.min_w > 1.0f;
  const bool need_k = k > 0 && k < V, need_p = top_p < 1.0;
  const bool need_sum = !greedy && !need_k && (need_p || rc.min_w == 0.0f);

  float part[PARTS], mine = -INFINITY;
  double sum = 0.0;                            // of exp((z - mine) / T)
  bool bad = false;
#pragma unroll
  for (int j = 0; j < PARTS; ++j) part[j] = -INFINITY;
  // below `floor` a weight counts as 2^-1000 in the sum, in place of less
  const double floor = -1000.0 / rc.log2e_t;
  row.batches([&](const u32x16& b, int) {
    float most = mine;
#pragma unroll
    for (int e = 0; e < BATCH; ++e) {
      const float z = Row<E>::logit(b, e);
      bad |= !(z < INFINITY);
      part[e * PARTS / BATCH] = fmaxf(part[e * PARTS / BATCH], z);
    }
#pragma unroll
    for (int j = 0; j < PARTS; ++j) most = fmaxf(most, part[j]);
    if (need_sum) {
      // the sum so far in terms of the new maximum (an infinite one: no sum)
      const double top = (double)most;
      sum *= exp2_normal(fmax((double)mine - top, floor), rc.log2e_t);
#pragma unroll
      for (int e = 0; e < BATCH; ++e)
        sum += exp2_normal(fmax((double)Row<E>::logit(b, e) - top, floor), rc.log2e_t);
    }
    mine = most;
  });
  const int ri = row.rest_index();
  if (ri >= 0) {
    const float z = load_logit(row.p + ri);
    bad |= !(z < INFINITY);
    const float most = fmaxf(mine, z);
    if (need_sum)
      sum = sum * exp2_neg((double)mine - (double)most, rc.log2e_t) +
            exp2_neg((double)z - (double)most, rc.log2e_t);
    part[0] = fmaxf(part[0], z);
    mine = most;
  }
  float least = INFINITY;
#pragma unroll
  for (int j = 0; j < PARTS; ++j) least = fminf(least, part[j] > -INFINITY ? part[j] : INFINITY);
  float hi = mine, lo = least;
  block_max_min(hi, lo);
  if (bad) set_err(err, DVS_ERR_NONFINITE);
  rc.zmax = hi;
  const bool empty = hi == -INFINITY;
  if (empty && tid == 0) set_err(err, DVS_ERR_NONFINITE);
  if (greedy || empty || hi == INFINITY) {
    // top-1: the lowest index of the maximum
    int at = 0x7fffffff;
    row.each_from(hi, [&](float z, int i) { if (z == hi && i < V) at = min(at, i); });
    at = first_index(at != 0x7fffffff, at, -1);
    rc.z = hi;
    rc.idx = at;
    rc.single = empty ? -1 : 1;
    rc.total = empty ? 0.0 : 1.0;
    if (tid == 0) {
      sh.rc = rc;
      sh.token = max(at, 0);                   // a row of NaN alone: 0
      sh.w = rc.total;
    }
    __syncthreads();
    return;
  }
  double whole = -1.0;                         // the row's weight
  if (need_sum) {
    sum *= exp2_neg((double)mine - (double)hi, rc.log2e_t);
    if (T > FLT_MAX) {                         // infinite: every token but the masked ones, once
      sum = 0.0;
      row.each([&](float z, int) { sum += weight(z, rc); });
    }
    whole = range_sums(sum);
  }
  float bound = -FLT_MAX;                      // tokens below are not kept
  if (!need_k && !need_p) {
    if (rc.min_w > 0.0f) {
      bound = weight_bound(hi, (double)T, (double)rc.min_w);
      whole = min_p_sum(row, rc, bound);
    }
    rc.z = bound;
    rc.total = whole;
    if (tid == 0) sh.rc = rc;
    __syncthreads();
    if (u >= 0.0f) draw_kept(row.p, V, row.nit, u);
    return;
  }
  const double target = fmax(top_p, 0.0) * whole;   // (top-p alone)
  const int kk = need_k ? k : 0;
  // (a third of the way from the share p to all: room for the sample's error)
  float sure = -FLT_MAX;
  bound = parts_bound(part, rc, V, lo, kk, (float)(target + 0.3 * (whole - target)));
  if (!need_k) {
    // tokens of less than (1 - p) / V of the weight each cannot hold 1 - p of it
    sure = weight_bound(hi, (double)T, (1.0 - fmax(top_p, 0.0)) * whole / (double)V);
    if (rc.min_w > 0.0f) sure = fmaxf(sure, weight_bound(hi, (double)T, (double)rc.min_w));
  }
  const double share = need_p ? top_p : 1.0;
  // bounds: 0 the parts', 1 the sure one, 2 the row's
  for (int level = bound > sure || need_k ? 0 : bound > -FLT_MAX ? 1 : 2;;) {
    if (level == 1) bound = sure;
    if (tid == 0) sh.rc = rc;                  // (seen after gather)
    if (level == 2) {
      __syncthreads();
      if (filter_flat(row.p, V, row.nit, sure, kk, target, whole, u)) return;
      bound = uniform(sh.lo);
    }
    int n = gather(row, bound);
    if (n > LIST && level < 2) {
      level = 2;
      continue;
    }
    const int keep = need_k ? min(k, n) : n;
    bool found = false;
    if (n > SMALL && n <= LIST && (!need_k || keep <= SMALL)) {
      const int left = shorten_list(n, bound, !need_k, keep, target, whole);
      if (left < 0 && level == 0) {
        level = 1;
        continue;
      }
      n = left < 0 ? n : left;
      found = !need_k && left > SMALL;
    }
    if (n <= SMALL) {
      if (!filter_small(n, min(keep, n), share, whole, u, level == 0)) {
        level = 1;
        continue;
      }
    } else if (n <= LIST) {
      filter_list(row.p, V, row.nit, n, bound, keep, share, whole, u, found);
    } else {
      filter_row_again(row.p, V, row.nit, n, bound, keep, share, whole, u);
    }
    return;
  }
}

};  // RowFilter

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------

template <int FT, typename E>
__global__ void __launch_bounds__(FT, 4) sample_filtered_kernel(
    const E* __restrict__ logits, long long ld, int V, int nit, RowParams par, int rows_per_param,
    const float* __restrict__ u, int u_stride, int32_t* __restrict__ token_out,
    float* __restrict__ prob_out, int32_t* err, int first) {
  auto& sh = RowFilter<FT>::shared();
  const int r = first + blockIdx.x, s = r / rows_per_param;
  const typename RowFilter<FT>::template Row<E> row(logits + (size_t)r * ld, V, nit);
  float uu = u[(size_t)s * u_stride + (r - s * rows_per_param)];
  if (!(uu > 0.0f)) uu = 0.0f;
  RowFilter<FT>::filter_row(row, par, s, uu, err);
  if (threadIdx.x == 0) {
    token_out[r] = sh.token;
    if (prob_out) prob_out[r] = sh.rc.total > 0.0 ? (float)(sh.w / sh.rc.total) : 0.0f;
  }
}

// Cuts of the verify rows (first S * (B + 1)) and draft rows (S * B) of a call.
template <int FT, typename E>
__global__ void __launch_bounds__(FT, 4) filter_rows_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int B, int nv, int V, int nit, RowParams par, RowCut* __restrict__ cuts,
    int32_t* err, int first) {
  const int r = first + blockIdx.x;
  const int per = r < nv ? B + 1 : B, i = r < nv ? r : r - nv;
  const int s = i / per, j = i - s * per;
  const E* z = r < nv ? zv + (size_t)s * vs + (size_t)j * vld : zd + (size_t)s * ds + (size_t)j * dld;
  const typename RowFilter<FT>::template Row<E> row(z, V, nit);
  RowFilter<FT>::filter_row(row, par, s, -1.0f, err);
  if (threadIdx.x == 0) {
    RowCut rc = RowFilter<FT>::shared().rc;
    rc.inv_total = rc.total > 0.0 ? 1.0 / rc.total : 0.0;
    cuts[r] = rc;
  }
}

__device__ __forceinline__ double prob_of(float z, int i, const RowCut& c) {
  if (c.single) return c.single > 0 && i == c.idx ? 1.0 : 0.0;
  return kept_weight(z, i, c) * c.inv_total;
}

// One workgroup per sequence: d_j accepted while u q_j(d_j) < p_j(d_j), then
// the final token from max(0, p - q) of the rejected draft's rows, or from the
// last verify row: a list in LDS of the tokens that p keeps, weighed together
// (8 sequences of V = 65536: 13 us, 17 by two walks over the row; those remain
// for tokens that do not fit a list).
template <typename E>
__global__ void __launch_bounds__(1024) accept_filtered_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int S, int B, int V, int nit, const RowCut* __restrict__ cuts,
    const int32_t* __restrict__ draft, int draft_width, const float* __restrict__ u, int u_stride,
    int32_t* __restrict__ accept_len, int32_t* __restrict__ token_out, int token_stride,
    int at_accepted, int first) {
  using F = RowFilter<1024>;
  auto& sh = F::shared();
  const int s = first + blockIdx.x, tid = threadIdx.x;
  const RowCut* cv = cuts + (size_t)s * (B + 1);
  const RowCut* cd = cuts + (size_t)S * (B + 1) + (size_t)s * B;
  const E* v = zv + (size_t)s * vs;
  const E* d = zd + (size_t)s * ds;
  if (tid == 0) sh.found = B;
  __syncthreads();
  for (int j = tid; j < B; j += 1024) {    // the first rejected draft
    const int t = draft[(size_t)s * draft_width + j];
    bool ok = false;
    if (t >= 0 && t < V) {
      const double p = prob_of(load_logit(v + (size_t)j * vld + t), t, cv[j]);
      const double q = prob_of(load_logit(d + (size_t)j * dld + t), t, cd[j]);
      ok = (double)u[(size_t)s * u_stride + j] * q < p;
    }
    if (!ok) atomicMin(&sh.found, j);
  }
  __syncthreads();
  const int A = sh.found;
  __syncthreads();
  float uu = u[(size_t)s * u_stride + B];
  if (!(uu > 0.0f)) uu = 0.0f;
  const RowCut p = cv[A];
  const typename F::template Row<E> row(v + (size_t)A * vld, V, nit);
  const RowCut q = cd[A < B ? A : 0];
  const E* zq = d + (size_t)(A < B ? A : 0) * dld;
  int t = -1;
  // the tokens of p, if they fit (no row without a number above -inf)
  int n = F::LIST + 1;
  if (p.single >= 0 && (p.z > -FLT_MAX || V <= F::LIST)) n = F::gather(row, p.z);
  // p - q, or p alone: after B acceptances, and where p and q are equal to the
  // last bit
  for (int step = A < B ? 0 : 1; step < 2 && t < 0 && p.single >= 0; ++step) {
    auto rest = [&](float z, int i) {
      double a = i < V ? prob_of(z, i, p) : 0.0;
      if (step == 0 && a > 0.0) a = fmax(a - prob_of(load_logit(zq + i), i, q), 0.0);
      return a;
    };
    if (n <= F::LIST) {
      auto fixed = [&](float z, int i) -> unsigned long long {   // sums of up to 1
        const double a = rest(z, i);
        return a > 0.0 ? max((unsigned long long)(a * 1152921504606846976.0 + 0.5), 1ull) : 0ull;
      };
      unsigned long long total;
      t = F::draw_list(v + (size_t)A * vld, V, n, fixed, uu, total);
    } else {
      double part = 0.0;
      row.each_from(p.z, [&](float z, int i) { part += rest(z, i); });
      const double total = F::range_sums(part);
      t = F::pick_index(row, rest, (double)uu * total);
    }
    __syncthreads();
  }
  if (t < 0) t = max(p.idx, 0);          // a row without a number above -inf
  if (tid == 0) {
    accept_len[s] = A;
    token_out[(size_t)s * token_stride + (at_accepted ? A : 0)] = t;
  }
}

size_t filter_cuts_bytes(int S, int B) { return (size_t)S * (2 * B + 1) * sizeof(RowCut); }

// Vectors per lane of a row.
template <typename E>
static int row_vectors(int V, int threads) {
  const int epv = 16 / (int)sizeof(E);
  return (V / epv + threads - 1) / threads;
}

// Calls f(threads): 1024 while every row has a CU of its own, else 512.
// V = 65536, us with 1024 / 512 threads:
//   rows      f32, top-p    f32, top-k    f32, min-p    bf16, top-k    bf16, mixed
//     32       43 / 52
//    256       58 / 78
//   1024      171 / 147     105 / 99      103 / 112      83 / 67       116 / 90
template <typename F>
static void by_rows(int rows, F f) {
  if (rows <= device_cus())
    f(IC<1024>{});
  else
    f(IC<512>{});
}

// Calls f(first, count) for `groups` workgroups, 2^21 at a time: a launch has less
// than 2^32 threads.
template <typename F>
static void by_launches(int groups, F f) {
  constexpr int MOST = 1 << 21;
  for (long long first = 0; first < groups; first += MOST)
    f((int)first, (int)(groups - first < MOST ? groups - first : MOST));
}

template <typename E>
static int launch_accept(const void* zv, long long vs, long long vld, const void* zd, long long ds,
                         long long dld, int S, int B, int V, const RowParams& par,
                         const int32_t* draft, int draft_width, const float* u, int u_stride,
                         int32_t* accept_len, int32_t* token_out, int token_stride,
                         int at_accepted, int32_t* err, void* ws, hipStream_t st) {
  RowCut* cuts = (RowCut*)ws;
  const int rows = S * (2 * B + 1);
  by_rows(rows, [&](auto threads) {
    constexpr int FT = decltype(threads)::value;
    by_launches(rows, [&](int first, int n) {
      hipLaunchKernelGGL((filter_rows_kernel<FT, E>), dim3(n), dim3(FT), 0, st, (const E*)zv, vs,
                         vld, (const E*)zd, ds, dld, B, S * (B + 1), V, row_vectors<E>(V, FT), par,
                         cuts, err, first);
    });
  });
  const int nit = row_vectors<E>(V, 1024);
  by_launches(S, [&](int first, int n) {
    hipLaunchKernelGGL(accept_filtered_kernel<E>, dim3(n), dim3(1024), 0, st, (const E*)zv, vs, vld,
                       (const E*)zd, ds, dld, S, B, V, nit, cuts, draft, draft_width, u, u_stride,
                       accept_len, token_out, token_stride, at_accepted, first);
  });
  return launch_status("accept_sampled");
}

template <typename E>
static void launch_sample(const void* logits, int rows, int V, long long ld, const RowParams& par,
                          int rows_per_param, const float* u, int u_stride, int32_t* token_out,
                          float* prob_out, int32_t* err, hipStream_t st) {
  by_rows(rows, [&](auto threads) {
    constexpr int FT = decltype(threads)::value;
    by_launches(rows, [&](int first, int n) {
      hipLaunchKernelGGL((sample_filtered_kernel<FT, E>), dim3(n), dim3(FT), 0, st,
                         (const E*)logits, ld, V, row_vectors<E>(V, FT), par, rows_per_param, u,
                         u_stride, token_out, prob_out, err, first);
    });
  });
}

int launch_sample_filtered(const void* logits, int dtype, int rows, int V, long long ld,
                           const RowParams& par, int rows_per_param, const float* u, int u_stride,
                           int32_t* token_out, float* prob_out, int32_t* err, hipStream_t st) {
  if (dtype == DVS_BF16)
    launch_sample<uint16_t>(logits, rows, V, ld, par, rows_per_param, u, u_stride, token_out,
                            prob_out, err, st);
  else
    launch_sample<float>(logits, rows, V, ld, par, rows_per_param, u, u_stride, token_out, prob_out,
                         err, st);
  return launch_status("sample_filtered");
}

int launch_accept_sampled(const void* zv, long long vs, long long vld, const void* zd,
                          long long ds, long long dld, int dtype, int S, int B, int V,
                          const RowParams& par, const int32_t* draft, int draft_width,
                          const float* u, int u_stride, int32_t* accept_len, int32_t* token_out,
                          int token_stride, int at_accepted, int32_t* err, void* ws,
                          hipStream_t st) {
  return dtype == DVS_BF16
             ? launch_accept<uint16_t>(zv, vs, vld, zd, ds, dld, S, B, V, par, draft, draft_width, u,
                                       u_stride, accept_len, token_out, token_stride, at_accepted,
                                       err, ws, st)
             : launch_accept<float>(zv, vs, vld, zd, ds, dld, S, B, V, par, draft, draft_width, u,
                                    u_stride, accept_len, token_out, token_stride, at_accepted, err,
                                    ws, st);
}

}  // namespace dvs

using namespace dvs;

extern "C" int sample_filtered(const void* logits, int32_t dtype, int32_t rows, int32_t V,
                               int64_t ld, const float* temperature, const int32_t* top_k,
                               const float* top_p, const float* min_p, int32_t rows_per_param,
                               const float* u, int32_t* token_out, float* prob_out,
                               int32_t* err_word, void* stream) {
  clear_error();
  DVS_CHECK_ARG(logits && u && token_out, "sample_filtered: NULL array argument");
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "sample_filtered: dtype %d", dtype);
  DVS_CHECK_ARG(rows >= 1 && V >= 1 && V <= (1 << 22), "sample_filtered: need rows >= 1 and 1 <= V <= 2^22");
  DVS_CHECK_ARG(ld >= V, "sample_filtered: row stride %lld < V", (long long)ld);
  DVS_CHECK_ARG(rows_per_param >= 1 && rows % rows_per_param == 0,
                "sample_filtered: rows (%d) must be groups of rows_per_param (%d)", rows,
                rows_per_param);
  return launch_sample_filtered(logits, dtype, rows, V, ld, RowParams{temperature, top_k, top_p, min_p},
                                rows_per_param, u, rows_per_param, token_out, prob_out, err_word,
                                (hipStream_t)stream);
}

extern "C" size_t dvs_accept_workspace_bytes(int32_t S, int32_t B, int32_t V) {
  if (S < 1 || B < 1 || V < 1 || V > (1 << 22)) return 0;
  return (filter_cuts_bytes(S, B) + 255) & ~(size_t)255;
}

extern "C" int accept_sampled(const void* z_verify, int64_t verify_seq, int64_t verify_ld,
                              const void* z_draft, int64_t draft_seq, int64_t draft_ld,
                              int32_t dtype, int32_t S, int32_t B, int32_t V,
                              const float* temperature, const int32_t* top_k, const float* top_p,
                              const float* min_p, const int32_t* draft, int32_t draft_width,
                              const float* u, int32_t* accept_len, int32_t* token_out,
                              int32_t* err_word, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  DVS_CHECK_ARG(z_verify && z_draft && draft && u && accept_len && token_out,
                "accept_sampled: NULL array argument");
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "accept_sampled: dtype %d", dtype);
  DVS_CHECK_ARG(S >= 1 && B >= 1 && V >= 1 && V <= (1 << 22),
                "accept_sampled: need S, B >= 1 and 1 <= V <= 2^22");
  DVS_CHECK_ARG((int64_t)S * (2 * (int64_t)B + 1) <= 0x7fffffff, "accept_sampled: too many rows");
  DVS_CHECK_ARG(verify_ld >= V && draft_ld >= V && verify_seq >= 0 && draft_seq >= 0,
                "accept_sampled: a row stride is less than V");
  DVS_CHECK_ARG(draft_width >= B, "accept_sampled: draft narrower than B");
  const size_t need = dvs_accept_workspace_bytes(S, B, V);
  if (!workspace || ws_bytes < need) {
    set_error("accept_sampled: workspace needs %zu bytes, got %zu", need, ws_bytes);
    return DVS_EWORKSPACE;
  }
  return launch_accept_sampled(z_verify, verify_seq, verify_ld, z_draft, draft_seq, draft_ld, dtype,
                               S, B, V, RowParams{temperature, top_k, top_p, min_p}, draft,
                               draft_width, u, B + 1, accept_len, token_out, 1, 0, err_word,
                               workspace, (hipStream_t)stream);
}
