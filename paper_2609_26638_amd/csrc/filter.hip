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
// hundred.  64-bit adds and multiplies run at the 32-bit rate on this chip.
//
// One workgroup of 1024 threads per row.  Wave w owns one contiguous range of
// the row, so the ranges' sums are in index order; a row of up to 65536
// logits is read once and stays in registers.
//   1. maximum and minimum;
//   2. a logit that no kept token lies below, and the tokens from there up as
//      a list in LDS: by the threads' own maxima for top-k (count_bound), by
//      the whole weight for top-p;
//   3. up to RANK candidates (a longer list is shortened by one histogram) are
//      ranked against each other, which gives the cut, the kept weight and the
//      draw at once (rank_cut);
//   4. otherwise (a flat distribution, a large k, many equal logits) a
//      histogram with a count and a weight sum per bin is narrowed to the bin
//      that holds the k-th token or the share p of the weight, until few
//      tokens are left (select_cut), over the list or over the row;
//   5. without a cut, or after 4: the kept weight per range, the range that
//      holds u * total, and one scan over that range's tokens (draw_kept).
// The row's registers are dead after step 2, or after the sums of step 5
// without a cut; what follows is kept out of line and reads the row again
// where it needs it, so that the registers of both are never live at once.
// Weights that atomics or an unordered list add up are fixed-point integers,
// whose sums do not depend on the order; the other sums have a fixed order.
// Results do not depend on timing, nor on the other rows of the call.
#include <math.h>

#include "dvs_common.h"

namespace dvs {

constexpr int FT = 1024;          // threads of a row's workgroup
constexpr int FW = FT / 64;
constexpr int BINS = 1024;        // one histogram bin per thread
constexpr int RANK = 512;         // tokens that are ranked against each other
constexpr int LIST = 8192;        // candidates held in LDS (64 KB)

// What a row's filters keep: weight >= min_w of the tokens with z > cut.z, or
// z == cut.z and index <= cut.idx.
struct RowCut {
  float zmax, z;     // largest logit; the cut's
  int idx;           // the cut's index among equal logits
  float min_w;       // min_p
  double log2e_t;    // log2(e) / T
  double total;      // kept weight
  int single;        // 1: only token idx is kept (weight 1); -1: no token
};

struct FilterShared {
  uint32_t cnt[BINS];
  unsigned long long mass[BINS];
  float lz[LIST];
  int li[LIST];
  double d[FW];
  unsigned long long u[FW];
  uint32_t c[FW];
  float f[FW], g[FW];
  int pick[2];
  int found, n, token;
  uint32_t fc;
  unsigned long long fm;
  double w;
  RowCut rc;
};

// The workgroup's LDS, for the functions that are kept out of line too.
__device__ __forceinline__ FilterShared& shared() {
  __shared__ FilterShared sh;
  return sh;
}

// 2^t for t <= 0: 2^n (1 + f P(f)), t = n + f, |f| <= 1/2.  P interpolates
// (2^f - 1) / f at Chebyshev nodes: 3.7e-14 relative.  0 for t below -1021,
// -inf and NaN (a masked logit, or one that is not a number).
__device__ __forceinline__ double exp2_neg(double t) {
  const double shift = 6755399441055744.0;     // 1.5 * 2^52: n in the low word
  const double s = t + shift;
  const double f = t - (s - shift);
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
  const int hi = __double2hiint(q) + (__double2loint(s) << 20);
  return t > -1021.0 ? __hiloint2double(hi, __double2loint(q)) : 0.0;
}

// exp((z - zmax) / T), zmax finite.
__device__ __forceinline__ double weight(float z, const RowCut& c) {
  return exp2_neg(((double)z - (double)c.zmax) * c.log2e_t);
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
__device__ __forceinline__ float vec_elem(const u32x4& x, int e) {
  if constexpr (sizeof(E) == 2)
    return __uint_as_float((e & 1) ? (x[e >> 1] & 0xffff0000u) : (x[e >> 1] << 16));
  else
    return __uint_as_float(x[e]);
}

// A row of V logits, in 16-byte vectors: wave w holds the nit * 64 vectors of
// its range, lane by lane.  NV > 0: they stay in registers (nit <= NV);
// NV = 0: every pass reads them again, four in flight.  Past the row's end
// the logits are -inf.
template <typename E, int NV>
struct Row {
  static constexpr int EPV = 16 / sizeof(E);
  const E* p;
  int V, nit, base;
  u32x4 v[NV > 0 ? NV : 1];

  __device__ __forceinline__ Row(const E* p_, int V_, int nit_) : p(p_), V(V_), nit(nit_) {
    base = ((threadIdx.x >> 6) * nit * 64 + (threadIdx.x & 63)) * EPV;
    if constexpr (NV > 0) {
#pragma unroll
      for (int it = 0; it < NV; ++it)
        if (it < nit) v[it] = read(it);
    }
  }
  __device__ __forceinline__ int at(int it) const { return base + it * 64 * EPV; }
  __device__ __forceinline__ u32x4 read(int it) const {
    const int i = at(it);
    if (i + EPV <= V) return load_vec(p + i);
    u32x4 x;
    if constexpr (sizeof(E) == 2) {
      uint32_t b[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) b[e] = i + e < V ? (uint32_t)p[i + e] : 0xff80u;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = b[2 * k] | (b[2 * k + 1] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < EPV; ++e) x[e] = i + e < V ? __float_as_uint(p[i + e]) : 0xff800000u;
    }
    return x;
  }
  // f(vector, index of its first logit)
  template <typename F>
  __device__ __forceinline__ void vectors(F f) const {
    if constexpr (NV > 0) {
#pragma unroll
      for (int it = 0; it < NV; ++it)
        if (it < nit) f(v[it], at(it));
    } else {
      for (int it = 0; it < nit; it += 4) {
        u32x4 b[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (it + k < nit) b[k] = read(it + k);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (it + k < nit) f(b[k], at(it + k));
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    vectors([&](const u32x4& x, int i) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) f(vec_elem<E>(x, e), i + e);
    });
  }
  // f(z, index) where some lane's vector reaches zlo; f decides by itself
  template <typename F>
  __device__ __forceinline__ void each_from(float zlo, F f) const {
    vectors([&](const u32x4& x, int i) {
      float m = vec_elem<E>(x, 0);
#pragma unroll
      for (int e = 1; e < EPV; ++e) m = fmaxf(m, vec_elem<E>(x, e));
      if (__ballot(m >= zlo)) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) f(vec_elem<E>(x, e), i + e);
      }
    });
  }
  __device__ __forceinline__ Row<E, 0> streamed() const { return Row<E, 0>(p, V, nit); }
};

// The candidates in LDS.
struct Candidates {
  int n;
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    const FilterShared& sh = shared();
    for (int i = threadIdx.x; i < n; i += FT) f(sh.lz[i], sh.li[i]);
  }
};

// ---------------------------------------------------------------------------
// over the workgroup
// ---------------------------------------------------------------------------

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

__device__ __forceinline__ void block_min_max(float& lo, float& hi) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    lo = fminf(lo, __shfl_xor(lo, off));
    hi = fmaxf(hi, __shfl_xor(hi, off));
  }
  if (lane == 0) { sh.f[wv] = lo; sh.g[wv] = hi; }
  __syncthreads();
  for (int i = 0; i < FW; ++i) { lo = fminf(lo, sh.f[i]); hi = fmaxf(hi, sh.g[i]); }
  __syncthreads();
}

// Inclusive scan over the workgroup of (count, mass), in thread order.
__device__ __forceinline__ void scan_bins(uint32_t& c, unsigned long long& m) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint32_t oc = __shfl_up(c, off);
    const unsigned long long om = __shfl_up(m, off);
    if (lane >= off) { c += oc; m += om; }
  }
  if (lane == 63) { sh.c[w] = c; sh.u[w] = m; }
  __syncthreads();
  uint32_t bc = 0;
  unsigned long long bm = 0;
  for (int i = 0; i < w; ++i) { bc += sh.c[i]; bm += sh.u[i]; }
  c += bc;
  m += bm;
  __syncthreads();
}

// Smallest index of a thread for which `yes` holds, `none` without one.
__device__ __forceinline__ int first_index(bool yes, int i, int none) {
  FilterShared& sh = shared();
  if (threadIdx.x == 0) sh.found = 0x7fffffff;
  __syncthreads();
  if (yes) atomicMin(&sh.found, i);
  __syncthreads();
  const int got = sh.found;
  __syncthreads();
  return got == 0x7fffffff ? none : got;
}

// Smallest index whose running weight (index order) exceeds t, given each
// wave's range sum in sh.d; the last index of positive weight when rounding
// (or u = 1) puts t past the sum; -1 when every weight is zero.  fn(z, i) is
// the weight of token i.
template <typename E, int NV, typename F>
__device__ int pick_index(const Row<E, NV>& row, F fn, double t) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int w = -1, last = -1;
  double excl = 0.0, run = 0.0;
  for (int i = 0; i < FW; ++i) {
    const double s = sh.d[i];
    if (s > 0.0) {
      last = i;
      if (w < 0 && run + s > t) { w = i; excl = run; }
      if (w < 0) run += s;
    }
  }
  if (last < 0) return -1;
  if (w < 0) { w = last; t = INFINITY; }
  // the range's vectors, one per thread and nit / FW more
  constexpr int EPV = Row<E, NV>::EPV;
  const int span = row.nit * 64 * EPV, lo = w * span, hi = min(row.V, lo + span);
  const int per = (row.nit + FW - 1) / FW * EPV;
  const int first = lo + tid * per;
  double part = 0.0;
  int lastpos = -1;
  auto walk = [&](auto&& f) {            // this thread's tokens, in index order
    for (int i0 = first; i0 < min(hi, first + per); i0 += EPV) {
      float z[EPV];
#pragma unroll
      for (int e = 0; e < EPV; ++e) z[e] = i0 + e < hi ? load_logit(row.p + i0 + e) : -INFINITY;
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        if (i0 + e < hi && f(fn(z[e], i0 + e), i0 + e)) return;
    }
  };
  walk([&](double x, int i) {
    part += x;
    if (x > 0.0) lastpos = i;
    return false;
  });
  double incl = part;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  double before = __shfl_up(incl, 1);
  if (lane == 0) before = 0.0;
  __syncthreads();                       // sh.d has been read by every thread
  if (lane == 63) sh.d[wv] = incl;
  if (tid == 0) { sh.pick[0] = 0x7fffffff; sh.pick[1] = -1; }
  __syncthreads();
  double base = excl;
  for (int i = 0; i < wv; ++i) base += sh.d[i];
  if (part > 0.0 && base + incl > t) {   // the first such thread holds the token
    double acc = base + before;
    int at = lastpos;
    walk([&](double x, int i) {
      acc += x;
      if (acc > t) at = i;
      return acc > t;
    });
    atomicMin(&sh.pick[0], at);
  }
  if (lastpos >= 0) atomicMax(&sh.pick[1], lastpos);
  __syncthreads();
  const int got = sh.pick[0] != 0x7fffffff ? sh.pick[0] : sh.pick[1];
  __syncthreads();
  return got;
}

// Every wave's range sum to sh.d; returns their sum, in order.
__device__ __forceinline__ double range_sums(double part) {
  FilterShared& sh = shared();
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  part = wave_sum(part);
  __syncthreads();
  if (lane == 0) sh.d[wv] = part;
  __syncthreads();
  double total = 0.0;
  for (int i = 0; i < FW; ++i) total += sh.d[i];
  return total;
}

// ---------------------------------------------------------------------------
// the cut
// ---------------------------------------------------------------------------

struct Cut {
  float z;
  int idx;
  unsigned long long mass;   // fixed-point weight through the cut
};

__device__ __forceinline__ unsigned long long fixed_weight(float z, const RowCut& c, double scale) {
  return (unsigned long long)(weight(z, c) * scale + 0.5);
}

// Bins over [zlo, zhi], the largest logits first: linear ones, which spread a
// row's logits well, or ones of the numbers' ordered keys, which end at single
// values whatever the spread.
struct Binning {
  float half, sc;
  uint32_t khi;
  int shift;
  bool linear;
  __device__ __forceinline__ Binning(float zhi, float zlo, bool lin) : linear(lin) {
    half = zhi * 0.5f;
    sc = fminf((float)BINS / (half - zlo * 0.5f), 3.0e38f);
    khi = order_key(zhi);
    shift = max(0, 22 - __clz(khi - order_key(zlo)));
  }
  __device__ __forceinline__ int operator()(float z) const {
    if (linear) return (int)fminf((half - z * 0.5f) * sc, (float)(BINS - 1));
    return (int)((khi - order_key(z)) >> shift);
  }
};

// The last token kept when the tokens of `src` with zlo <= z <= zhi (n of
// them, in order) are kept up to the k-th (by_mass false), or up to the first
// at which the weight reaches `target` (by_mass true; the last one if none
// does).  Weights are summed only when `masses` is set.
template <typename Src, typename E>
__device__ Cut select_cut(const Src& src, const Row<E, 0>& row, const RowCut& rc, double scale,
                          int n, float zhi, float zlo, bool by_mass, bool masses, uint32_t k,
                          double target) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x;
  uint32_t above_c = 0;
  unsigned long long above_m = 0;
  for (int level = 0; n > RANK && zlo < zhi; ++level) {
    const Binning bin(zhi, zlo, level == 0);
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
    n = sh.n;
    above_c += sh.fc;
    above_m += sh.fm;
    float lo = INFINITY, hi = -INFINITY;
    src.each([&](float z, int) {
      if (z <= zhi && z >= zlo && bin(z) == b) { lo = fminf(lo, z); hi = fmaxf(hi, z); }
    });
    block_min_max(lo, hi);
    zlo = lo;
    zhi = hi;
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
    auto one = [&](float z, int) { return z == zhi ? 1.0 : 0.0; };
    double part = 0.0;
    row.each([&](float z, int i) { part += one(z, i); });
    range_sums(part);
    cut.z = zhi;
    cut.idx = pick_index(row, one, (double)keep - 0.5);
    cut.mass = above_m + w * (unsigned long long)keep;
    return cut;
  }
  // rank what is left (at most RANK tokens), in the histogram's memory
  float* lz = (float*)sh.cnt;
  int* li = (int*)sh.cnt + RANK;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  src.each([&](float z, int i) {
    if (z <= zhi && z >= zlo) {
      const int at = atomicAdd(&sh.n, 1);
      if (at < RANK) { lz[at] = z; li[at] = i; }
    }
  });
  __syncthreads();
  n = min(sh.n, RANK);
  float z = 0.f;
  int idx = 0, rank = 0;
  if (tid < n) {
    z = lz[tid];
    idx = li[tid];
    for (int j = 0; j < n; ++j) {
      const float oz = lz[j];
      rank += oz > z || (oz == z && li[j] < idx);
    }
    sh.mass[rank] = masses ? fixed_weight(z, rc, scale) : 0;
  }
  __syncthreads();
  uint32_t c = tid < n;
  unsigned long long m = tid < n ? sh.mass[tid] : 0;
  scan_bins(c, m);
  const bool here = by_mass ? (double)(above_m + m) >= target : above_c + c >= k;
  const int at = first_index(tid < n && here, tid, n - 1);
  if (tid < n && rank == at) { sh.f[0] = z; sh.n = idx; }
  if (tid == at) sh.fm = m;
  __syncthreads();
  cut.z = sh.f[0];
  cut.idx = sh.n;
  cut.mass = above_m + sh.fm;
  __syncthreads();
  return cut;
}

// The draw among the kept tokens, given each wave's kept weight in sh.d;
// sh.token and sh.w (its weight).
template <typename E>
__device__ __noinline__ void draw_kept(const E* p, int V, int nit, float u) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const Row<E, 0> row(p, V, nit);
  const int t = pick_index(row, [&](float z, int i) { return kept_weight(z, i, rc); },
                           (double)u * rc.total);
  if (threadIdx.x == 0) {
    sh.token = t;
    sh.w = t < 0 ? 0.0 : kept_weight(load_logit(p + t), t, rc);
  }
  __syncthreads();
}

// Cut, kept weight and draw in general; n tokens reach `bound`, in LDS if they
// are at most LIST.  whole: weight that top-p is a share of, < 0: of the kept
// by top-k.  u < 0: no draw.
template <typename E>
__device__ __noinline__ void filter_general(const E* p, int V, int nit, int n, float bound, int k,
                                            double top_p, double whole, float u) {
  FilterShared& sh = shared();
  RowCut rc = sh.rc;
  const Row<E, 0> row(p, V, nit);
  const Candidates list{n};
  const float hi = rc.zmax;
  const double scale = ldexp(1.0, __clz(V) + 30);   // V * scale <= 2^62
  const bool need_p = top_p < 1.0;
  whole *= scale;
  for (int step = k < n ? 0 : 1; step < (need_p ? 2 : 1); ++step) {   // top-k, top-p
    if (step && whole < 0.0) {                      // top-k keeps all
      double part = 0.0;
      row.each([&](float z, int) { part += weight(z, rc); });
      whole = range_sums(part) * scale;
    }
    const double target = fmax(top_p, 0.0) * whole;
    const Cut c = n <= LIST ? select_cut(list, row, rc, scale, n, hi, bound, step == 1, need_p,
                                         (uint32_t)k, target)
                            : select_cut(row, row, rc, scale, n, hi, bound, step == 1, need_p,
                                         (uint32_t)k, target);
    if (c.z > rc.z || (c.z == rc.z && c.idx < rc.idx)) { rc.z = c.z; rc.idx = c.idx; }
    if (!step) whole = (double)c.mass;
  }
  double part = 0.0;
  row.each_from(rc.z, [&](float z, int i) { part += kept_weight(z, i, rc); });
  rc.total = range_sums(part);
  if (threadIdx.x == 0) sh.rc = rc;
  __syncthreads();
  if (u >= 0.0f) draw_kept(p, V, nit, u);
}

// Shortens a list of RANK < n <= LIST candidates to those in the histogram
// bins up to the one that holds the k-th token, or (by_mass) in which the
// weight reaches `target`.  Returns how many they are; n, and the list as it
// was, if more than RANK.
__device__ __noinline__ int shorten_list(int n, float bound, bool by_mass, int k, double target) {
  FilterShared& sh = shared();
  const RowCut rc = sh.rc;
  const int tid = threadIdx.x;
  const double scale = 562949953421312.0;      // 2^49: LIST weights stay below 2^63
  const Binning bin(rc.zmax, bound, true);
  sh.cnt[tid] = 0;
  sh.mass[tid] = 0;
  __syncthreads();
  float z[LIST / FT];
  int idx[LIST / FT];
#pragma unroll
  for (int j = 0; j < LIST / FT; ++j) {
    const int i = j * FT + tid;
    if (i < n) {
      z[j] = sh.lz[i];
      idx[j] = sh.li[i];
      const int b = bin(z[j]);
      atomicAdd(&sh.cnt[b], 1u);
      if (by_mass) atomicAdd(&sh.mass[b], fixed_weight(z[j], rc, scale));
    }
  }
  __syncthreads();
  uint32_t c = sh.cnt[tid];
  unsigned long long m = sh.mass[tid];
  scan_bins(c, m);
  // (a target past every weight by rounding: the last bin)
  const int b = first_index(by_mass ? (double)m >= target * scale : c >= (uint32_t)k, tid, BINS - 1);
  if (tid == b) sh.found = (int)c;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  const int left = sh.found;
  __syncthreads();
  if (left > RANK) return n;
#pragma unroll
  for (int j = 0; j < LIST / FT; ++j) {
    const int i = j * FT + tid;
    if (i < n && bin(z[j]) <= b) {
      const int at = atomicAdd(&sh.n, 1);
      sh.lz[at] = z[j];
      sh.li[at] = idx[j];
    }
  }
  __syncthreads();
  return left;
}

// All cuts and the draw over the n <= RANK candidates in LDS: each thread
// counts the candidates ahead of its own; sorted by that rank, a scan of the
// weights gives the prefixes.  Kept tokens then find their running weight in
// index order by another count.  k: tokens kept by top-k (n: all); top_p < 1:
// top-p of `whole` (< 0: of the k tokens').  u < 0: no draw.
__device__ __noinline__ void rank_cut(int n, int k, double top_p, double whole, float u) {
  FilterShared& sh = shared();
  RowCut rc = sh.rc;
  const int tid = threadIdx.x;
  const double scale = 9007199254740992.0;     // 2^53: RANK weights stay below 2^63
  unsigned long long* key = sh.mass;           // larger logit, then lower index, first
  unsigned long long* w = sh.mass + RANK;      // by rank
  float z = 0.f;
  int idx = 0;
  unsigned long long mine = 0, own = 0;
  bool big = false;
  double x = 0.0;
  if (tid < n) {
    z = sh.lz[tid];
    idx = sh.li[tid];
    x = weight(z, rc);
    big = x >= (double)rc.min_w;
    own = x > 0.0 ? max((unsigned long long)(x * scale + 0.5), 1ull) : 0ull;
    mine = ((unsigned long long)order_key(z) << 32) | (uint32_t)~idx;
    key[tid] = mine;
  }
  __syncthreads();
  int rank = 0;
  if (tid < n) {
#pragma unroll 4
    for (int j = 0; j < n; ++j) rank += key[j] > mine;
    w[rank] = own;
  }
  __syncthreads();
  uint32_t c = tid < n;
  unsigned long long m = tid < n ? w[tid] : 0;
  scan_bins(c, m);
  int keep = k;
  if (top_p < 1.0) {
    if (tid == k - 1) sh.fm = m;
    __syncthreads();
    const double target = fmax(top_p, 0.0) * (whole < 0.0 ? (double)sh.fm : whole * scale);
    keep = first_index(tid < k && (double)m >= target, tid, k - 1) + 1;
  }
  const bool kept = tid < n && rank < keep && (big || rank == 0);
  if (tid < n) w[tid] = kept ? own : 0;        // now by candidate
  if (tid < n && rank == keep - 1) { sh.rc.z = z; sh.rc.idx = idx; }
  if (tid == 0) { sh.pick[0] = 0x7fffffff; sh.pick[1] = -1; }
  __syncthreads();
  unsigned long long all = 0, run = 0;
  if (kept || tid == 0) {
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const unsigned long long o = w[j];
      all += o;
      run += (int)~(uint32_t)key[j] <= idx ? o : 0;
    }
    if (tid == 0) sh.rc.total = (double)all / scale;
    if (u >= 0.0f && kept && own > 0) {
      if ((double)run > (double)u * (double)all) atomicMin(&sh.pick[0], idx);
      atomicMax(&sh.pick[1], idx);
    }
  }
  __syncthreads();
  const int token = sh.pick[0] != 0x7fffffff ? sh.pick[0] : sh.pick[1];
  if (kept && idx == token) { sh.token = token; sh.w = x; }
  __syncthreads();
}

// A logit that at least k tokens of the row reach: the k-th largest of the
// threads' own maxima is one; here the smallest of those in the histogram bins
// up to the one where their count reaches k.
__device__ __forceinline__ float count_bound(float mine, float hi, uint32_t k) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x;
  const bool any = mine > -INFINITY;
  float lo = any ? mine : INFINITY, top = hi;
  block_min_max(lo, top);
  if (!(lo < hi)) return -INFINITY;
  const Binning bin(hi, lo, true);
  sh.cnt[tid] = 0;
  __syncthreads();
  const int b = any ? bin(mine) : BINS;
  if (any) atomicAdd(&sh.cnt[b], 1u);
  __syncthreads();
  uint32_t c = sh.cnt[tid];
  unsigned long long none = 0;
  scan_bins(c, none);
  const int at = first_index(c >= k, tid, -1);
  if (at < 0) return -INFINITY;                // fewer threads than k hold a logit
  lo = b <= at ? mine : INFINITY;
  top = hi;
  block_min_max(lo, top);
  return lo;
}

// Reads a row, finds what its filters keep (sh.rc) and, for u >= 0, draws a
// token (sh.token, sh.w: its weight).
template <typename E, int NV>
__device__ __forceinline__ void filter_row(const Row<E, NV>& row, const RowParams& par, int pi,
                                           float u, int32_t* err) {
  FilterShared& sh = shared();
  const int tid = threadIdx.x, V = row.V;
  const float T = par.temperature ? par.temperature[pi] : 1.0f;
  const int k = par.top_k ? par.top_k[pi] : 0;
  const double top_p = par.top_p ? (double)par.top_p[pi] : 1.0;
  float hi = -INFINITY, lo = INFINITY;
  bool bad = false;
  row.each([&](float z, int) {
    bad |= !(z < INFINITY);
    hi = fmaxf(hi, z);
    lo = fminf(lo, z > -INFINITY ? z : INFINITY);
  });
  const float mine = hi;
  if (bad) set_err(err, DVS_ERR_NONFINITE);
  block_min_max(lo, hi);

  RowCut rc;
  rc.zmax = hi;
  rc.z = -INFINITY;
  rc.idx = 0x7fffffff;
  rc.min_w = par.min_p ? par.min_p[pi] : 0.0f;
  if (!(rc.min_w > 0.0f)) rc.min_w = 0.0f;
  rc.log2e_t = 1.4426950408889634 / (double)T;
  rc.total = 0.0;
  rc.single = 0;
  const bool empty = hi == -INFINITY;
  if (empty && tid == 0) set_err(err, DVS_ERR_NONFINITE);
  if (!(T > 0.0f) || k == 1 || rc.min_w > 1.0f || empty || hi == INFINITY) {
    // top-1: the lowest index of the maximum
    int at = 0x7fffffff;
    row.each([&](float z, int i) { if (z == hi && i < V) at = min(at, i); });
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
  const bool need_k = k > 0 && k < V, need_p = top_p < 1.0;
  float bound = lo;                            // tokens below are not kept
  if (rc.min_w > 0.0f && !(need_k && need_p)) {
    // w < min_p surely, whatever the roundings on the way
    const double d = (double)T * log((double)rc.min_w);
    bound = fmaxf(bound, (float)((double)hi + d * (1.0 + 1e-6)) - fabsf(hi) * 1e-6f);
  }
  double whole = -1.0;
  if (need_k) {
    if (k <= FT) bound = fmaxf(bound, count_bound(mine, hi, (uint32_t)k));
  } else {
    // the whole weight: for top-p, and as the kept weight where nothing cuts
    const double least = need_p ? 0.0 : (double)rc.min_w;
    double part = 0.0;
    row.each_from(need_p ? lo : bound, [&](float z, int) {
      const double w = weight(z, rc);
      part += w >= least ? w : 0.0;
    });
    whole = range_sums(part);
    if (!need_p) {
      rc.z = bound;
      rc.total = whole;
      if (tid == 0) sh.rc = rc;
      __syncthreads();
      if (u >= 0.0f) draw_kept(row.p, V, row.nit, u);
      return;
    }
    // tokens of less than (1 - p) / V of the weight each cannot hold 1 - p of it
    const double d = (double)T * log((1.0 - fmax(top_p, 0.0)) * whole / (double)V);
    bound = fmaxf(bound, (float)((double)hi + d * (1.0 + 1e-6)) - fabsf(hi) * 1e-6f);
  }
  if (tid == 0) { sh.n = 0; sh.rc = rc; }
  __syncthreads();
  row.each_from(bound, [&](float z, int i) {
    const unsigned long long m = __ballot(z >= bound);
    if (m) {
      const int lane = tid & 63, leader = __ffsll((long long)m) - 1;
      int first = 0;
      if (lane == leader) first = atomicAdd(&sh.n, (int)__popcll(m));
      const int at = __shfl(first, leader) + __popcll(m & ((1ull << lane) - 1));
      if (z >= bound && at < LIST) { sh.lz[at] = z; sh.li[at] = i; }
    }
  });
  __syncthreads();
  int n = sh.n;
  __syncthreads();
  const int kk = need_k ? min(k, n) : n;
  if (n > RANK && n <= LIST && kk <= RANK)
    n = shorten_list(n, bound, false, kk, 0.0);
  else if (n > RANK && n <= LIST && !need_k)
    n = shorten_list(n, bound, true, 0, fmax(top_p, 0.0) * whole);
  if (n <= RANK)
    rank_cut(n, min(kk, n), need_p ? top_p : 1.0, whole, u);
  else
    filter_general(row.p, V, row.nit, n, bound, kk, need_p ? top_p : 1.0, whole, u);
}

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------

template <typename E, int NV>
__global__ void __launch_bounds__(FT) sample_filtered_kernel(
    const E* __restrict__ logits, long long ld, int V, int nit, RowParams par, int rows_per_param,
    const float* __restrict__ u, int u_stride, int32_t* __restrict__ token_out,
    float* __restrict__ prob_out, int32_t* err) {
  FilterShared& sh = shared();
  const int r = blockIdx.x, s = r / rows_per_param;
  const Row<E, NV> row(logits + (size_t)r * ld, V, nit);
  float uu = u[(size_t)s * u_stride + (r - s * rows_per_param)];
  if (!(uu > 0.0f)) uu = 0.0f;
  filter_row(row, par, s, uu, err);
  if (threadIdx.x == 0) {
    token_out[r] = sh.token;
    if (prob_out) prob_out[r] = sh.rc.total > 0.0 ? (float)(sh.w / sh.rc.total) : 0.0f;
  }
}

// Cuts of the verify rows (first S * (B + 1)) and draft rows (S * B) of a call.
template <typename E, int NV>
__global__ void __launch_bounds__(FT) filter_rows_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int B, int nv, int V, int nit, RowParams par, RowCut* __restrict__ cuts,
    int32_t* err) {
  const int r = blockIdx.x;
  const int per = r < nv ? B + 1 : B, i = r < nv ? r : r - nv;
  const int s = i / per, j = i - s * per;
  const E* z = r < nv ? zv + (size_t)s * vs + (size_t)j * vld : zd + (size_t)s * ds + (size_t)j * dld;
  const Row<E, NV> row(z, V, nit);
  filter_row(row, par, s, -1.0f, err);
  if (threadIdx.x == 0) cuts[r] = shared().rc;
}

__device__ __forceinline__ double prob_of(float z, int i, const RowCut& c) {
  if (c.single) return c.single > 0 && i == c.idx ? 1.0 : 0.0;
  const double w = kept_weight(z, i, c);
  return w > 0.0 ? w / c.total : 0.0;
}

// One workgroup per sequence: d_j accepted while u q_j(d_j) < p_j(d_j), then
// the final token from max(0, p - q) of the rejected draft's rows, or from the
// last verify row.
template <typename E>
__global__ void __launch_bounds__(FT) accept_filtered_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int S, int B, int V, int nit, const RowCut* __restrict__ cuts,
    const int32_t* __restrict__ draft, int draft_width, const float* __restrict__ u, int u_stride,
    int32_t* __restrict__ accept_len, int32_t* __restrict__ token_out, int token_stride,
    int at_accepted) {
  FilterShared& sh = shared();
  const int s = blockIdx.x, tid = threadIdx.x;
  const RowCut* cv = cuts + (size_t)s * (B + 1);
  const RowCut* cd = cuts + (size_t)S * (B + 1) + (size_t)s * B;
  const E* v = zv + (size_t)s * vs;
  const E* d = zd + (size_t)s * ds;
  if (tid == 0) sh.found = B;
  __syncthreads();
  for (int j = tid; j < B; j += FT) {    // the first rejected draft
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
  const Row<E, 0> row(v + (size_t)A * vld, V, nit);
  auto alone = [&](float z, int i) { return i < V ? prob_of(z, i, p) : 0.0; };
  int t = -1;
  if (A < B) {
    const RowCut q = cd[A];
    const E* zq = d + (size_t)A * dld;
    auto rest = [&](float z, int i) {
      const double a = alone(z, i);
      return a > 0.0 ? fmax(a - prob_of(load_logit(zq + i), i, q), 0.0) : 0.0;
    };
    double part = 0.0;
    row.each_from(p.z, [&](float z, int i) { part += rest(z, i); });
    const double total = range_sums(part);
    t = pick_index(row, rest, (double)uu * total);
  }
  if (t < 0) {                           // all accepted, or p and q equal to the last bit
    double part = 0.0;
    row.each_from(p.z, [&](float z, int i) { part += alone(z, i); });
    const double total = range_sums(part);
    t = pick_index(row, alone, (double)uu * total);
  }
  if (t < 0) t = max(p.idx, 0);          // a row without a number above -inf
  if (tid == 0) {
    accept_len[s] = A;
    token_out[(size_t)s * token_stride + (at_accepted ? A : 0)] = t;
  }
}

size_t filter_cuts_bytes(int S, int B) { return (size_t)S * (2 * B + 1) * sizeof(RowCut); }

// Calls f(integral constant NV) with the vectors per lane that hold a row of
// nit: a workgroup of more registers than the row needs would spill nothing
// but leave the loops over absent vectors in.  0: the row is read again by
// each pass.
template <typename E, typename F>
static void by_vectors(int V, F f) {
  const int per = FT * 16 / (int)sizeof(E), nit = (V + per - 1) / per;
  constexpr int MOST = sizeof(E) == 4 ? 16 : 8;
  if (nit <= 1) f(IC<1>{}, nit);
  else if (nit <= 4) f(IC<4>{}, nit);
  else if (nit <= MOST) f(IC<MOST>{}, nit);
  else f(IC<0>{}, nit);
}

template <typename E>
static int launch_accept(const void* zv, long long vs, long long vld, const void* zd, long long ds,
                         long long dld, int S, int B, int V, const RowParams& par,
                         const int32_t* draft, int draft_width, const float* u, int u_stride,
                         int32_t* accept_len, int32_t* token_out, int token_stride,
                         int at_accepted, int32_t* err, void* ws, hipStream_t st) {
  RowCut* cuts = (RowCut*)ws;
  by_vectors<E>(V, [&](auto nv, int nit) {
    constexpr int NV = decltype(nv)::value;
    hipLaunchKernelGGL((filter_rows_kernel<E, NV>), dim3(S * (2 * B + 1)), dim3(FT), 0, st,
                       (const E*)zv, vs, vld, (const E*)zd, ds, dld, B, S * (B + 1), V, nit, par,
                       cuts, err);
    hipLaunchKernelGGL(accept_filtered_kernel<E>, dim3(S), dim3(FT), 0, st, (const E*)zv, vs,
                       vld, (const E*)zd, ds, dld, S, B, V, nit, cuts, draft, draft_width, u,
                       u_stride, accept_len, token_out, token_stride, at_accepted);
  });
  return launch_status("accept_sampled");
}

template <typename E>
static void launch_sample(const void* logits, int rows, int V, long long ld, const RowParams& par,
                          int rows_per_param, const float* u, int u_stride, int32_t* token_out,
                          float* prob_out, int32_t* err, hipStream_t st) {
  by_vectors<E>(V, [&](auto nv, int nit) {
    constexpr int NV = decltype(nv)::value;
    hipLaunchKernelGGL((sample_filtered_kernel<E, NV>), dim3(rows), dim3(FT), 0, st,
                       (const E*)logits, ld, V, nit, par, rows_per_param, u, u_stride, token_out,
                       prob_out, err);
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
  DVS_CHECK_ARG(rows >= 1 && V >= 1 && V <= (1 << 30), "sample_filtered: need rows >= 1 and 1 <= V <= 2^30");
  DVS_CHECK_ARG(ld >= V, "sample_filtered: row stride %lld < V", (long long)ld);
  DVS_CHECK_ARG(rows_per_param >= 1 && rows % rows_per_param == 0,
                "sample_filtered: rows (%d) must be groups of rows_per_param (%d)", rows,
                rows_per_param);
  return launch_sample_filtered(logits, dtype, rows, V, ld, RowParams{temperature, top_k, top_p, min_p},
                                rows_per_param, u, rows_per_param, token_out, prob_out, err_word,
                                (hipStream_t)stream);
}

extern "C" size_t dvs_accept_workspace_bytes(int32_t S, int32_t B, int32_t V) {
  if (S < 1 || B < 1 || V < 1 || V > (1 << 30)) return 0;
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
  DVS_CHECK_ARG(S >= 1 && B >= 1 && V >= 1 && V <= (1 << 30),
                "accept_sampled: need S, B >= 1 and 1 <= V <= 2^30");
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
