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
// the row, so the ranges' sums are in index order:
//   1. maximum, minimum and count of the finite logits;
//   2. the cut (select_cut): a histogram over the logit range with a count and
//      a weight sum per bin, the bin that holds the k-th token or the share p
//      of the weight, narrowed until few tokens are left, and these ranked;
//   3. the sums of the kept weights per range, the range that holds u * total,
//      and one scan over that range's tokens.
// The histogram's weights are fixed-point integers, so its atomics give the
// same sums in any order; the sums of step 3 have a fixed order.  Results do
// not depend on timing, nor on the other rows of the call.
#include <math.h>

#include "dvs_common.h"

namespace dvs {

constexpr int FT = 1024;          // threads of a row's workgroup
constexpr int FW = FT / 64;
constexpr int BINS = 1024;        // one histogram bin per thread
constexpr int RANK = 512;         // tokens that are ranked against each other

// What a row's filters keep.  total = 0: not yet summed.
struct RowCut {
  float zmax, z;     // largest logit; the cut's
  int idx;           // the cut's index among equal logits
  float min_w;       // min_p
  double inv_t, total;
};

struct FilterShared {
  uint32_t cnt[BINS];
  unsigned long long mass[BINS];
  float lz[RANK];
  int li[RANK];
  unsigned long long lw[RANK];
  double d[FW];
  unsigned long long u[FW];
  uint32_t c[FW];
  float f[FW], g[FW];
  int pick[2];
  int found, n;
  uint32_t fc;
  unsigned long long fm;
};

// exp((z - zmax) / T): 1 at the maximum (also an infinite one), 0 for a masked
// logit (-inf).
__device__ __forceinline__ double weight(float z, const RowCut& c) {
  if (z == c.zmax) return 1.0;
  if (z == -INFINITY) return 0.0;
  return exp(((double)z - (double)c.zmax) * c.inv_t);
}

__device__ __forceinline__ bool before_cut(float z, int idx, const RowCut& c) {
  return z > c.z || (z == c.z && idx <= c.idx);
}

__device__ __forceinline__ double kept_weight(float z, int idx, const RowCut& c) {
  if (!before_cut(z, idx, c)) return 0.0;
  const double w = weight(z, c);
  return w >= (double)c.min_w ? w : 0.0;
}

__device__ __forceinline__ float load_logit(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float load_logit(const uint16_t* p, int i) { return bf16_bits_to_f32(p[i]); }

// Order-preserving key of a number (-0 as +0).
__device__ __forceinline__ uint32_t order_key(float z) {
  uint32_t u = __float_as_uint(z);
  if ((u & 0x7fffffffu) == 0) u = 0;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// A wave's contiguous range of a row.
struct Range {
  int lo, hi;
};

__device__ __forceinline__ Range wave_range(int V, int w) {
  const int per = ((V + FW - 1) / FW + 63) & ~63;
  Range r;
  r.lo = min(V, w * per);
  r.hi = min(V, r.lo + per);
  return r;
}

// ---------------------------------------------------------------------------
// sums over the workgroup
// ---------------------------------------------------------------------------

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Inclusive scan over the workgroup of (count, mass), in thread order.
__device__ __forceinline__ void scan_bins(uint32_t& c, unsigned long long& m, FilterShared& sh) {
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

// Smallest index whose running weight (index order) exceeds t, given each
// wave's range sum in sh.d; the last index of positive weight when rounding
// (or u = 1) puts t past the sum; -1 when every weight is zero.  fn(i) is the
// weight of token i.
template <typename F>
__device__ int pick_index(F fn, int V, double t, FilterShared& sh) {
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
  if (w < 0) { w = last; excl = -1.0; t = INFINITY; }
  const Range r = wave_range(V, w);
  const int per = (r.hi - r.lo + FT - 1) / FT;
  const int lo = min(r.hi, r.lo + tid * per), hi = min(r.hi, lo + per);
  double part = 0.0;
  int lastpos = -1;
  for (int i = lo; i < hi; ++i) {
    const double x = fn(i);
    part += x;
    if (x > 0.0) lastpos = i;
  }
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
  double base = excl < 0.0 ? 0.0 : excl;
  for (int i = 0; i < wv; ++i) base += sh.d[i];
  if (part > 0.0 && base + incl > t) {   // the first such thread holds the token
    double acc = base + before;
    int at = lastpos;
    for (int i = lo; i < hi; ++i) {
      acc += fn(i);
      if (acc > t) { at = i; break; }
    }
    atomicMin(&sh.pick[0], at);
  }
  if (lastpos >= 0) atomicMax(&sh.pick[1], lastpos);
  __syncthreads();
  const int got = sh.pick[0] != 0x7fffffff ? sh.pick[0] : sh.pick[1];
  __syncthreads();
  return got;
}

// Sums fn over every wave's range into sh.d; returns their sum, in order.
template <typename F>
__device__ double range_sums(F fn, int V, FilterShared& sh) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const Range r = wave_range(V, wv);
  double part = 0.0;
  for (int i = r.lo + lane; i < r.hi; i += 64) part += fn(i);
  part = wave_sum(part);
  __syncthreads();
  if (lane == 0) sh.d[wv] = part;
  __syncthreads();
  double total = 0.0;
  for (int i = 0; i < FW; ++i) total += sh.d[i];
  return total;
}

// The r-th lowest index (r >= 1) whose logit equals z; -1 when there is none.
template <typename E>
__device__ int nth_equal(const E* row, int V, float z, int r, FilterShared& sh) {
  auto one = [&](int i) { return load_logit(row, i) == z ? 1.0 : 0.0; };
  range_sums(one, V, sh);
  return pick_index(one, V, (double)r - 0.5, sh);
}

// ---------------------------------------------------------------------------
// the cut
// ---------------------------------------------------------------------------

struct Cut {
  float z;
  int idx;
  unsigned long long mass;   // fixed-point weight through the cut
};

// Fixed-point weight: sums of V of them stay below 2^63.
__device__ __forceinline__ unsigned long long fixed_weight(float z, const RowCut& c, double scale) {
  return (unsigned long long)(weight(z, c) * scale + 0.5);
}

// The last token kept when the tokens with zlo <= z <= zhi (n of them, in
// order) are kept up to the k-th (by_mass false), or up to the first at which
// the weight reaches `target` (by_mass true; the last one if none does).
// Weights are summed only when `masses` is set.
template <typename E>
__device__ Cut select_cut(const E* row, int V, const RowCut& rc, double scale, int n, float zhi,
                          float zlo, bool by_mass, bool masses, uint32_t k, double target,
                          FilterShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  uint32_t above_c = 0;
  unsigned long long above_m = 0;
  const Range r = wave_range(V, wv);
  for (int level = 0; n > RANK && zlo < zhi; ++level) {
    // first linear bins, which spread a row's logits well; then bins of the
    // numbers' ordered keys, which end at single values whatever the spread
    const float half = zhi * 0.5f;
    const float sc = fminf((float)BINS / (half - zlo * 0.5f), 3.0e38f);
    const uint32_t khi = order_key(zhi), span = khi - order_key(zlo);
    const int shift = max(0, 22 - __clz(span));
    auto bin = [&](float z) -> int {
      if (level == 0) return (int)fminf((half - z * 0.5f) * sc, (float)(BINS - 1));
      return (int)((khi - order_key(z)) >> shift);
    };
    sh.cnt[tid] = 0;
    sh.mass[tid] = 0;
    __syncthreads();
    for (int i = r.lo + lane; i < r.hi; i += 64) {
      const float z = load_logit(row, i);
      if (z <= zhi && z >= zlo) {
        const int b = bin(z);
        atomicAdd(&sh.cnt[b], 1u);
        if (masses) atomicAdd(&sh.mass[b], fixed_weight(z, rc, scale));
      }
    }
    __syncthreads();
    const uint32_t own_c = sh.cnt[tid];
    uint32_t c = own_c;
    unsigned long long m = sh.mass[tid];
    const unsigned long long own_m = m;
    scan_bins(c, m, sh);
    if (tid == 0) sh.found = 0x7fffffff;
    __syncthreads();
    const bool here = by_mass ? (double)(above_m + m) >= target : above_c + c >= k;
    if (own_c && here) atomicMin(&sh.found, tid);
    __syncthreads();
    int b = sh.found;
    if (b == 0x7fffffff) {               // the target lies past every weight: the last bin
      __syncthreads();
      if (tid == 0) sh.found = 0;
      __syncthreads();
      if (own_c) atomicMax(&sh.found, tid);
      __syncthreads();
      b = sh.found;
    }
    if (tid == b) { sh.n = (int)own_c; sh.fc = c - own_c; sh.fm = m - own_m; }
    __syncthreads();
    n = sh.n;
    above_c += sh.fc;
    above_m += sh.fm;
    float lo = INFINITY, hi = -INFINITY;
    for (int i = r.lo + lane; i < r.hi; i += 64) {
      const float z = load_logit(row, i);
      if (z <= zhi && z >= zlo && bin(z) == b) { lo = fminf(lo, z); hi = fmaxf(hi, z); }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      lo = fminf(lo, __shfl_xor(lo, off));
      hi = fmaxf(hi, __shfl_xor(hi, off));
    }
    if (lane == 0) { sh.f[wv] = lo; sh.g[wv] = hi; }
    __syncthreads();
    for (int i = 0; i < FW; ++i) { lo = fminf(lo, sh.f[i]); hi = fmaxf(hi, sh.g[i]); }
    zlo = lo;
    zhi = hi;
    __syncthreads();
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
    cut.idx = nth_equal(row, V, zhi, keep, sh);
    cut.mass = above_m + w * (unsigned long long)keep;
    return cut;
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  for (int i = r.lo + lane; i < r.hi; i += 64) {
    const float z = load_logit(row, i);
    if (z <= zhi && z >= zlo) {
      const int at = atomicAdd(&sh.n, 1);
      if (at < RANK) { sh.lz[at] = z; sh.li[at] = i; }
    }
  }
  __syncthreads();
  n = min(sh.n, RANK);
  float z = 0.f;
  int idx = 0, rank = 0;
  if (tid < n) {
    z = sh.lz[tid];
    idx = sh.li[tid];
    for (int j = 0; j < n; ++j) {
      const float oz = sh.lz[j];
      rank += oz > z || (oz == z && sh.li[j] < idx);
    }
    sh.lw[rank] = masses ? fixed_weight(z, rc, scale) : 0;
  }
  __syncthreads();
  uint32_t c = tid < n;
  unsigned long long m = tid < n ? sh.lw[tid] : 0;
  scan_bins(c, m, sh);
  if (tid == 0) sh.found = n - 1;
  __syncthreads();
  const bool here = by_mass ? (double)(above_m + m) >= target : above_c + c >= k;
  if (tid < n && here) atomicMin(&sh.found, tid);
  __syncthreads();
  const int at = sh.found;
  if (tid < n && rank == at) { sh.f[0] = z; sh.n = idx; }
  if (tid == at) sh.fm = m;
  __syncthreads();
  cut.z = sh.f[0];
  cut.idx = sh.n;
  cut.mass = above_m + sh.fm;
  __syncthreads();
  return cut;
}

// Reads a row and finds what its filters keep; the kept weights' range sums
// are in sh.d afterwards.
template <typename E>
__device__ RowCut filter_row(const E* row, int V, const RowParams& par, int pi, int32_t* err,
                             FilterShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const Range r = wave_range(V, wv);
  float hi = -INFINITY, lo = INFINITY;
  uint32_t n = 0;
  bool bad = false;
  for (int i = r.lo + lane; i < r.hi; i += 64) {
    const float z = load_logit(row, i);
    bad |= !(z < INFINITY);
    hi = fmaxf(hi, z);
    if (z > -INFINITY) { lo = fminf(lo, z); ++n; }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    hi = fmaxf(hi, __shfl_xor(hi, off));
    lo = fminf(lo, __shfl_xor(lo, off));
    n += __shfl_xor(n, off);
  }
  if (lane == 0) { sh.f[wv] = hi; sh.g[wv] = lo; sh.c[wv] = n; }
  if (bad) set_err(err, DVS_ERR_NONFINITE);
  __syncthreads();
  n = 0;
  for (int i = 0; i < FW; ++i) { hi = fmaxf(hi, sh.f[i]); lo = fminf(lo, sh.g[i]); n += sh.c[i]; }
  __syncthreads();

  const float T = par.temperature ? par.temperature[pi] : 1.0f;
  int k = par.top_k ? par.top_k[pi] : 0;
  const double p = par.top_p ? (double)par.top_p[pi] : 1.0;
  RowCut rc;
  rc.zmax = hi;
  rc.z = -INFINITY;
  rc.idx = 0x7fffffff;
  rc.min_w = par.min_p ? par.min_p[pi] : 0.0f;
  if (!(rc.min_w > 0.0f)) rc.min_w = 0.0f;
  rc.inv_t = 1.0 / (double)T;
  if (n == 0 && tid == 0) set_err(err, DVS_ERR_NONFINITE);
  if (!(T > 0.0f) || k == 1 || rc.min_w > 1.0f || n == 0 || hi == INFINITY) {
    rc.z = hi;                           // top-1: the lowest index of the maximum
    rc.idx = nth_equal(row, V, hi, 1, sh);
    rc.min_w = 0.0f;
    rc.inv_t = 0.0;
  } else {
    const bool need_k = k > 0 && (uint32_t)k < n, need_p = p < 1.0;
    const double scale = ldexp(1.0, __clz(V) + 30);   // V * scale <= 2^62
    double whole = 0.0;
    if (need_k) {
      const Cut c = select_cut(row, V, rc, scale, (int)n, hi, lo, false, need_p, (uint32_t)k, 0.0,
                               sh);
      rc.z = c.z;
      rc.idx = c.idx;
      whole = (double)c.mass;
    }
    if (need_p) {
      if (!need_k)
        whole = range_sums([&](int i) { return weight(load_logit(row, i), rc); }, V, sh) * scale;
      const Cut c = select_cut(row, V, rc, scale, (int)n, hi, lo, true, true, 0,
                               fmax(p, 0.0) * whole, sh);
      if (c.z > rc.z || (c.z == rc.z && c.idx < rc.idx)) { rc.z = c.z; rc.idx = c.idx; }
    }
  }
  rc.total = range_sums([&](int i) { return kept_weight(load_logit(row, i), i, rc); }, V, sh);
  return rc;
}

// ---------------------------------------------------------------------------
// kernels
// ---------------------------------------------------------------------------

template <typename E>
__global__ void __launch_bounds__(FT) sample_filtered_kernel(
    const E* __restrict__ logits, long long ld, int V, RowParams par, int rows_per_param,
    const float* __restrict__ u, int u_stride, int32_t* __restrict__ token_out,
    float* __restrict__ prob_out, int32_t* err) {
  __shared__ FilterShared sh;
  const int row = blockIdx.x, s = row / rows_per_param;
  const E* z = logits + (size_t)row * ld;
  const RowCut rc = filter_row(z, V, par, s, err, sh);
  float uu = u[(size_t)s * u_stride + (row - s * rows_per_param)];
  if (!(uu > 0.0f)) uu = 0.0f;
  const int t = pick_index([&](int i) { return kept_weight(load_logit(z, i), i, rc); }, V,
                           (double)uu * rc.total, sh);
  if (threadIdx.x == 0) {
    token_out[row] = max(t, 0);          // a row of NaN alone: 0
    if (prob_out)
      prob_out[row] = rc.zmax == -INFINITY ? 0.0f
                                           : (float)(kept_weight(load_logit(z, t), t, rc) / rc.total);
  }
}

// Cuts of the verify rows (first S * (B + 1)) and draft rows (S * B) of a call.
template <typename E>
__global__ void __launch_bounds__(FT) filter_rows_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int B, int nv, int V, RowParams par, RowCut* __restrict__ cuts, int32_t* err) {
  __shared__ FilterShared sh;
  const int row = blockIdx.x;
  const int per = row < nv ? B + 1 : B, i = row < nv ? row : row - nv;
  const int s = i / per, j = i - s * per;
  const E* z = row < nv ? zv + (size_t)s * vs + (size_t)j * vld : zd + (size_t)s * ds + (size_t)j * dld;
  const RowCut rc = filter_row(z, V, par, s, err, sh);
  if (threadIdx.x == 0) cuts[row] = rc;
}

__device__ __forceinline__ double prob_of(float z, int i, const RowCut& c) {
  return c.total > 0.0 ? kept_weight(z, i, c) / c.total : 0.0;
}

// One workgroup per sequence: d_j accepted while u q_j(d_j) < p_j(d_j), then
// the final token from max(0, p - q) of the rejected draft's rows, or from the
// last verify row.
template <typename E>
__global__ void __launch_bounds__(FT) accept_filtered_kernel(
    const E* __restrict__ zv, long long vs, long long vld, const E* __restrict__ zd, long long ds,
    long long dld, int S, int B, int V, const RowCut* __restrict__ cuts,
    const int32_t* __restrict__ draft, int draft_width, const float* __restrict__ u, int u_stride,
    int32_t* __restrict__ accept_len, int32_t* __restrict__ token_out, int token_stride,
    int at_accepted) {
  __shared__ FilterShared sh;
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
      const double p = prob_of(load_logit(v + (size_t)j * vld, t), t, cv[j]);
      const double q = prob_of(load_logit(d + (size_t)j * dld, t), t, cd[j]);
      ok = (double)u[(size_t)s * u_stride + j] * q < p;
    }
    if (!ok) atomicMin(&sh.found, j);
  }
  __syncthreads();
  const int A = sh.found;
  float uu = u[(size_t)s * u_stride + B];
  if (!(uu > 0.0f)) uu = 0.0f;
  const RowCut p = cv[A];
  const E* zp = v + (size_t)A * vld;
  auto alone = [&](int i) { return prob_of(load_logit(zp, i), i, p); };
  int t = -1;
  if (A < B) {
    const RowCut q = cd[A];
    const E* zq = d + (size_t)A * dld;
    auto rest = [&](int i) {
      const double a = alone(i);
      return a > 0.0 ? fmax(a - prob_of(load_logit(zq, i), i, q), 0.0) : 0.0;
    };
    const double total = range_sums(rest, V, sh);
    t = pick_index(rest, V, (double)uu * total, sh);
  }
  if (t < 0) {                           // all accepted, or p and q equal to the last bit
    const double total = range_sums(alone, V, sh);
    t = pick_index(alone, V, (double)uu * total, sh);
  }
  if (tid == 0) {
    accept_len[s] = A;
    token_out[(size_t)s * token_stride + (at_accepted ? A : 0)] = max(t, 0);
  }
}

size_t filter_cuts_bytes(int S, int B) { return (size_t)S * (2 * B + 1) * sizeof(RowCut); }

template <typename E>
static int launch_accept(const void* zv, long long vs, long long vld, const void* zd, long long ds,
                         long long dld, int S, int B, int V, const RowParams& par,
                         const int32_t* draft, int draft_width, const float* u, int u_stride,
                         int32_t* accept_len, int32_t* token_out, int token_stride,
                         int at_accepted, int32_t* err, void* ws, hipStream_t st) {
  RowCut* cuts = (RowCut*)ws;
  hipLaunchKernelGGL(filter_rows_kernel<E>, dim3(S * (2 * B + 1)), dim3(FT), 0, st, (const E*)zv,
                     vs, vld, (const E*)zd, ds, dld, B, S * (B + 1), V, par, cuts, err);
  const int rc = launch_status("accept_sampled (filters)");
  if (rc) return rc;
  hipLaunchKernelGGL(accept_filtered_kernel<E>, dim3(S), dim3(FT), 0, st, (const E*)zv, vs, vld,
                     (const E*)zd, ds, dld, S, B, V, cuts, draft, draft_width, u, u_stride,
                     accept_len, token_out, token_stride, at_accepted);
  return launch_status("accept_sampled (accept)");
}

int launch_sample_filtered(const void* logits, int dtype, int rows, int V, long long ld,
                           const RowParams& par, int rows_per_param, const float* u, int u_stride,
                           int32_t* token_out, float* prob_out, int32_t* err, hipStream_t st) {
  if (dtype == DVS_BF16)
    hipLaunchKernelGGL(sample_filtered_kernel<uint16_t>, dim3(rows), dim3(FT), 0, st,
                       (const uint16_t*)logits, ld, V, par, rows_per_param, u, u_stride, token_out,
                       prob_out, err);
  else
    hipLaunchKernelGGL(sample_filtered_kernel<float>, dim3(rows), dim3(FT), 0, st,
                       (const float*)logits, ld, V, par, rows_per_param, u, u_stride, token_out,
                       prob_out, err);
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
