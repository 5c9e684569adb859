// attn_tree: attention of a window of drafted rows, whose keys and values are
// in the paged cache already, over the cache and each row's ancestors.
#include <math.h>

#include <algorithm>

#include "dvs_common.h"

namespace dvs {

static size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }

__device__ __forceinline__ void store4(float* p, f32x4 v) { *(f32x4*)p = v; }
__device__ __forceinline__ void store4(__bf16* p, f32x4 v) {
  *(bf16x4*)p = __builtin_convertvector(v, bf16x4);
}

constexpr int MAX_SEQS = 1024;      // sequences a launch takes
constexpr int FW = 4, NW = 8;       // waves of a workgroup: few query rows, many
constexpr float WEIGHT_MAX = 2048.f, RESCALE_LOG2 = 11.5f;   // (2^11.5 is above the first)
constexpr int MERGE_FEW = 1024; // row groups up to which the merge takes more waves

struct TreeAttn {
  const void *q, *k_pool, *v_pool;
  const int32_t *table, *kv_len, *mask;
  void* out;
  int32_t* err;
  int S, R, W, Hq, Hkv, G, rows, n_rt, max_pages, pool_pages;
  int n_wide;      // workgroups of NW waves over an item's rows (0: tiles not through LDS)
  int split;       // items are cut where a share ends, and merged by a launch of its own
  float scale_log2;
  float* part_o;   // [slot][quad][lane] x 4
  float* part_ml;  // [slot][group][lane] x (m, l)
  int2* meta;      // [item] segments, share of the first
};

// ---------------------------------------------------------------------------
// Matrix instructions of 16 x 16: a lane is (m, quarter) or (n, quarter), with
// m, n = lane & 15.  S^T[key, row] = K Q^T puts a query row in a lane's column
// n, its keys in the four quarters; the exponentials are then the second
// operand of O^T[d, row] += V^T P^T as they lie: the quarter's keys of P in a
// lane are those of its piece of V.
//
// bf16: 32 keys a tile.  16x16x32 wants 8 consecutive keys a quarter of P, and
// a result holds 4 rows a quarter: the first of two products takes the keys
// 8 (m / 4) + m % 4, the second those 4 further on, so that their results side
// by side are the keys 8 quarter .. + 7.
// fp32: 16 keys a tile, 16x16x4: product i of four takes element i of every
// lane's 16 bytes, in QK (4 elements of d a quarter) and PV (4 keys a quarter).
//
// Either way K and V are D / 16 pieces of 16 bytes a lane a tile, straight
// from the cache page.
// ---------------------------------------------------------------------------
template <typename T>
struct Tile;

template <>
struct Tile<__bf16> {
  static constexpr int KEYS = 32, PAGES = 2, NK = 8, NS = 2;   // keys a lane, results
  template <int D>
  static __device__ __forceinline__ int k_page(int m, int) { return m >> 3; }
  // offset in a page of a lane's piece 0 of K, and from there to piece i: the
  // first and the second product's keys by turns
  template <int D>
  static __device__ __forceinline__ uint32_t k_off(int m, int quarter) {
    return (uint32_t)(((8 * ((m >> 2) & 1) + (m & 3)) * D + quarter * 8) * 2);
  }
  template <int D>
  static constexpr int k_piece(int i) { return ((i & 1) * 4 * D + (i >> 1) * 32) * 2; }
  static __device__ __forceinline__ int v_page(int quarter) { return quarter >> 1; }
  static __device__ __forceinline__ uint32_t v_off(int m, int quarter) {
    return (uint32_t)((m * 16 + (quarter & 1) * 8) * 2);
  }
  // element of the head at which a lane's piece i of a query row starts
  static constexpr int NQ_DIV = 32;
  static __device__ __forceinline__ int q_elem(int quarter, int i) { return i * 32 + quarter * 8; }
};

template <>
struct Tile<float> {
  static constexpr int KEYS = 16, PAGES = 1, NK = 4, NS = 1;
  template <int D>
  static __device__ __forceinline__ int k_page(int, int) { return 0; }
  template <int D>
  static __device__ __forceinline__ uint32_t k_off(int m, int quarter) {
    return (uint32_t)((m * D + quarter * 4) * 4);
  }
  template <int D>
  static constexpr int k_piece(int i) { return i * 64; }
  static __device__ __forceinline__ int v_page(int) { return 0; }
  static __device__ __forceinline__ uint32_t v_off(int m, int quarter) {
    return (uint32_t)((m * 16 + quarter * 4) * 4);
  }
  static constexpr int NQ_DIV = 16;
  static __device__ __forceinline__ int q_elem(int quarter, int i) { return i * 16 + quarter * 4; }
};

__device__ __forceinline__ float rows_max(float v) {   // over the four quarters
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const f32x2 b = halves_pair(v);
  return fmaxf(b[0], b[1]);
}
__device__ __forceinline__ float rows_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const f32x2 b = halves_pair(v);
  return b[0] + b[1];
}

// Bits i < N: whether window row r sees key key0 + i.  any: the row's mask has
// a bit (it sees the cache).
template <int N>
__device__ __forceinline__ uint32_t seen_bits(const TreeAttn& p, const uint32_t* mask, int r, bool any,
                                              int key0, int L) {
  constexpr uint32_t ALL = (1u << N) - 1;
  if (!any) return 0;
  const int o = key0 - L;   // window slot of the first key
  if (!mask) {
    const int n = r - o + 1;
    return n <= 0 ? 0 : (n >= N ? ALL : (1u << n) - 1);
  }
  if (o + N <= 0) return ALL;
  const int lo = max(o, 0), w = lo >> 5, sh = lo & 31;
  uint64_t bits = 0;
  if (w < p.W) bits = mask[w];
  if (w + 1 < p.W) bits |= (uint64_t)mask[w + 1] << 32;
  uint32_t b = (uint32_t)(bits >> sh);
  if (p.R - lo < 32) b &= p.R > lo ? (1u << (p.R - lo)) - 1 : 0;   // no slot past the window
  if (o < 0) b = b << -o | ((1u << -o) - 1);
  return b & ALL;
}

// One tile's softmax: scores to weights 2^(s - m).  m is a reference, not the
// maximum so far: any m will do that keeps the weights in range, and the
// division by l is exact about it.  So a tile takes m as it is, and only where
// a lane's weights add up to more than WEIGHT_MAX (or to no number: m starts at
// -inf) the rows' maxima are found, m moves to those that exceed it by RESCALE_LOG2,
// and the tile's weights are made again (long documents 540 us with the maxima
// of every tile, 458 without).  A row that moves would have called for it by
// itself: what it gives does not depend on the rows beside it.
template <typename T>
struct Weights;
template <>
struct Weights<__bf16> {   // a lane's 8 keys, rounded once: what the matrix instruction takes
  typedef bf16x8 type;
  // l is summed before the rounding
  static __device__ __forceinline__ float make(const f32x4* s, float scale_log2, float ref, bf16x8& w) {
    f32x4 e[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) e[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], scale_log2, -ref));
    u32x4 pk;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      pk[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                               f32x2{e[i >> 1][2 * (i & 1)], e[i >> 1][2 * (i & 1) + 1]}, bf16x2));
    w = __builtin_bit_cast(bf16x8, pk);
    return ((e[0][0] + e[0][1]) + (e[0][2] + e[0][3])) + ((e[1][0] + e[1][1]) + (e[1][2] + e[1][3]));
  }
};
template <>
struct Weights<float> {    // 4 keys
  typedef f32x4 type;
  static __device__ __forceinline__ float make(const f32x4* s, float scale_log2, float ref, f32x4& w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(fmaf(s[0][i], scale_log2, -ref));
    return (w[0] + w[1]) + (w[2] + w[3]);
  }
};

template <typename T, int NS, int NG, int DG>
__device__ __forceinline__ void softmax_tile(const f32x4 (&s)[NG][NS], typename Weights<T>::type (&w)[NG],
                                             float scale_log2, float (&m)[NG], float (&l)[NG],
                                             f32x4 (&o)[NG][DG]) {
  float sum[NG];
  bool over = false;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    sum[g] = Weights<T>::make(s[g], scale_log2, m[g], w[g]);
    over |= !(sum[g] <= WEIGHT_MAX);
  }
  if (__ballot(over)) {
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float t = fmaxf(fmaxf(s[g][0][0], s[g][0][1]), fmaxf(s[g][0][2], s[g][0][3]));
      if constexpr (NS == 2)
        t = fmaxf(t, fmaxf(fmaxf(s[g][1][0], s[g][1][1]), fmaxf(s[g][1][2], s[g][1][3])));
      const float cand = rows_max(t) * scale_log2;
      if (cand > m[g] + RESCALE_LOG2) {
        const float a = __builtin_amdgcn_exp2f(m[g] - cand);
        m[g] = cand;
        l[g] *= a;
#pragma unroll
        for (int d = 0; d < DG; ++d) o[g][d] *= a;
      }
      sum[g] = Weights<T>::make(s[g], scale_log2, m[g] == -INFINITY ? 0.f : m[g], w[g]);
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) l[g] += sum[g];
}

// The sequences' tiles side by side: how many lie before each of them, which
// sequence a tile belongs to, and the lengths.  Sequences that do not fit their
// table have none.  Up to 64: in registers, a lane a sequence, every wave for
// itself; more: in LDS, by the whole workgroup.
struct SeqTiles {
  int S, total;
  int upto, len;             // of sequence `lane`
  const int *s_seq, *s_len;
  bool in_lds;

  __device__ __forceinline__ int before(int s) const {
    if (in_lds) return s_seq[s];
    return s == 0 ? 0 : __builtin_amdgcn_readlane(upto, s - 1);
  }
  __device__ __forceinline__ int length(int s) const {
    return in_lds ? s_len[s] : __builtin_amdgcn_readlane(len, s);
  }
  __device__ __forceinline__ int find(int t) const {   // t < total
    if (!in_lds) return __popcll(__ballot((threadIdx.x & 63) < S && upto <= t));
    int lo = 0, hi = S;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_seq[mid] <= t) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

__device__ __forceinline__ int scan64(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(v, off);
    if (lane >= off) v += o;
  }
  return v;
}

// By a workgroup of WAVES waves (s_tot: a word each).
template <int WAVES>
__device__ __forceinline__ SeqTiles seq_tiles(const TreeAttn& p, int keys, int (&s_seq)[MAX_SEQS + 1],
                                              int (&s_len)[MAX_SEQS], int (&s_tot)[WAVES]) {
  const int tid = threadIdx.x, lane = tid & 63;
  auto tiles_of = [&](int s, int L) {
    if (s >= p.S) return 0;
    if (L < 0 || (long long)L + p.R > (long long)p.max_pages * DVS_PAGE_SIZE) {
      if (blockIdx.x == 0) set_err(p.err, DVS_ERR_MAX_PAGES);
      return 0;
    }
    return (L + p.R + keys - 1) / keys;
  };
  if (p.S <= 64) {
    const int L = p.kv_len[min(lane, p.S - 1)], upto = scan64(tiles_of(lane, L));
    return SeqTiles{p.S, __builtin_amdgcn_readlane(upto, 63), upto, L, nullptr, nullptr, false};
  }
  int carry = 0;
  for (int s0 = 0; s0 < p.S; s0 += WAVES * 64) {
    const int s = s0 + tid, L = s < p.S ? p.kv_len[s] : 0;
    if (s < p.S) s_len[s] = L;
    const int t = scan64(tiles_of(s, L));
    if (s0) __syncthreads();
    if (lane == 63) s_tot[tid >> 6] = t;
    __syncthreads();
    int before = carry;
#pragma nounroll
    for (int w = 0; w < WAVES; ++w) {
      const int v = s_tot[w];
      if (w < (tid >> 6)) before += v;
      carry += v;
    }
    if (s < p.S) s_seq[1 + s] = before + t;
  }
  if (tid == 0) s_seq[0] = 0;
  __syncthreads();
  return SeqTiles{p.S, s_seq[p.S], 0, 0, s_seq, s_len, true};
}

// Consecutive workgroups on one XCD (blockIdx goes round the eight): row tiles
// of an item then find its keys in their L2.
__device__ __forceinline__ int xcd_block(int n) {   // of n workgroups
  const int q = n >> 3, rem = n & 7, x = blockIdx.x & 7, i = blockIdx.x >> 3;
  return x * q + min(x, rem) + i;
}

// This workgroup's share of the key tiles, in order of sequences, then items of a
// sequence (per_seq of them): [u, u_end) of share `id`, whose row tile is rt of
// `wide`.  Split: equal shares, which cut items; else whole items.
// A share has some tiles at least, by the sequences' mean length: the merge grows
// with the parts of an item (us, one sequence, one row: 16000 keys in shares of 8 /
// 16 / 32 tiles 27.4 / 21.4 / 23.5, 8000 of 8 / 10 18.6 / 18.0; 8 of 100-400, 128 rows, 4
// / 8 21.7 / 24.7).  Workgroups that this leaves without any are the last, so that
// the others lie on all XCDs (one of 16000: 28 on three of them, 21.7 on all; 8
// of 500 in tables of 32768, 16 rows, 20.4 / 10.7).
struct Share {
  int id, rt, u, u_end, size;
};
__device__ __forceinline__ Share share_of(const TreeAttn& p, const SeqTiles& seqs, int per_seq, int wide) {
  const int U = seqs.total * per_seq;
  int n = gridDim.x / wide, size = 1;
  if (p.split) {
    const int mean = seqs.total / p.S;
    const int least = p.n_wide ? (mean <= 32 ? 4 : max(8, mean / 64)) : max(4, mean / 24);
    size = max((U + n - 1) / n, least);
    n = (U + size - 1) / size;
  }
  if ((int)blockIdx.x >= n * wide) return Share{0, 0, 0, 0, size};
  const int block = xcd_block(n * wide), id = block / wide, rt = block - id * wide;
  if (p.split) return Share{id, rt, id * size, (int)min((long long)(id + 1) * size, (long long)U), size};
  auto start = [&](uint32_t i) {
    const int s = i / per_seq;
    if (s >= p.S) return U;
    return seqs.before(s) * per_seq + (int)(i - s * per_seq) * (seqs.before(s + 1) - seqs.before(s));
  };
  const uint32_t items = p.S * per_seq;   // at most 2^22, n at most 2 a CU
  return Share{id, rt, start(id * items / n), start((id + 1) * items / n), size};
}

// A lane's NG query rows: row n of a KV head is window row n / G, head n % G of
// its group.  Every load is sent out before any is waited for.  any: the row's
// mask (NULL: causal) has a bit of the window.
template <typename T, int D, int NG>
struct Rows {
  static constexpr int NQ = D / Tile<T>::NQ_DIV;
  int first, kvh, r[NG];
  bool any[NG];
  u32x4 q[NG][NQ];

  __device__ __forceinline__ bool valid(const TreeAttn& p, int g) const {
    return first + g * 16 + (int)(threadIdx.x & 15) < p.rows;
  }
  // the row in q and out (one that is not there: the first)
  __device__ __forceinline__ size_t at(const TreeAttn& p, int s, int g) const {
    const int h = valid(p, g) ? first + g * 16 + (int)(threadIdx.x & 15) - r[g] * p.G : 0;
    return (((size_t)s * p.R + r[g]) * p.Hq + kvh * p.G + h) * D;
  }
  __device__ __forceinline__ const uint32_t* mask(const TreeAttn& p, int s, int g) const {
    return p.mask ? (const uint32_t*)p.mask + ((size_t)s * p.R + r[g]) * p.W : nullptr;
  }

  __device__ __forceinline__ void load(const TreeAttn& p, int s, int kv_head, int first_row) {
    const int lane = threadIdx.x & 63, m16 = lane & 15, quarter = lane >> 4;
    first = first_row;
    kvh = kv_head;
    uint32_t bits[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      r[g] = valid(p, g) ? (first + g * 16 + m16) / p.G : 0;
      const T* src = (const T*)p.q + at(p, s, g);
#pragma unroll
      for (int i = 0; i < NQ; ++i) q[g][i] = *(const u32x4*)(src + Tile<T>::q_elem(quarter, i));
      bits[g] = 1;
    }
    if (p.mask) {
#pragma unroll
      for (int g = 0; g < NG; ++g) bits[g] = mask(p, s, g)[p.W - 1] & (0xffffffffu >> (31 - ((p.R - 1) & 31)));
      for (int i = 0; i < p.W - 1; ++i)
#pragma unroll
        for (int g = 0; g < NG; ++g) bits[g] |= mask(p, s, g)[i];
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      any[g] = valid(p, g) && bits[g] != 0;
      // (padding: NaN there would take every tile's slower way)
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        if (!any[g]) q[g][i] = u32x4{0, 0, 0, 0};
    }
  }
};

// A page id of the table, 0 (and the error) for one outside the pool.
__device__ __forceinline__ int checked_page(const TreeAttn& p, int id) {
  if (id >= 0 && id < p.pool_pages) return id;
  set_err(p.err, DVS_ERR_BAD_PAGE);
  return 0;
}

// A value that a row does not see must not reach it, and 0 times an infinity or a
// NaN would.  In the window's tiles such values are therefore taken out of the
// product, and added to the rows that see them (slots behind the last row hold
// anything, others seldom such: finding out is a product with zeros, or in fp32
// a multiplication each).  bits: of a lane's row and its quarter's keys;
// values(key): the key's, 16 elements from one of the head to the next.
template <typename T, int NG, int DG, class F>
__device__ __forceinline__ void clean_values(u32x4 (&vf)[DG], const uint32_t (&bits)[NG], f32x4 (&o)[NG][DG],
                                             F values) {
  const int quarter = (threadIdx.x & 63) >> 4;
  bool found = false;
  if constexpr (sizeof(T) == 2) {
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DG; ++d)
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]), bf16x8{}, z, 0, 0, 0);
    found = z[0] != 0.f || z[1] != 0.f || z[2] != 0.f || z[3] != 0.f;
  } else {
    float z = 0.f;
#pragma unroll
    for (int d = 0; d < DG; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) z = fmaf(__uint_as_float(vf[d][e]), 0.f, z);
    found = z != 0.f;
  }
  if (!__ballot(found)) return;
#pragma unroll
  for (int d = 0; d < DG; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((vf[d][e] & 0x7f800000) == 0x7f800000) vf[d][e] &= sizeof(T) == 2 ? 0xffff : 0;
      if (sizeof(T) == 2 && (vf[d][e] & 0x7f80) == 0x7f80) vf[d][e] &= 0xffff0000;
    }
  constexpr int NK = Tile<T>::NK;
  uint32_t sees[NG], some = 0;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    uint32_t b = bits[g] << quarter * NK;
    b |= __shfl_xor((int)b, 16);
    sees[g] = b | __shfl_xor((int)b, 32);
    some |= sees[g];
  }
#pragma nounroll
  for (int key = 0; key < Tile<T>::KEYS; ++key) {
    if (!__ballot(some >> key & 1)) continue;
    const char* v = (const char*)values(key);
    const uint32_t off = quarter * 64 * (uint32_t)sizeof(T);
#pragma unroll
    for (int d = 0; d < DG; ++d) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = (float)*(const T*)(v + off + (d * 16 + i) * 16 * (int)sizeof(T));
        const bool odd = (__float_as_uint(x) & 0x7f800000) == 0x7f800000;
#pragma unroll
        for (int g = 0; g < NG; ++g) o[g][d][i] += odd && (sees[g] >> key & 1) ? x : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);   // (few registers are free here)
    }
  }
}

// End of a segment: the output, or a part of it (O, m and l in 32 bits).  l is
// 0 exactly for a row that sees nothing (or no score above -inf), whatever its O
// holds.
template <typename T, int D, int NG>
__device__ __forceinline__ void finish_rows(const TreeAttn& p, int s, const Rows<T, D, NG>& row,
                                            const float (&m)[NG], float (&l)[NG],
                                            const f32x4 (&o)[NG][D / 16], int nseg, size_t slot) {
  const int lane = threadIdx.x & 63, m16 = lane & 15, quarter = lane >> 4;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    l[g] = rows_sum(l[g]);
    if (!row.any[g]) l[g] = 0.f;
    if (nseg > 1) {
      if (quarter == 0) *(f32x2*)(p.part_ml + ((slot * NG + g) * 16 + m16) * 2) = f32x2{m[g], l[g]};
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        *(f32x4*)(p.part_o + ((slot * NG + g) * (D / 16) + d) * 256 + lane * 4) = o[g][d];
    } else if (row.valid(p, g)) {
      T* dst = (T*)p.out + row.at(p, s, g) + quarter * 4;
      const float inv = 1.f / l[g];
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        f32x4 x = o[g][d] * inv;
        if (l[g] == 0.f) x = f32x4{0.f, 0.f, 0.f, 0.f};
        store4(dst + d * 16, x);
      }
    }
  }
}

// The same where the workgroup's waves hold parts of one segment: joined in LDS,
// a wave every fourth 16 elements of the head.
template <typename T, int D, int NG>
__device__ __forceinline__ void finish_together(const TreeAttn& p, int s, const Rows<T, D, NG>& row,
                                                const float (&m)[NG], float (&l)[NG],
                                                const f32x4 (&o)[NG][D / 16], int nseg, size_t slot,
                                                f32x4* s_o, f32x2* s_ml) {
  constexpr int DG = D / 16;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m16 = lane & 15, quarter = lane >> 4;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    l[g] = rows_sum(l[g]);
    s_ml[(w * NG + g) * 64 + lane] = f32x2{m[g], row.any[g] ? l[g] : 0.f};
#pragma unroll
    for (int d = 0; d < DG; ++d) s_o[((w * NG + g) * DG + d) * 64 + lane] = o[g][d];
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    f32x2 ml[FW];
    float M = -INFINITY, sum = 0.f, e[FW];
#pragma unroll
    for (int i = 0; i < FW; ++i) {
      ml[i] = s_ml[(i * NG + g) * 64 + lane];
      if (ml[i][1] != 0.f) M = fmaxf(M, ml[i][0]);
    }
#pragma unroll
    for (int i = 0; i < FW; ++i) {
      e[i] = ml[i][1] != 0.f ? __builtin_amdgcn_exp2f(ml[i][0] - M) : 0.f;
      if (ml[i][1] != 0.f) sum = fmaf(e[i], ml[i][1], sum);
    }
    if (nseg > 1 && w == 0 && quarter == 0)
      *(f32x2*)(p.part_ml + ((slot * NG + g) * 16 + m16) * 2) = f32x2{M, sum};
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* dst = (T*)p.out + row.at(p, s, g) + quarter * 4;
#pragma unroll
    for (int d0 = 0; d0 < DG; d0 += FW) {
      const int d = d0 + w;
      if (d >= DG) break;
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < FW; ++i) {
        const f32x4 y = s_o[((i * NG + g) * DG + d) * 64 + lane];
        if (ml[i][1] != 0.f) {
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = fmaf(e[i], y[j], x[j]);
        }
      }
      if (nseg > 1) *(f32x4*)(p.part_o + ((slot * NG + g) * DG + d) * 256 + lane * 4) = x;
      else if (row.valid(p, g)) store4(dst + d * 16, x * inv);
    }
  }
  __syncthreads();
}

// ---------------------------------------------------------------------------
// Few query rows of a KV head, or few tiles: a workgroup takes NG groups of 16 of them and a run
// of key tiles, a quarter of it a wave, straight from the cache into registers:
// the next tile's keys are on their way under this one's softmax, its values
// under the next one's scores.  The waves' results are joined in LDS (a wave on
// its own, with a part of its own for the merge, took, us: 64 sequences of 1k-8k,
// one row 117 / 111; 32 of 1k-8k, 16 rows 75 / 67; one of 16000, one row 28 / 21).
//
// What bounds it: long caches, the cache (64 sequences, one row, 556 MB: 111 us,
// 5.0 TB/s of the 5.1 - 5.2 that a copy reaches); one sequence, latency: the lengths,
// then the page ids, then keys and values, 1 - 2 us each, then the second launch
// (2000 keys, one row 13.7 us, 128 rows 15.0); fp32, the matrix instructions (32
// sequences of 1k-4k, 64 rows: 149 us, half their rate).
// ---------------------------------------------------------------------------
template <typename T, int D, int NG>
__global__ void __launch_bounds__(FW * 64, 2) tree_attn_wave_kernel(TreeAttn p) {
  using TL = Tile<T>;
  constexpr int KEYS = TL::KEYS, NP = D / 16, DG = D / 16, NS = TL::NS;
  constexpr int PAGE_B = 16 * D * (int)sizeof(T);
  __shared__ int s_seq[MAX_SEQS + 1], s_len[MAX_SEQS], s_tot[FW];
  __shared__ f32x4 s_o[FW * NG * DG * 64];
  __shared__ f32x2 s_ml[FW * NG * 64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m16 = lane & 15, quarter = lane >> 4;
  const int HN = p.Hkv * p.n_rt;
  const SeqTiles seqs = seq_tiles<FW>(p, KEYS, s_seq, s_len, s_tot);
  const Share sh = share_of(p, seqs, HN, 1);
  const int share_id = __builtin_amdgcn_readfirstlane(sh.id);
  const int u_end = __builtin_amdgcn_readfirstlane(sh.u_end), share = __builtin_amdgcn_readfirstlane(sh.size);
  int u = __builtin_amdgcn_readfirstlane(sh.u);
  const char* kp = (const char*)p.k_pool;
  const char* vp = (const char*)p.v_pool;
  const uint32_t koff = TL::template k_off<D>(m16, quarter), voff = TL::v_off(m16, quarter);
  const int kpage = TL::template k_page<D>(m16, quarter), vpage = TL::v_page(quarter);

  while (u < u_end) {
    const int s = __builtin_amdgcn_readfirstlane(seqs.find(u / HN));
    const int L = __builtin_amdgcn_readfirstlane(seqs.length(s));
    const int U0 = __builtin_amdgcn_readfirstlane(seqs.before(s)) * HN;
    const int tiles = __builtin_amdgcn_readfirstlane(seqs.before(s + 1)) - U0 / HN;
    const int qi = (u - U0) / tiles, first = u - U0 - qi * tiles, n = min(tiles - first, u_end - u);
    const int P0 = U0 + qi * tiles;
    const int k = p.split ? share_id - P0 / share : 0;
    const int nseg = p.split ? (P0 + tiles - 1) / share - P0 / share + 1 : 1;
    u += n;
    const int j0 = first + n * w / FW, j1 = first + n * (w + 1) / FW;   // this wave's
    const int it = s * HN + qi, kvh = qi / p.n_rt, rt = qi - kvh * p.n_rt;
    if (p.split && k == 0 && threadIdx.x == 0) p.meta[it] = int2{nseg, share_id};
    const int n_valid = (L + p.R + 15) >> 4;
    const int32_t* pt = p.table + (size_t)s * p.max_pages;
    // the ids of the next 64 pages, a lane each (checked only when the queries'
    // loads have gone out too)
    auto page_ids = [&](int j) { return pt[min(j * TL::PAGES + lane, n_valid - 1)]; };
    int ids = page_ids(j0), ids_at = j0;
    Rows<T, D, NG> row;
    row.load(p, s, kvh, rt * NG * 16);
    f32x4 o[NG][DG];
    float m[NG], l[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int d = 0; d < DG; ++d) o[g][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    u32x4 kf[NP], vf[NP];
    auto base_of = [&](const char* pool, int j, int page) {
      const int at = (j - ids_at) * TL::PAGES;
      int id = __builtin_amdgcn_readlane(ids, at);
      if constexpr (TL::PAGES == 2) {
        const int id1 = __builtin_amdgcn_readlane(ids, at + 1);
        id = page ? id1 : id;
      }
      return pool + ((size_t)(uint32_t)id * p.Hkv + kvh) * PAGE_B;
    };
    auto load_k = [&](int j) {
      const char* b = base_of(kp, j, kpage) + koff;
#pragma unroll
      for (int i = 0; i < NP; ++i) kf[i] = *(const u32x4*)(b + TL::template k_piece<D>(i));
    };
    auto load_v = [&](int j) {
      const char* b = base_of(vp, j, vpage) + voff;
#pragma unroll
      for (int i = 0; i < NP; ++i) vf[i] = *(const u32x4*)(b + i * 256 * sizeof(T));
    };
    ids = checked_page(p, ids);
    if (j0 < j1) {
      load_k(j0);
      load_v(j0);
    }
    for (int j = j0; j < j1; ++j) {
      f32x4 sc[NG][NS];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
#pragma unroll
        for (int t = 0; t < NS; ++t) sc[g][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int g = 0; g < NG; ++g)
            sc[g][i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, kf[i]), __builtin_bit_cast(bf16x8, row.q[g][i >> 1]), sc[g][i & 1], 0, 0, 0);
        } else {
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[g][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][e]), __uint_as_float(row.q[g][i][e]),
                                                              sc[g][0], 0, 0, 0);
        }
      }
      const bool more = j + 1 < j1;
      // the ids run out: those of the tiles from j on (this tile's are still
      // needed for nothing, the next one's are)
      if (more && (j + 2 - ids_at) * TL::PAGES > 64) {
        ids_at = j + 1;
        ids = checked_page(p, page_ids(ids_at));
      }
      if (more) load_k(j + 1);
      const int key0 = j * KEYS + quarter * TL::NK;
      const bool masked = (j + 1) * KEYS > L;
      uint32_t bits[NG];
      if (masked) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t b = bits[g] = seen_bits<TL::NK>(p, row.mask(p, s, g), row.r[g], row.any[g], key0, L);
#pragma unroll
          for (int i = 0; i < TL::NK; ++i)
            if (!(b >> i & 1)) sc[g][i >> 2][i & 3] = -INFINITY;
        }
      }
      typename Weights<T>::type pf[NG];
      softmax_tile<T, NS, NG, DG>(sc, pf, p.scale_log2, m, l, o);
      if (masked)
        clean_values<T>(vf, bits, o, [&](int key) {
          const int page = __builtin_amdgcn_readfirstlane(checked_page(p, pt[min(j * TL::PAGES + (key >> 4), n_valid - 1)]));
          return (const T*)(vp + ((size_t)(uint32_t)page * p.Hkv + kvh) * PAGE_B) + (key & 15);
        });
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int d = 0; d < DG; ++d)
            o[g][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]), pf[g], o[g][d], 0, 0, 0);
        } else {
#pragma unroll
          for (int d = 0; d < DG; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[g][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[d][e]), pf[g][e], o[g][d], 0, 0, 0);
        }
      }
      if (more) load_v(j + 1);
    }
    const size_t slot = (size_t)share_id * 2 + (k == 0 ? 1 : 0);
    finish_together<T, D, NG>(p, s, row, m, l, o, nseg, slot, s_o, s_ml);
  }
}

// ---------------------------------------------------------------------------
// Many query rows of a KV head (bf16): a workgroup of eight waves, 16 or 32 rows
// each, over 32-key tiles that all of them read from LDS, copied there straight
// from the cache, STAGES tiles at a time.  The next tile's scores are made under
// this tile's softmax (matrix and vector unit), then this tile's values are added.
//
// What bounds it, long documents (256 rows, 1.44 GB, 0.36 PFLOP; 410 - 430 us): no
// unit alone.  A SIMD's matrix core is busy for 42% of the time, its vector ALU
// for 41, both at once for 8, neither for 25, and 36% of a wave's cycles are
// waits; the cache is read once (1.001 of its bytes), without bank conflicts in
// LDS.  The copies alone take 253 us, the arithmetic alone 309; with both the
// clock falls from 2.4 to 1.7 - 2.0 GHz.  Taking the softmax and the products in turns
// by two halves of the waves, 32x32 products, reads ahead of their use and 64 rows
// a wave were all tried: 442 - 530.
//
// LDS rows of K (a key, 2 D bytes) have their 16-byte chunks permuted so that
// the 16 lanes that an access of 16 bytes serves at once (0-3, 12-15, 20-27 of
// 32, or the others) lie in 16 different bank groups; V needs no such order.
// The stages are variables of their own and the loop over them is unrolled:
// the compiler then knows that a read of one does not touch the copies on
// their way into the others, and does not wait for those.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ int k_swizzle(int row) {
  if constexpr (D == 128) return (row & 3) | ((row >> 1) & 12);
  else if constexpr (D == 96) return ((row >> 2) & 2) ^ (((row >> 4) & 1) * 3);
  else return ((row >> 1) & 1) | ((row >> 2) & 6);
}

template <int N>
__device__ __forceinline__ void wait_loads() {   // at most N vector loads on their way
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// Without a wait for this wave's copies; its reads of LDS have ended (what they
// read may be overwritten once every wave is past).
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D, int NG>
__global__ void __launch_bounds__(NW * 64, 2) tree_attn_tile_kernel(TreeAttn p) {
  constexpr int KEYS = 32, DG = D / 16, STAGES = 6;
  constexpr int PAGE_B = 32 * D, TILE_B = 2 * PAGE_B;   // bytes of a page, of a tile's K (or V)
  constexpr int SEGS = PAGE_B / 1024;                   // copies of 1 KB a page
  // copies of a wave a tile, all of one page: half a page, or where that is no
  // whole number (three to a page) two, and the third by the other wave, twice
  constexpr int NPL = (SEGS + 1) / 2;
  constexpr int STAGE_B = 2 * TILE_B;
  __shared__ __attribute__((aligned(1024))) char st0[STAGE_B], st1[STAGE_B], st2[STAGE_B], st3[STAGE_B], st4[STAGE_B],
      st5[STAGE_B];
  __shared__ int s_seq[MAX_SEQS + 1], s_len[MAX_SEQS], s_tot[NW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m16 = lane & 15, quarter = lane >> 4;
  const SeqTiles seqs = seq_tiles<NW>(p, KEYS, s_seq, s_len, s_tot);
  const Share sh = share_of(p, seqs, p.Hkv, p.n_wide);
  const int share_id = __builtin_amdgcn_readfirstlane(sh.id), rt = __builtin_amdgcn_readfirstlane(sh.rt);
  const int u_end = __builtin_amdgcn_readfirstlane(sh.u_end), share = __builtin_amdgcn_readfirstlane(sh.size);
  int u = __builtin_amdgcn_readfirstlane(sh.u);
  // copies: pages 0, 1 of K, then of V; lane's source offset in the page, of
  // its 16 bytes of each 1 KB
  const int cpage = w >> 1;
  auto seg = [&](int i) { return min((w & 1) * NPL + i, SEGS - 1); };
  const char* pool = (const char*)(cpage < 2 ? p.k_pool : p.v_pool);
  uint32_t soff[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    const int off = seg(i) * 1024 + lane * 16;
    if (cpage < 2) {
      const int row = off / (2 * D), c = (off - row * 2 * D) >> 4;
      soff[i] = row * 2 * D + ((c ^ k_swizzle<D>(cpage * 16 + row)) << 4);
    } else {
      soff[i] = off;
    }
  }
  // fragments: K of product t = 0 (t = 1: four rows on), chunk ks * 4 + quarter
  const int krow = 8 * (m16 >> 2) + (m16 & 3), ksw = k_swizzle<D>(krow);
  int kfrag[D / 32];
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) kfrag[ks] = krow * 2 * D + (((ks * 4 + quarter) ^ ksw) << 4);
  const int vfrag = TILE_B + (quarter >> 1) * PAGE_B + m16 * 32 + ((quarter & 1) << 4);
  bool again = false;

  while (u < u_end) {
    const int s = __builtin_amdgcn_readfirstlane(seqs.find(u / p.Hkv));
    const int L = __builtin_amdgcn_readfirstlane(seqs.length(s));
    const int U0 = __builtin_amdgcn_readfirstlane(seqs.before(s)) * p.Hkv;
    const int tiles = __builtin_amdgcn_readfirstlane(seqs.before(s + 1)) - U0 / p.Hkv;
    const int kvh = (u - U0) / tiles, j0 = u - U0 - kvh * tiles, j1 = min(tiles, j0 + (u_end - u));
    const int P0 = U0 + kvh * tiles;
    const int k = p.split ? share_id - P0 / share : 0;
    const int nseg = p.split ? (P0 + tiles - 1) / share - P0 / share + 1 : 1;
    u += j1 - j0;
    const int sub = rt * NW + w;                         // this wave's NG * 16 rows of the item
    const bool work = sub * NG * 16 < p.rows;
    const int it = (s * p.Hkv + kvh) * p.n_rt + sub;
    if (p.split && work && k == 0 && lane == 0) p.meta[it] = int2{nseg, (share_id * p.n_wide + rt) * NW + w};
    const int n_valid = (L + p.R + 15) >> 4;
    const int32_t* pt = p.table + (size_t)s * p.max_pages;
    // the wave's page of the next 64 tiles, a lane each
    auto page_ids = [&](int j) { return pt[min((j + lane) * 2 + (cpage & 1), n_valid - 1)]; };
    int ids = page_ids(j0), ids_at = j0;
    Rows<__bf16, D, NG> row;
    row.load(p, s, kvh, sub * NG * 16);
    // The queries' loads end here, and the registers are then as if made anew:
    // the compiler cannot tell inside the loop that they have ended, and would
    // wait for the tiles' copies as well.
    wait_loads<0>();
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) asm volatile("" : "+v"(row.q[g][i]));
    ids = checked_page(p, ids);
    asm volatile("" : "+v"(ids));
    f32x4 o[NG][DG];
    float m[NG], l[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      m[g] = -INFINITY;
      l[g] = 0.f;
#pragma unroll
      for (int d = 0; d < DG; ++d) o[g][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (again) __syncthreads();   // the last segment's tiles are read
    again = true;
    auto issue = [&](char* stage, int j) {
      if (j - ids_at >= 64) {
        ids_at = j;
        ids = checked_page(p, page_ids(j));
      }
      const int id = __builtin_amdgcn_readlane(ids, j - ids_at);
      const char* base = pool + ((size_t)(uint32_t)id * p.Hkv + kvh) * PAGE_B;
      char* to = stage + cpage * PAGE_B;
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        __builtin_amdgcn_global_load_lds((const void*)(base + soff[i]),
                                         (__attribute__((address_space(3))) void*)(to + seg(i) * 1024), 16, 0, 0);
    };
    auto scores = [&](const char* tile, f32x4 (&sc)[NG][2]) {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[g][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const bf16x8 kf = *(const bf16x8*)(tile + kfrag[ks] + t * 4 * 2 * D);
#pragma unroll
          for (int g = 0; g < NG; ++g)
            sc[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8, row.q[g][ks]), sc[g][t], 0, 0, 0);
        }
    };
    // Step j: the next tile's scores into `nxt` under this tile's softmax (`cur`
    // holds its scores), then this tile's values.  At its start the next
    // tile's copies are awaited, this wave's and by the barrier everybody's,
    // and the stage of the tile before this one, which every wave is past,
    // takes tile j + STAGES - 1.
    auto step = [&](auto masked, auto last, const char* tile, const char* next, char* free, int j,
                    f32x4 (&cur)[NG][2], f32x4 (&nxt)[NG][2]) {
      constexpr bool MASKED = decltype(masked)::value != 0, LAST = decltype(last)::value != 0;
      if constexpr (!LAST) {
        if (j + STAGES - 2 < j1) wait_loads<(STAGES - 3) * NPL>();
        else if (j + 3 < j1) wait_loads<2 * NPL>();
        else if (j + 2 < j1) wait_loads<NPL>();
        else wait_loads<0>();
        barrier();
        if (j + STAGES - 1 < j1) issue(free, j + STAGES - 1);
      }
      if (!work) return;
      uint32_t bits[NG];
      if constexpr (MASKED) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t b = bits[g] = seen_bits<8>(p, row.mask(p, s, g), row.r[g], row.any[g], j * KEYS + quarter * 8, L);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!(b >> i & 1)) cur[g][i >> 2][i & 3] = -INFINITY;
        }
      }
      if constexpr (!LAST) scores(next, nxt);
      // the values' reads are on their way under the softmax
      u32x4 vf[DG];
#pragma unroll
      for (int d = 0; d < DG; ++d) vf[d] = *(const u32x4*)(tile + vfrag + d * 512);
      bf16x8 pf[NG];
      softmax_tile<__bf16, 2, NG, DG>(cur, pf, p.scale_log2, m, l, o);
      if constexpr (MASKED)
        clean_values<__bf16>(vf, bits, o, [&](int key) {
          return (const __bf16*)(tile + TILE_B + (key >> 4) * PAGE_B) + (key & 15);
        });
#pragma unroll
      for (int d = 0; d < DG; ++d) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
          o[g][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]), pf[g], o[g][d], 0, 0, 0);
      }
    };
    auto stage = [&](auto c) -> char* {
      constexpr int I = decltype(c)::value % STAGES;
      if constexpr (I == 0) return st0;
      else if constexpr (I == 1) return st1;
      else if constexpr (I == 2) return st2;
      else if constexpr (I == 3) return st3;
      else if constexpr (I == 4) return st4;
      else return st5;
    };
    static_for<0, STAGES - 1>([&](auto c) {
      if (j0 + decltype(c)::value < j1) issue(stage(c), j0 + decltype(c)::value);
    });
    if (j0 + STAGES - 2 < j1) wait_loads<(STAGES - 2) * NPL>();
    else if (j0 + 3 < j1) wait_loads<3 * NPL>();
    else if (j0 + 2 < j1) wait_loads<2 * NPL>();
    else if (j0 + 1 < j1) wait_loads<NPL>();
    else wait_loads<0>();
    barrier();
    f32x4 sa[NG][2], sb[NG][2];
    if (work) scores(st0, sa);
    // steps below L whose tile is not the last, then those that reach the window
    const int jm = max(j0, min(j1 - 1, L / KEYS));
    for (int j = j0; j < jm; j += STAGES)
      static_for<0, STAGES>([&](auto c) {
        constexpr int C = decltype(c)::value;
        if (j + C < jm) {
          if constexpr (C % 2 == 0) step(IC<0>{}, IC<0>{}, stage(c), stage(IC<C + 1>{}), stage(IC<C + STAGES - 1>{}), j + C, sa, sb);
          else step(IC<0>{}, IC<0>{}, stage(c), stage(IC<C + 1>{}), stage(IC<C + STAGES - 1>{}), j + C, sb, sa);
        }
      });
    auto at = [&](int j) {
      const int i = (j - j0) % STAGES;
      return i == 0 ? st0 : i == 1 ? st1 : i == 2 ? st2 : i == 3 ? st3 : i == 4 ? st4 : st5;
    };
    if ((jm - j0) & 1) {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int t = 0; t < 2; ++t) sa[g][t] = sb[g][t];
    }
    for (int j = jm; j + 1 < j1; ++j) {
      step(IC<1>{}, IC<0>{}, at(j), at(j + 1), at(j + STAGES - 1), j, sa, sb);
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int t = 0; t < 2; ++t) sa[g][t] = sb[g][t];
    }
    step(IC<1>{}, IC<1>{}, at(j1 - 1), st0, st0, j1 - 1, sa, sb);
    if (!work) continue;
    const size_t slot = (size_t)((share_id * p.n_wide + rt) * NW + w) * 2 + (k == 0 ? 1 : 0);
    finish_rows<__bf16, D, NG>(p, s, row, m, l, o, nseg, slot);
  }
}

// The segments of a split item, in their order: a wave a (group of 16 rows, NQ
// times 16 elements of the head), SB segments on their way at a time.  Few items:
// more waves and more segments at a time; many: fewer and longer ones (pieces and
// segments at a time, whole calls: long documents 1, 8 460 us; 8, 2 450; 4, 4 445;
// serving 97.0, 96.7 and 94.4).
template <typename T, int D, int NG, int NQ, int SB>
__global__ void __launch_bounds__(256) tree_attn_merge_kernel(TreeAttn p) {
  constexpr int DG = D / 16, PER = NG * DG / NQ;
  const int lane = threadIdx.x & 63, m16 = lane & 15, quarter = lane >> 4;
  const long long task = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int HN = p.Hkv * p.n_rt;
  const int it = (int)(task / PER), gd = (int)(task - (long long)it * PER) * NQ, g = gd / DG, d0 = gd % DG;
  if (it >= p.S * HN) return;
  const int s = it / HN, qi = it - s * HN, kvh = qi / p.n_rt, rt = qi - kvh * p.n_rt;
  const int2 mt = p.meta[it];
  const int L = p.kv_len[s];
  if (L < 0 || (long long)L + p.R > (long long)p.max_pages * DVS_PAGE_SIZE) return;
  const int nseg = mt.x, first = mt.y;
  if (nseg <= 1) return;
  const int n = (rt * NG + g) * 16 + m16;
  const int step = p.n_wide ? p.n_wide * NW : 1;   // from a share's slot to the next one's
  auto slot = [&](int c) { return (size_t)(first + c * step) * 2 + (c == 0 ? 1 : 0); };
  auto ml_of = [&](int c) { return *(const f32x2*)(p.part_ml + ((slot(c) * NG + g) * 16 + m16) * 2); };
  f32x4 acc[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float M = -INFINITY, l = 0.f;
  for (int c0 = 0; c0 < nseg; c0 += SB) {
    f32x2 ml[SB];
    f32x4 x[SB][NQ];
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      const int c = min(c0 + b, nseg - 1);
      ml[b] = ml_of(c);
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        x[b][i] = *(const f32x4*)(p.part_o + ((slot(c) * NG + g) * DG + d0 + i) * 256 + lane * 4);
    }
    float top = M;
#pragma unroll
    for (int b = 0; b < SB; ++b)
      if (ml[b][1] != 0.f) top = fmaxf(top, ml[b][0]);   // the last segment's repeats change nothing
    const float back = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - top);
    const float ref = top == -INFINITY ? 0.f : top;
    M = top;
    l *= back;
#pragma unroll
    for (int i = 0; i < NQ; ++i) acc[i] *= back;
#pragma unroll
    for (int b = 0; b < SB; ++b) {
      if (c0 + b >= nseg || ml[b][1] == 0.f) continue;
      const float e = __builtin_amdgcn_exp2f(ml[b][0] - ref);
      l = fmaf(e, ml[b][1], l);
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(e, x[b][i][j], acc[i][j]);
    }
  }
  if (n >= p.rows) return;
  const int r = n / p.G, h = kvh * p.G + n - r * p.G;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* dst = (T*)p.out + (((size_t)s * p.R + r) * p.Hq + h) * D + d0 * 16 + quarter * 4;
#pragma unroll
  for (int i = 0; i < NQ; ++i) store4(dst + i * 16, acc[i] * inv);
}

struct TreePlan {
  int ng, n_rt, n_wide, grid, split, seqs;   // seqs: sequences a launch takes
  size_t off_ml, off_o, bytes;
};

constexpr long long MAX_ROWS = 1 << 20;   // query rows of a sequence, all heads

static bool tree_fits(int R, int Hq, int max_pages) {   // what the kernels count in 32 bits
  return (long long)R * Hq <= MAX_ROWS && (long long)R * Hq * max_pages < (1LL << 30) && max_pages <= TREE_MAX_PAGES;
}

static TreePlan tree_plan(int S, int R, int Hq, int Hkv, int D, int max_pages, int dtype) {
  TreePlan pl{};
  const int rows = R * (Hq / Hkv);
  const int keys = dtype == DVS_BF16 ? Tile<__bf16>::KEYS : Tile<float>::KEYS;
  const int max_tiles = (int)(((long long)max_pages * DVS_PAGE_SIZE + keys - 1) / keys);
  const int cus = device_cus();
  // Few tiles (under three a wave of 16 rows): 16 rows a wave, and not the tiles
  // through LDS, so that there are as many waves as can be (us, 16 rows a wave /
  // otherwise: 256 rows, one sequence of 2048 19.7 / 26.8; 128 rows, one of 4000 20.0
  // / 20.8, of 8000 25.7 / 24.2, of 16000 43 / 30; 64 rows, 8 of 1k-2k 21.3 / 20.2; fp32,
  // 128 rows, one of 2048 24.4 / 29.2, 64 rows, 32 of 1k-4k 204 / 149).  Short tables
  // need no merge, and may be more: 16 of 300-900, 128 rows 21.4 / 23.2.
  const long long a_wave = (long long)std::min(S, MAX_SEQS) * Hkv * ((rows + 15) / 16) * max_tiles / (8 * cus);
  const bool few = a_wave < (max_tiles <= 32 ? 8 : 3);
  // Tiles through LDS otherwise, for more than 16 rows (us, waves on their own /
  // through LDS: 32 rows, 32 sequences of 1k-8k 73.2 / 69.5, 16 of 3k-6k 44.6 / 38.5;
  // 16 rows, 32 of 1k-8k 64.7 / 66.5), in short tables for more than 32 (32 rows,
  // 256 of 100-400 38.9 / 44.4).
  const bool wide = dtype == DVS_BF16 && !few && rows > (max_tiles <= 32 ? 32 : 16);
  pl.ng = !few && rows > (wide ? NW * 16 : 16) ? 2 : 1;
  pl.n_rt = (rows + pl.ng * 16 - 1) / (pl.ng * 16);
  const long long per_seq = (long long)Hkv * pl.n_rt * max_tiles;
  pl.seqs = (int)std::max<long long>(1, std::min<long long>({S, MAX_SEQS, (1LL << 30) / per_seq,
                                                             (1LL << 22) / ((long long)Hkv * pl.n_rt)}));
  const long long items = (long long)pl.seqs * Hkv * pl.n_rt;
  // Through LDS: a workgroup a CU, whose waves take 16 rows each up to 128 rows, 32
  // beyond (128 rows, two workgroups of four waves of 32 / eight of 16, us: 32 of 1k-8k
  // 92 / 87.5, 64 of 1k-1.9k 66.8 / 48.5); two workgroups where the registers are enough
  // (heads of 64, 128 rows, 32 of 1k-8k, one / two 54.7 / 51.0).
  if (wide) {
    pl.n_wide = (pl.n_rt + NW - 1) / NW;
    pl.grid = std::max(1, (D == 64 && pl.ng == 1 ? 2 : 1) * cus / pl.n_wide);
  } else {
    pl.grid = 2 * cus;
  }
  // Whole items, and no merge, where a wave's tiles then are at most 8 more than
  // with all cut to equal shares: a merge and its launch take that long (cut /
  // whole, us: 64 sequences of 200-500, 16 rows 20.3 / 13.1; 256 of 100-400, 32 rows
  // 58.6 / 38.5; 128 of 500-1900 87.9 / 75.1).  Only tables of up to 64 tiles: lengths
  // differ, and a long one must not be left to a wave.
  const int per = wide ? 1 : FW;   // waves that share a segment's tiles
  const long long units = (long long)pl.seqs * Hkv * (wide ? 1 : pl.n_rt), tiles = units * max_tiles;
  const long long whole = (units + pl.grid - 1) / pl.grid * ((max_tiles + per - 1) / per);
  const long long cut = std::max(1LL, tiles / ((long long)pl.grid * per));
  pl.split = max_tiles > 64 || whole - cut > 8;
  pl.grid = (int)std::min<long long>(pl.grid, pl.split ? (tiles + 3) / 4 : units);
  if (wide) pl.grid *= pl.n_wide;
  if (pl.split) {
    const size_t slots = (size_t)pl.grid * (wide ? NW : 1) * 2;
    pl.off_ml = al256((size_t)items * sizeof(int2));
    pl.off_o = pl.off_ml + al256(slots * pl.ng * 16 * 2 * sizeof(float));
    pl.bytes = pl.off_o + slots * pl.ng * 16 * D * sizeof(float);
  } else {
    pl.bytes = 256;
  }
  return pl;
}

template <typename T, int D, int NG>
static void launch_merge(long long groups, const TreeAttn& p, hipStream_t st) {
  constexpr int MANY = D == 96 ? 3 : 4;
  if (groups < MERGE_FEW)
    hipLaunchKernelGGL((tree_attn_merge_kernel<T, D, NG, 1, 8>), dim3((unsigned)((groups * (D / 16) + 3) / 4)), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((tree_attn_merge_kernel<T, D, NG, MANY, 4>), dim3((unsigned)((groups * (D / 16 / MANY) + 3) / 4)), dim3(256), 0, st, p);
}

template <typename T, int D>
static void launch_tree(const TreePlan& pl, const TreeAttn& p, hipStream_t st) {
  if (pl.n_wide) {
    if constexpr (sizeof(T) == 2) {
      if (pl.ng == 2) hipLaunchKernelGGL((tree_attn_tile_kernel<D, 2>), dim3(pl.grid), dim3(NW * 64), 0, st, p);
      else hipLaunchKernelGGL((tree_attn_tile_kernel<D, 1>), dim3(pl.grid), dim3(NW * 64), 0, st, p);
    }
  } else {
    if (pl.ng == 2) hipLaunchKernelGGL((tree_attn_wave_kernel<T, D, 2>), dim3(pl.grid), dim3(FW * 64), 0, st, p);
    else hipLaunchKernelGGL((tree_attn_wave_kernel<T, D, 1>), dim3(pl.grid), dim3(FW * 64), 0, st, p);
  }
  if (!pl.split) return;
  const long long groups = (long long)p.S * p.Hkv * p.n_rt * pl.ng;
  if (pl.ng == 2) launch_merge<T, D, 2>(groups, p, st);
  else launch_merge<T, D, 1>(groups, p, st);
}

}  // namespace dvs

using namespace dvs;

extern "C" size_t dvs_tree_workspace_bytes(int32_t S, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                                           int32_t max_pages, int32_t dtype) {
  if (S < 1 || R < 1 || R > 1024 || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 ||
      (D != 64 && D != 96 && D != 128) || max_pages < 1 || (dtype != DVS_F32 && dtype != DVS_BF16) ||
      !tree_fits(R, Hq, max_pages))
    return 0;
  return tree_plan(S, R, Hq, Hkv, D, max_pages, dtype).bytes;
}

extern "C" int attn_tree(const void* q, const void* k_pool, const void* v_pool,
                         const int32_t* page_table, const int32_t* kv_len, const int32_t* tree_mask,
                         int32_t S, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                         int32_t max_pages, int32_t num_pool_pages, float softmax_scale,
                         int32_t dtype, void* out, int32_t* err_word, void* workspace,
                         size_t ws_bytes, void* stream) {
  clear_error();
  DVS_CHECK_ARG(q && k_pool && v_pool && page_table && kv_len && out, "attn_tree: NULL array argument");
  DVS_CHECK_ARG(S >= 1 && R >= 1 && R <= 1024, "attn_tree: need S >= 1 and 1 <= R <= 1024");
  DVS_CHECK_ARG(Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0, "attn_tree: Hq %% Hkv != 0");
  DVS_CHECK_ARG(max_pages >= 1 && num_pool_pages >= 1, "attn_tree: empty page table/pool");
  DVS_CHECK_ARG(softmax_scale > 0.f && isfinite(softmax_scale), "attn_tree: softmax_scale must be positive");
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "attn_tree: dtype %d", dtype);
  DVS_CHECK_SUPPORTED(D == 64 || D == 96 || D == 128, "attn_tree: head_dim %d", D);
  DVS_CHECK_ARG((((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_pool | (uintptr_t)v_pool) & 15) == 0,
                "attn_tree: q, out and the pools must start on 16 bytes");
  DVS_CHECK_SUPPORTED(tree_fits(R, Hq, max_pages), "attn_tree: R * Hq must be at most 2^20, its product with max_pages below 2^30, max_pages below 2^27 - 3");
  const TreePlan pl = tree_plan(S, R, Hq, Hkv, D, max_pages, dtype);
  if (!workspace || ws_bytes < pl.bytes) {
    set_error("attn_tree: workspace needs %zu bytes, got %zu", pl.bytes, ws_bytes);
    return DVS_EWORKSPACE;
  }
  DVS_CHECK_ARG(((uintptr_t)workspace & 255) == 0, "attn_tree: workspace must start on 256 bytes");
  TreeAttn p{};
  p.k_pool = k_pool; p.v_pool = v_pool; p.err = err_word;
  p.R = R; p.W = (R + 31) / 32; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.rows = R * p.G;
  p.n_rt = pl.n_rt; p.max_pages = max_pages; p.pool_pages = num_pool_pages;
  p.n_wide = pl.n_wide; p.split = pl.split;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.meta = (int2*)workspace;
  p.part_ml = (float*)((char*)workspace + pl.off_ml);
  p.part_o = (float*)((char*)workspace + pl.off_o);
  hipStream_t st = (hipStream_t)stream;
  const size_t row = (size_t)R * Hq * D * (dtype == DVS_BF16 ? 2 : 4);
  for (int s0 = 0; s0 < S; s0 += pl.seqs) {
    p.S = std::min(S - s0, pl.seqs);
    p.q = (const char*)q + s0 * row;
    p.out = (char*)out + s0 * row;
    p.table = page_table + (size_t)s0 * max_pages;
    p.kv_len = kv_len + s0;
    p.mask = tree_mask ? tree_mask + (size_t)s0 * R * p.W : nullptr;
    if (dtype == DVS_BF16) {
      if (D == 128) launch_tree<__bf16, 128>(pl, p, st);
      else if (D == 96) launch_tree<__bf16, 96>(pl, p, st);
      else launch_tree<__bf16, 64>(pl, p, st);
    } else {
      if (D == 128) launch_tree<float, 128>(pl, p, st);
      else if (D == 96) launch_tree<float, 96>(pl, p, st);
      else launch_tree<float, 64>(pl, p, st);
    }
    const int rc = launch_status("attn_tree");
    if (rc) return rc;
  }
  return DVS_OK;
}
