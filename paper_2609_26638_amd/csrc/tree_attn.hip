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
constexpr float RESCALE_LOG2 = 8.f, WEIGHT_MAX = 8 * 256.f;
constexpr int TILE_ROWS = 32, TILE_MIN_TILES = 2048, TILE_SHARE = 8;
constexpr int WAVE_WHOLE = 8, WAVE_SHARE = 4;
constexpr int MERGE_FEW = 1024;

struct TreeAttn {
  const void *q, *k_pool, *v_pool;
  const int32_t *table, *kv_len, *mask;
  void* out;
  int32_t* err;
  int S, R, W, Hq, Hkv, G, rows, n_rt, max_pages, pool_pages;
  int n_wide;      // row tiles of 128 (0: waves on their own)
  int split;       // items are cut where a wave's share ends, and merged by a launch of its own
  int share_min;   // tiles of a share, at least
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
// a lane's weights add up to more than 8 x 2^RESCALE_LOG2 (or to no number: m
// starts at -inf) the rows' maxima are found, m moves to those that exceed it by
// RESCALE_LOG2, and the tile's weights are made again.  Long documents: 520 us
// with the maxima of every tile, XXX without.
template <int NS, int NG, int DG>
__device__ __forceinline__ void softmax_tile(const f32x4 (&s)[NG][NS], f32x4 (&w)[NG][NS],
                                             float scale_log2, float (&m)[NG], float (&l)[NG],
                                             f32x4 (&o)[NG][DG]) {
  float sum[NG];
  bool over = false;
  auto weigh = [&](int g, float ref) {
#pragma unroll
    for (int t = 0; t < NS; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[g][t][i] = __builtin_amdgcn_exp2f(fmaf(s[g][t][i], scale_log2, -ref));
    sum[g] = (w[g][0][0] + w[g][0][1]) + (w[g][0][2] + w[g][0][3]);
    if constexpr (NS == 2) sum[g] += (w[g][1][0] + w[g][1][1]) + (w[g][1][2] + w[g][1][3]);
  };
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    weigh(g, m[g]);
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
      weigh(g, m[g] == -INFINITY ? 0.f : m[g]);
    }
  }
#pragma unroll
  for (int g = 0; g < NG; ++g) l[g] += sum[g];
}

// Tiles before each sequence (s_seq[0 .. S]) and the lengths, by the whole
// workgroup; sequences that do not fit their table have none.
__device__ __forceinline__ void seq_tiles(const TreeAttn& p, int keys, int* s_seq, int* s_len, int* s_tot) {
  const int tid = threadIdx.x, lane = tid & 63, nw = blockDim.x >> 6;
  int carry = 0;
  for (int s0 = 0; s0 < p.S; s0 += blockDim.x) {
    const int s = s0 + tid;
    int t = 0;
    if (s < p.S) {
      const int L = p.kv_len[s];
      s_len[s] = L;
      if (L < 0 || (long long)L + p.R > (long long)p.max_pages * DVS_PAGE_SIZE) {
        if (blockIdx.x == 0) set_err(p.err, DVS_ERR_MAX_PAGES);
      } else {
        t = (L + p.R + keys - 1) / keys;
      }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(t, off);
      if (lane >= off) t += v;
    }
    if (s0) __syncthreads();
    if (lane == 63) s_tot[tid >> 6] = t;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < nw; ++w) {
      const int v = s_tot[w];
      if (w < (tid >> 6)) before += v;
      carry += v;
    }
    if (s < p.S) s_seq[1 + s] = before + t;
  }
  if (tid == 0) s_seq[0] = 0;
  __syncthreads();
}

// The sequence that holds tile u of one item a sequence.
__device__ __forceinline__ int find_seq(const int* s_seq, int S, int u) {
  int lo = 0, hi = S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s_seq[mid] <= u) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Consecutive workgroups on one XCD (blockIdx goes round the eight): row tiles
// of an item then find its keys in their L2.
__device__ __forceinline__ int xcd_block() {
  const int n = gridDim.x, q = n >> 3, rem = n & 7, x = blockIdx.x & 7, i = blockIdx.x >> 3;
  return x * q + min(x, rem) + i;
}

// Whether a row's mask (NULL: causal) has a bit of the window.
__device__ __forceinline__ bool sees_any(const TreeAttn& p, const uint32_t* mask) {
  if (!mask) return true;
  uint32_t bits = 0;
  for (int i = 0; i < p.W; ++i) bits |= i == p.W - 1 && (p.R & 31) ? mask[i] & ((1u << (p.R & 31)) - 1) : mask[i];
  return bits != 0;
}

// The two halves of word e of 8 bf16 values whose bits of `un` are set.
__device__ __forceinline__ uint32_t pair_mask(uint32_t un, int e) {
  return (un >> (2 * e) & 1 ? 0xffffu : 0u) | (un >> (2 * e + 1) & 1 ? 0xffff0000u : 0u);
}

// The weights of a lane's 8 keys, rounded once (bf16: what the matrix
// instruction takes; l is summed before the rounding).
__device__ __forceinline__ bf16x8 weights_bf16(const f32x4 (&s)[2]) {
  u32x4 pk;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    pk[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                                             f32x2{s[e >> 1][2 * (e & 1)], s[e >> 1][2 * (e & 1) + 1]}, bf16x2));
  return __builtin_bit_cast(bf16x8, pk);
}

// End of a segment: the output, or a part of it (O, m and l in 32 bits).  l is
// 0 exactly for a row that sees nothing, whatever its O holds.
template <typename T, int D, int NG>
__device__ __forceinline__ void finish_rows(const TreeAttn& p, int s, const int (&r)[NG], const int (&h)[NG],
                                            const bool (&valid)[NG], const bool (&any)[NG],
                                            const float (&m)[NG], float (&l)[NG],
                                            const f32x4 (&o)[NG][D / 16], int nseg, size_t slot) {
  const int lane = threadIdx.x & 63, m16 = lane & 15, quarter = lane >> 4;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    l[g] = rows_sum(l[g]);
    if (!any[g]) l[g] = 0.f;
    if (nseg > 1) {
      if (quarter == 0) *(f32x2*)(p.part_ml + ((slot * NG + g) * 16 + m16) * 2) = f32x2{m[g], l[g]};
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
        *(f32x4*)(p.part_o + ((slot * NG + g) * (D / 16) + d) * 256 + lane * 4) = o[g][d];
    } else if (valid[g]) {
      T* dst = (T*)p.out + (((size_t)s * p.R + r[g]) * p.Hq + h[g]) * D + quarter * 4;
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

// ---------------------------------------------------------------------------
// Every wave on its own: NG groups of 16 query rows (row n of a KV head is
// window row n / G, head n % G of its group) and a share of the key tiles,
// straight from the cache into registers; the next tile's keys are on their
// way under this one's softmax, its values under the next one's scores.
// ---------------------------------------------------------------------------
template <typename T, int D, int NG>
__global__ void __launch_bounds__(256, 2) tree_attn_wave_kernel(TreeAttn p) {
  using TL = Tile<T>;
  constexpr int KEYS = TL::KEYS, NP = D / 16, NQP = D / TL::NQ_DIV, DG = D / 16, NS = TL::NS;
  constexpr int PAGE_B = 16 * D * (int)sizeof(T);
  __shared__ int s_seq[MAX_SEQS + 1], s_len[MAX_SEQS], s_tot[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m16 = lane & 15, quarter = lane >> 4;
  const int HN = p.Hkv * p.n_rt;
  const int share_id = xcd_block() * 4 + w, n_shares = gridDim.x * 4;
  int u = share_id, u_end = p.S * HN, share = 0;
  if (p.split) {
    seq_tiles(p, KEYS, s_seq, s_len, s_tot);
    const int U = s_seq[p.S] * HN;
    share = max((U + n_shares - 1) / n_shares, p.share_min);
    u = min((long long)share_id * share, (long long)U);
    u_end = min(u + share, U);
  }
  const char* kp = (const char*)p.k_pool;
  const char* vp = (const char*)p.v_pool;
  const uint32_t koff = TL::template k_off<D>(m16, quarter), voff = TL::v_off(m16, quarter);
  const int kpage = TL::template k_page<D>(m16, quarter), vpage = TL::v_page(quarter);

  while (u < u_end) {
    int s, qi, j0, j1, tiles, k = 0, nseg = 1, L;
    if (p.split) {
      s = find_seq(s_seq, p.S, u / HN);
      L = s_len[s];
      tiles = s_seq[s + 1] - s_seq[s];
      const int local = u - s_seq[s] * HN;
      qi = local / tiles;
      j0 = local - qi * tiles;
      j1 = min(tiles, j0 + (u_end - u));
      const int P0 = s_seq[s] * HN + qi * tiles;
      k = share_id - P0 / share;
      nseg = (P0 + tiles - 1) / share - P0 / share + 1;
      u += j1 - j0;
    } else {
      s = u / HN;
      qi = u - s * HN;
      L = p.kv_len[s];
      u += n_shares;
      if (L < 0 || (long long)L + p.R > (long long)p.max_pages * DVS_PAGE_SIZE) {
        if (lane == 0) set_err(p.err, DVS_ERR_MAX_PAGES);
        continue;
      }
      j0 = 0;
      j1 = tiles = (L + p.R + KEYS - 1) / KEYS;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    L = __builtin_amdgcn_readfirstlane(L);
    const int it = s * HN + qi, kvh = qi / p.n_rt, rt = qi - kvh * p.n_rt;
    if (p.split && k == 0 && lane == 0) p.meta[it] = int2{nseg, share_id};
    const int n_valid = (L + p.R + 15) >> 4;
    const int32_t* pt = p.table + (size_t)s * p.max_pages;
    // the ids of the next 64 pages, a lane each
    auto page_ids = [&](int j) {
      int id = pt[min(j * TL::PAGES + lane, n_valid - 1)];
      if (id < 0 || id >= p.pool_pages) {
        set_err(p.err, DVS_ERR_BAD_PAGE);
        id = 0;
      }
      return id;
    };
    int ids = page_ids(j0), ids_at = j0;
    // this lane's query rows
    int r[NG], h[NG];
    bool valid[NG], any[NG];
    const uint32_t* mask[NG];
    u32x4 q[NG][NQP];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int n = (rt * NG + g) * 16 + m16;
      valid[g] = n < p.rows;
      r[g] = valid[g] ? n / p.G : 0;
      h[g] = kvh * p.G + (valid[g] ? n - r[g] * p.G : 0);
      const T* src = (const T*)p.q + (((size_t)s * p.R + r[g]) * p.Hq + h[g]) * D;
#pragma unroll
      for (int i = 0; i < NQP; ++i) q[g][i] = *(const u32x4*)(src + TL::q_elem(quarter, i));
      mask[g] = p.mask ? (const uint32_t*)p.mask + ((size_t)s * p.R + r[g]) * p.W : nullptr;
      any[g] = valid[g] && sees_any(p, mask[g]);
    }
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
    load_k(j0);
    load_v(j0);
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
                __builtin_bit_cast(bf16x8, kf[i]), __builtin_bit_cast(bf16x8, q[g][i >> 1]), sc[g][i & 1], 0, 0, 0);
        } else {
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[g][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[i][e]), __uint_as_float(q[g][i][e]),
                                                              sc[g][0], 0, 0, 0);
        }
      }
      const bool more = j + 1 < j1;
      // the ids run out: those of the tiles from j on (this tile's are still
      // needed for nothing, the next one's are)
      if (more && (j + 2 - ids_at) * TL::PAGES > 64) {
        ids_at = j + 1;
        ids = page_ids(ids_at);
      }
      if (more) load_k(j + 1);
      const int key0 = j * KEYS + quarter * TL::NK;
      const bool masked = (j + 1) * KEYS > L;
      if (masked) {
        uint32_t un = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t b = seen_bits<TL::NK>(p, mask[g], r[g], any[g], key0, L);
          un |= b;
#pragma unroll
          for (int i = 0; i < TL::NK; ++i)
            if (!(b >> i & 1)) sc[g][i >> 2][i & 3] = -INFINITY;
        }
        // values that none of the wave's rows sees may be anything: zero
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) un |= __shfl_xor((int)un, off);
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2)
              vf[i][e] &= pair_mask(un, e);
            else
              vf[i][e] &= un >> e & 1 ? 0xffffffffu : 0u;
          }
      }
      f32x4 wt[NG][NS];
      softmax_tile<NS, NG, DG>(sc, wt, p.scale_log2, m, l, o);
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        if constexpr (sizeof(T) == 2) {
          const bf16x8 pf = weights_bf16(wt[g]);
#pragma unroll
          for (int d = 0; d < DG; ++d)
            o[g][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[d]), pf, o[g][d], 0, 0, 0);
        } else {
#pragma unroll
          for (int d = 0; d < DG; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              o[g][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[d][e]), wt[g][0][e], o[g][d], 0, 0, 0);
        }
      }
      if (more) load_v(j + 1);
    }
    finish_rows<T, D, NG>(p, s, r, h, valid, any, m, l, o, nseg, (size_t)share_id * 2 + (k == 0 ? 1 : 0));
  }
}

// ---------------------------------------------------------------------------
// Many query rows of a KV head (bf16): a workgroup of four waves, 32 rows each,
// over 32-key tiles that all of them read from LDS.  A wave copies one page of
// every tile, K (waves 0, 1) or V (2, 3), straight to LDS, STAGES - 1 tiles
// ahead.  Row tiles of 128 rows take the same key range side by side on one
// XCD (its L2 then gives the second reader what the first has fetched).
//
// LDS rows of K (a key, 2 D bytes) have their 16-byte chunks permuted so that
// the 16 keys of one product, read at the same chunk, lie in 16 different bank
// groups; in V (an element of the head, 32 bytes a page) the two halves swap.
// The stages are variables of their own and the loop over them is unrolled:
// the compiler then knows that a read of one does not touch the copies on
// their way into the others, and does not wait for those.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ int k_swizzle(int row) {
  if constexpr (D == 128) return (row & 3) | ((row >> 1) & 12);
  else if constexpr (D == 96) return (row >> 3) & 3;
  else return ((row >> 1) & 1) | ((row >> 2) & 6);
}
__device__ __forceinline__ int v_swizzle(int d) { return ((d >> 2) ^ (d >> 3)) & 1; }

template <int N>
__device__ __forceinline__ void wait_loads() {   // at most N vector loads on their way
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

template <int D>
__global__ void __launch_bounds__(256, 2) tree_attn_tile_kernel(TreeAttn p) {
  constexpr int KEYS = 32, NG = 2, DG = D / 16, STAGES = 4;
  constexpr int PAGE_B = 32 * D, TILE_B = 2 * PAGE_B;   // bytes of a page, of a tile's K (or V)
  constexpr int NPL = PAGE_B / 1024;                    // copies of a wave a tile
  constexpr int STAGE_B = 2 * TILE_B;
  __shared__ __attribute__((aligned(1024))) char st0[STAGE_B], st1[STAGE_B], st2[STAGE_B], st3[STAGE_B];
  __shared__ int s_seq[MAX_SEQS + 1], s_len[MAX_SEQS], s_tot[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m16 = lane & 15, quarter = lane >> 4;
  const int block = xcd_block(), n_shares = gridDim.x / p.n_wide;
  const int share_id = block / p.n_wide, rt = block - share_id * p.n_wide;
  seq_tiles(p, KEYS, s_seq, s_len, s_tot);
  const int U = s_seq[p.S] * p.Hkv;
  const int share = max((U + n_shares - 1) / n_shares, p.share_min);
  int u = (int)min((long long)share_id * share, (long long)U);
  const int u_end = min(u + share, U);
  // copies: lane's source offset in the page, of its 16 bytes of each 1 KB
  const char* pool = (const char*)(w < 2 ? p.k_pool : p.v_pool);
  uint32_t soff[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    const int off = i * 1024 + lane * 16;
    if (w < 2) {
      const int row = off / (2 * D), c = (off - row * 2 * D) >> 4;
      soff[i] = row * 2 * D + ((c ^ k_swizzle<D>((w & 1) * 16 + row)) << 4);
    } else {
      const int d = off >> 5;
      soff[i] = d * 32 + ((((off >> 4) & 1) ^ v_swizzle(d)) << 4);
    }
  }
  // fragments: K of product t = 0 (t = 1: four rows on), chunk ks * 4 + quarter
  const int krow = 8 * (m16 >> 2) + (m16 & 3), ksw = k_swizzle<D>(krow);
  int kfrag[D / 32];
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) kfrag[ks] = krow * 2 * D + (((ks * 4 + quarter) ^ ksw) << 4);
  const int vfrag = TILE_B + (quarter >> 1) * PAGE_B + m16 * 32 + (((quarter & 1) ^ v_swizzle(m16)) << 4);
  bool again = false;

  while (u < u_end) {
    const int s = __builtin_amdgcn_readfirstlane(find_seq(s_seq, p.S, u / p.Hkv));
    const int L = __builtin_amdgcn_readfirstlane(s_len[s]);
    const int tiles = s_seq[s + 1] - s_seq[s];
    const int local = u - s_seq[s] * p.Hkv;
    const int kvh = local / tiles, j0 = local - kvh * tiles, j1 = min(tiles, j0 + (u_end - u));
    const int P0 = s_seq[s] * p.Hkv + kvh * tiles;
    const int k = share_id - P0 / share, nseg = (P0 + tiles - 1) / share - P0 / share + 1;
    u += j1 - j0;
    const int sub = rt * 4 + w;                         // this wave's 32 rows of the item
    const bool work = sub * 32 < p.rows;
    const int it = (s * p.Hkv + kvh) * p.n_rt + sub;
    if (work && k == 0 && lane == 0) p.meta[it] = int2{nseg, (share_id * p.n_wide + rt) * 4 + w};
    const int n_valid = (L + p.R + 15) >> 4;
    const int32_t* pt = p.table + (size_t)s * p.max_pages;
    // the wave's page of the next 64 tiles, a lane each
    auto page_ids = [&](int j) {
      int id = pt[min((j + lane) * 2 + (w & 1), n_valid - 1)];
      if (id < 0 || id >= p.pool_pages) {
        set_err(p.err, DVS_ERR_BAD_PAGE);
        id = 0;
      }
      return id;
    };
    int ids = page_ids(j0), ids_at = j0;
    int r[NG], h[NG];
    bool valid[NG], any[NG];
    const uint32_t* mask[NG];
    u32x4 q[NG][D / 32];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int n = (sub * NG + g) * 16 + m16;
      valid[g] = n < p.rows;
      r[g] = valid[g] ? n / p.G : 0;
      h[g] = kvh * p.G + (valid[g] ? n - r[g] * p.G : 0);
      const __bf16* src = (const __bf16*)p.q + (((size_t)s * p.R + r[g]) * p.Hq + h[g]) * D + quarter * 8;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) q[g][i] = *(const u32x4*)(src + i * 32);
      mask[g] = p.mask ? (const uint32_t*)p.mask + ((size_t)s * p.R + r[g]) * p.W : nullptr;
      any[g] = valid[g] && sees_any(p, mask[g]);
    }
    // The queries' loads end here, and the registers are then as if made anew:
    // the compiler cannot tell inside the loop that they have ended, and would
    // wait for the tiles' copies as well.
    wait_loads<0>();
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) asm volatile("" : "+v"(q[g][i]));
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
        ids = page_ids(j);
      }
      const int id = __builtin_amdgcn_readlane(ids, j - ids_at);
      const char* base = pool + ((size_t)(uint32_t)id * p.Hkv + kvh) * PAGE_B;
      char* to = stage + w * PAGE_B;
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        __builtin_amdgcn_global_load_lds((const void*)(base + soff[i]),
                                         (__attribute__((address_space(3))) void*)(to + i * 1024), 16, 0, 0);
    };
    // Tile j, in `tile`: this wave's copies of it have arrived (those of later
    // tiles may be on their way), then everybody's; the stage that the tile
    // before left free takes tile j + STAGES - 1.
    auto step = [&](auto masked, char* tile, char* next, int j) {
      constexpr bool MASKED = decltype(masked)::value != 0;
      if (j + STAGES - 1 <= j1) wait_loads<(STAGES - 2) * NPL>();
      else if (j + 1 < j1) wait_loads<NPL>();
      else wait_loads<0>();
      __builtin_amdgcn_s_barrier();
      if (j + STAGES - 1 < j1) issue(next, j + STAGES - 1);
      if (!work) return;
      f32x4 sc[NG][2], wt[NG][2];
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
            sc[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8, q[g][ks]), sc[g][t], 0, 0, 0);
        }
      uint32_t un = 0;
      if constexpr (MASKED) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t b = seen_bits<8>(p, mask[g], r[g], any[g], j * KEYS + quarter * 8, L);
          un |= b;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!(b >> i & 1)) sc[g][i >> 2][i & 3] = -INFINITY;
        }
        // values that none of the wave's rows sees may be anything: zero
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) un |= __shfl_xor((int)un, off);
      }
      softmax_tile<2, NG, DG>(sc, wt, p.scale_log2, m, l, o);
      bf16x8 pf[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) pf[g] = weights_bf16(wt[g]);
#pragma unroll
      for (int d = 0; d < DG; ++d) {
        u32x4 vf = *(const u32x4*)(tile + vfrag + d * 512);
        if constexpr (MASKED) {
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[e] &= pair_mask(un, e);
        }
#pragma unroll
        for (int g = 0; g < NG; ++g)
          o[g][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), pf[g], o[g][d], 0, 0, 0);
      }
    };
    auto stage = [&](auto c) -> char* {
      constexpr int I = decltype(c)::value % STAGES;
      if constexpr (I == 0) return st0;
      else if constexpr (I == 1) return st1;
      else if constexpr (I == 2) return st2;
      else return st3;
    };
    static_for<0, STAGES - 1>([&](auto c) {
      if (j0 + decltype(c)::value < j1) issue(stage(c), j0 + decltype(c)::value);
    });
    // tiles below L, then the few that reach the window
    const int jm = max(j0, min(j1, L / KEYS));
    for (int j = j0; j < jm; j += STAGES)
      static_for<0, STAGES>([&](auto c) {
        constexpr int C = decltype(c)::value;
        if (j + C < jm) step(IC<0>{}, stage(c), stage(IC<C + STAGES - 1>{}), j + C);
      });
    for (int j = jm; j < j1; ++j) {
      const int i = (j - j0) % STAGES;
      char* at = i == 0 ? st0 : i == 1 ? st1 : i == 2 ? st2 : st3;
      char* free = i == 0 ? st3 : i == 1 ? st0 : i == 2 ? st1 : st2;
      step(IC<1>{}, at, free, j);
    }
    if (!work) continue;
    const size_t slot = (size_t)((share_id * p.n_wide + rt) * 4 + w) * 2 + (k == 0 ? 1 : 0);
    finish_rows<__bf16, D, NG>(p, s, r, h, valid, any, m, l, o, nseg, slot);
  }
}

// The segments of a split item, in their order: a wave a (group of 16 rows, NQ
// times 16 elements of the head), SB segments on their way at a time.  Few items:
// more waves and more segments at a time; many: fewer and longer ones (2048 items
// of two segments, 128 wide: 33 us with one piece a wave, XXX with all eight).
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
  const int step = p.n_wide ? p.n_wide * 4 : 1;   // from a share's slot to the next one's
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
  int ng, n_rt, n_wide, grid, split, share_min, seqs;   // seqs: sequences a launch takes
  size_t off_ml, off_o, bytes;
};

static TreePlan tree_plan(int S, int R, int Hq, int Hkv, int D, int max_pages, int dtype) {
  TreePlan pl{};
  const int rows = R * (Hq / Hkv);
  const int keys = dtype == DVS_BF16 ? Tile<__bf16>::KEYS : Tile<float>::KEYS;
  const int max_tiles = (max_pages * DVS_PAGE_SIZE + keys - 1) / keys;
  pl.ng = rows > 16 ? 2 : 1;
  pl.n_rt = (rows + pl.ng * 16 - 1) / (pl.ng * 16);
  const long long per_seq = (long long)Hkv * pl.n_rt * max_tiles;
  pl.seqs = (int)std::max<long long>(1, std::min<long long>(std::min(S, MAX_SEQS), (1LL << 30) / per_seq));
  const long long items = (long long)pl.seqs * Hkv * pl.n_rt;
  const int cus = device_cus();
  const long long kv_tiles = (long long)pl.seqs * Hkv * max_tiles;
  if (dtype == DVS_BF16 && rows > TILE_ROWS && kv_tiles >= TILE_MIN_TILES) {
    pl.n_wide = (rows + 127) / 128;
    pl.split = 1;
    pl.share_min = TILE_SHARE;
    const long long shares = std::min<long long>(std::max(1, 2 * cus / pl.n_wide), (kv_tiles + TILE_SHARE - 1) / TILE_SHARE);
    pl.grid = (int)(shares * pl.n_wide);
  } else {
    pl.split = max_tiles > WAVE_WHOLE;
    pl.share_min = WAVE_SHARE;
    const long long tiles = items * max_tiles;
    pl.grid = (int)std::min<long long>(2 * cus, ((pl.split ? (tiles + WAVE_SHARE - 1) / WAVE_SHARE : items) + 3) / 4);
  }
  if (pl.split) {
    const size_t slots = (size_t)pl.grid * 4 * 2;
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
  if (groups < MERGE_FEW)
    hipLaunchKernelGGL((tree_attn_merge_kernel<T, D, NG, 1, 8>), dim3((unsigned)((groups * (D / 16) + 3) / 4)), dim3(256), 0, st, p);
  else
    hipLaunchKernelGGL((tree_attn_merge_kernel<T, D, NG, D / 16, 2>), dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, st, p);
}

template <typename T, int D>
static void launch_tree(const TreePlan& pl, const TreeAttn& p, hipStream_t st) {
  if (pl.n_wide) {
    if constexpr (sizeof(T) == 2) hipLaunchKernelGGL(tree_attn_tile_kernel<D>, dim3(pl.grid), dim3(256), 0, st, p);
  } else if (pl.ng == 2) {
    hipLaunchKernelGGL((tree_attn_wave_kernel<T, D, 2>), dim3(pl.grid), dim3(256), 0, st, p);
  } else {
    hipLaunchKernelGGL((tree_attn_wave_kernel<T, D, 1>), dim3(pl.grid), dim3(256), 0, st, p);
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
      (D != 64 && D != 96 && D != 128) || max_pages < 1 || (dtype != DVS_F32 && dtype != DVS_BF16))
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
  const TreePlan pl = tree_plan(S, R, Hq, Hkv, D, max_pages, dtype);
  if (!workspace || ws_bytes < pl.bytes) {
    set_error("attn_tree: workspace needs %zu bytes, got %zu", pl.bytes, ws_bytes);
    return DVS_EWORKSPACE;
  }
  DVS_CHECK_SUPPORTED((long long)Hkv * pl.n_rt * max_pages < (1LL << 30), "attn_tree: too many pages");
  TreeAttn p{};
  p.k_pool = k_pool; p.v_pool = v_pool; p.err = err_word;
  p.R = R; p.W = (R + 31) / 32; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.rows = R * p.G;
  p.n_rt = pl.n_rt; p.max_pages = max_pages; p.pool_pages = num_pool_pages;
  p.n_wide = pl.n_wide; p.split = pl.split; p.share_min = pl.share_min;
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
