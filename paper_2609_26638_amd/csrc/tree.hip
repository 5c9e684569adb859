// A step over a tree of drafted tokens: tree_masks, kv_append_rope and
// accept_commit_tree (the attention between them is in tree_attn.hip).
//
// Row 0 of a window is the last committed token x0, every other row a drafted
// token whose parent is an earlier row.  A row attends to the cache and to its
// ancestors, is rotated at position kv_len + depth, and sits in the cache slot
// kv_len + row, so that siblings share a position but not a slot.  The commit
// keeps the slots of one path and moves them to the front of the window.
#include <math.h>

#include <algorithm>

#include "dvs_common.h"

namespace dvs {

constexpr int TREE_MAX_ROWS = 1024;

// ---------------------------------------------------------------------------
// tree_masks
//
// mask(r) = {r} U mask(parent r).  A wave holds 64 consecutive rows, a row a
// lane.  Pointer doubling inside the wave (log2 64 rounds of mask(r) |=
// mask(up r), up r = up(up r)) gives every row's ancestors among the 64 as one
// 64-bit word; the topmost of them, its lowest bit, names the parent further
// up by which the chain leaves the wave's rows.  With these in LDS a row goes up
// its chain a block of 64 rows at a time, a word of its mask a block.
// ---------------------------------------------------------------------------
struct MaskRow {
  uint64_t in;   // ancestors among the wave's rows, itself among them
  int up;        // the parent by which the chain leaves them; < 0: it ends
};

__device__ __forceinline__ uint64_t shfl64(uint64_t v, int src) {
  const uint32_t lo = __shfl((int)(uint32_t)v, src), hi = __shfl((int)(uint32_t)(v >> 32), src);
  return (uint64_t)hi << 32 | lo;
}

// N blocks of 64 rows at a time, block i from row first + i * step.  p: the row's
// parent, or below -1 for a row of the padding.
template <int N>
__device__ __forceinline__ void wave_ancestors(const int (&p)[N], int first, int step, int lane, MaskRow (&m)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) m[i] = MaskRow{1ull << lane, p[i] >= first + i * step ? p[i] - first - i * step : -1};
#pragma unroll
  for (int round = 0; round < 6; ++round)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int src = m[i].up >= 0 ? m[i].up : lane;
      const uint64_t other = shfl64(m[i].in, src);
      const int next = __shfl(m[i].up, src);
      m[i].in |= other;
      m[i].up = m[i].up >= 0 ? next : -1;
    }
#pragma unroll
  for (int i = 0; i < N; ++i) m[i].up = __shfl(p[i], __ffsll((unsigned long long)m[i].in) - 1);
}

// A row's parent as the kernels take it: a row that names itself or a later
// one is no tree's.
__device__ __forceinline__ int checked_parent(int p, int r, int32_t* err) {
  if (p >= r) {
    set_err(err, DVS_ERR_BAD_TREE);
    return -2;
  }
  return p;
}

// Up to 64 rows: a wave a sequence.  Latency: 2.3 us for 64 sequences of 64 rows.
__global__ void __launch_bounds__(256) tree_masks_small_kernel(const int32_t* __restrict__ parent,
                                                               int S, int R,
                                                               int32_t* __restrict__ mask,
                                                               int32_t* __restrict__ depth,
                                                               int32_t* __restrict__ err) {
  const int lane = threadIdx.x & 63, s = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (s >= S) return;
  const int p[1] = {lane < R ? checked_parent(parent[(size_t)s * R + lane], lane, err) : -2};
  MaskRow rows[1];
  wave_ancestors(p, 0, 0, lane, rows);
  const MaskRow m = rows[0];
  if (lane >= R) return;
  const bool in_tree = m.up == -1;
  const size_t at = (size_t)s * R + lane;
  if (depth) depth[at] = in_tree ? __popcll(m.in) - 1 : -1;
  const uint64_t w = in_tree ? m.in : 0;
  if (R > 32)
    *(u32x2*)(mask + 2 * at) = u32x2{(uint32_t)w, (uint32_t)(w >> 32)};
  else
    mask[at] = (int32_t)(uint32_t)w;
}

// More rows, up to NB blocks of 64: a workgroup takes 256 of a sequence's, makes
// the blocks up to its last row, then a wave its 64 rows' words, in registers,
// which go out through LDS, side by side.  The words to write bound it (128
// sequences of 1000 rows, 17 MB: 8.1 us; copied row by row from the parent's in 16
// steps of a workgroup a sequence: 18.4).  The first words reach memory late, after
// a chain of parents that is all latency.
template <int NB>
__global__ void __launch_bounds__(256) tree_masks_kernel(const int32_t* __restrict__ parent, int R,
                                                         int parts, bool wide, int32_t* __restrict__ mask,
                                                         int32_t* __restrict__ depth,
                                                         int32_t* __restrict__ err) {
  constexpr int LD = 2 * NB + 4;   // words of a staged row: 16 lanes' 16 bytes in 16 bank groups
  __shared__ uint64_t s_in[NB * 64];
  __shared__ int s_up[NB * 64];
  __shared__ __attribute__((aligned(16))) uint32_t s_out[4][64 * LD];
  const int s = blockIdx.x / parts, part = blockIdx.x - s * parts;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, W = (R + 31) / 32;
  const size_t base = (size_t)s * R;
  const int blocks = min((R + 63) / 64, part * 4 + 4);
  constexpr int N = (NB + 3) / 4;
  int p[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int b = i * 4 + w, r = b * 64 + lane;
    p[i] = b < blocks && r < R ? parent[base + r] : -2;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = checked_parent(p[i], (i * 4 + w) * 64 + lane, err);
  MaskRow m[N];
  wave_ancestors(p, w * 64, 256, lane, m);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int b = i * 4 + w, r = b * 64 + lane;
    if (b < blocks) {
      s_in[r] = m[i].in;
      s_up[r] = m[i].up;
    }
  }
  __syncthreads();
  const int first = part * 256 + w * 64, r = first + lane;
  const bool live = first < R;
  u32x4 word[NB / 2];
  int up = live ? r : -2, d = -1;
#pragma unroll
  for (int b = NB - 1; b >= 0; --b) {
    uint64_t m = 0;
    if (up >= b * 64) {   // (the chain's next row is in block b: those above are done)
      m = s_in[up];
      up = s_up[up];
      d += __popcll(m);
    }
    word[b / 2][b % 2 * 2] = (uint32_t)m;
    word[b / 2][b % 2 * 2 + 1] = (uint32_t)(m >> 32);
  }
  if (live) {
    if (r < R && depth) depth[base + r] = up == -1 ? d : -1;
#pragma unroll
    for (int i = 0; i < NB / 2; ++i)
      *(u32x4*)(s_out[w] + lane * LD + i * 4) = up == -1 ? word[i] : u32x4{0, 0, 0, 0};
  }
  __syncthreads();
  if (!live) return;
  uint32_t* to = (uint32_t*)mask + (base + first) * W;
  const int unit = wide ? 4 : 1, per_row = W / unit, n = min(64, R - first) * per_row;
  int row = lane / per_row, c = lane - row * per_row;
  const int drow = 64 / per_row, dc = 64 - drow * per_row;
  for (int i = lane; i < n; i += 64) {
    const uint32_t* from = s_out[w] + row * LD + c * unit;
    if (wide) *(u32x4*)(to + i * 4) = *(const u32x4*)from;
    else to[i] = *from;
    row += drow;
    c += dc;
    if (c >= per_row) {
      c -= per_row;
      ++row;
    }
  }
}

// ---------------------------------------------------------------------------
// kv_append_rope
//
// A pair (a, b) = (x_i, x_{i + h}), h = rot_dim / 2, turns by the angle
// pos * theta^(-i / h):  (a cos - b sin, b cos + a sin).  A workgroup takes the
// rows of one page of the window (up to 16) and a run of heads (queries, then
// keys, then values): the page's sines and cosines are made once for all of
// its heads.  Values go through LDS, so that the head-dim-major page of V is
// written in whole 16-byte pieces (8 or 4 slots of an element).
//
// What bounds it: prefills, the rows read and written (8 x 1088 rows of 16 + 2 x 4
// heads of 96, 80 MB: 17.4 us, 4.6 TB/s of the 5.1 that a copy reaches; half a us
// more without the loads ahead and with a head of V at a time); single
// tokens, latency (lengths, then page and row, then stores: 6.2 us for 64).
// ---------------------------------------------------------------------------
struct AppendParams {
  const void *q, *k, *v;
  long long q_seq, q_ld, k_seq, k_ld, v_seq, v_ld;
  void *k_pool, *v_pool, *q_out;
  const int32_t *table, *kv_len, *depth;
  int32_t* err;
  int S, R, Hq, Hkv, max_pages, pool_pages, half, n_pages, n_groups, per_group;
  // quarter turns a position: theta^(-i / half) * 2 / pi, in 64 bits, so that
  // far positions keep their angle (what is left after whole quarters is
  // taken in 32)
  double turns[64];
};

template <typename T, bool ALIGNED>
struct Piece {   // 16 bytes of a head's row
  static constexpr int N = 16 / sizeof(T);
  T e[N];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (ALIGNED) {
      *(u32x4*)e = *(const u32x4*)p;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = p[i];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (ALIGNED) {
      *(u32x4*)p = *(const u32x4*)e;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = e[i];
    }
  }
};

// T: float or __bf16.  ALIGNED: every row of q, k, v and q_out starts on 16
// bytes (pool rows always do).
template <typename T, int D, bool ALIGNED>
__global__ void __launch_bounds__(256) append_rope_kernel(AppendParams p) {
  constexpr int N = 16 / sizeof(T);
  constexpr int PAIRS = D / (2 * N);    // items of a row: two pieces each
  constexpr int VLD = D + 16 / sizeof(T);
  __shared__ float2 s_cs[16][65];
  constexpr int VH = 8 / (int)sizeof(T);   // heads of V in LDS at a time
  __shared__ __attribute__((aligned(16))) T s_v[VH * 16 * VLD];
  __shared__ int s_live[16];
  const int tid = threadIdx.x;
  const int g = blockIdx.x % p.n_groups, sp = blockIdx.x / p.n_groups;
  const int pi = sp % p.n_pages, s = sp / p.n_pages;
  const int L = p.kv_len[s];
  if (L < 0 || (long long)L + p.R > (long long)p.max_pages * DVS_PAGE_SIZE) {
    if (g == 0 && pi == 0 && tid == 0) set_err(p.err, DVS_ERR_MAX_PAGES);
    return;
  }
  const int pg = L / DVS_PAGE_SIZE + pi;             // logical page
  const int r0 = pg * DVS_PAGE_SIZE - L;             // row of its slot 0
  if (r0 >= p.R) return;
  const int page = p.table[(size_t)s * p.max_pages + pg];
  const bool in_pool = page >= 0 && page < p.pool_pages;
  if (!in_pool && g == 0 && tid == 0) set_err(p.err, DVS_ERR_BAD_PAGE);
  const int u0 = g * p.per_group, u1 = min(u0 + p.per_group, p.Hq + 2 * p.Hkv);
  const T* q = (const T*)p.q + s * p.q_seq;
  const T* k = (const T*)p.k + s * p.k_seq;
  const T* v = (const T*)p.v + s * p.v_seq;
  // queries and keys: the first pieces are on their way under the angles, the
  // next ones under a piece's products
  const int items = (min(u1, p.Hq + p.Hkv) - u0) * 16 * PAIRS;
  Piece<T, ALIGNED> na, nb;
  auto place = [&](int i, int& u, int& j, int& lo, int& hi, bool& turn) {
    const int c = i % PAIRS;
    j = i / PAIRS % 16;
    u = u0 + i / (16 * PAIRS);
    turn = c * N < p.half;
    lo = turn ? c * N : 2 * p.half + 2 * (c * N - p.half);
    hi = turn ? p.half + c * N : lo + N;
  };
  auto fetch = [&](int i) {
    int u, j, lo, hi;
    bool turn;
    if (i >= items) return;
    place(i, u, j, lo, hi, turn);
    const int r = r0 + j;
    if (r < 0 || r >= p.R) return;
    const T* src = u >= p.Hq ? k + r * p.k_ld + (u - p.Hq) * D : q + r * p.q_ld + (long long)u * D;
    na.load(src + lo);
    nb.load(src + hi);
  };
  fetch(tid);
  // live rows and their angles
  for (int i = tid; i < 16 * max(p.half, 1); i += 256) {
    const int j = i % 16, e = i / 16, r = r0 + j;
    int d = -1;
    if (r >= 0 && r < p.R) d = p.depth ? p.depth[(size_t)s * p.R + r] : r;
    if (e == 0) s_live[j] = d >= 0;
    if (d < 0 || p.half == 0) continue;
    const double t = (double)((long long)L + d) * p.turns[e];
    const double n = rint(t);
    float sn, cs;
    sincospif(0.5f * (float)(t - n), &sn, &cs);
    switch ((long long)n & 3) {
      case 0: s_cs[j][e] = float2{cs, sn}; break;
      case 1: s_cs[j][e] = float2{-sn, cs}; break;
      case 2: s_cs[j][e] = float2{-cs, -sn}; break;
      default: s_cs[j][e] = float2{sn, -cs}; break;
    }
  }
  __syncthreads();
  for (int i = tid; i < items; i += 256) {
    int u, j, lo, hi;
    bool turn;
    place(i, u, j, lo, hi, turn);
    const int r = r0 + j;
    const bool key = u >= p.Hq;
    Piece<T, ALIGNED> a = na, b = nb;
    fetch(i + 256);
    if (!s_live[j] || (key && !in_pool)) continue;
    if (turn) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float2 w = s_cs[j][lo + e];
        const float x = (float)a.e[e], y = (float)b.e[e];
        a.e[e] = (T)(x * w.x - y * w.y);
        b.e[e] = (T)(y * w.x + x * w.y);
      }
    }
    if (key) {
      T* dst = (T*)p.k_pool + (((size_t)page * p.Hkv + (u - p.Hq)) * 16 + j) * D;
      ((Piece<T, true>&)a).store(dst + lo);
      ((Piece<T, true>&)b).store(dst + hi);
    } else if (p.q_out) {
      T* dst = (T*)p.q_out + (((size_t)s * p.R + r) * p.Hq + u) * D;
      a.store(dst + lo);
      b.store(dst + hi);
    }
  }
  if (!in_pool) return;
  // values, VH heads at a time
  for (int ub = max(u0, p.Hq + p.Hkv); ub < u1; ub += VH) {
    const int nh = min(VH, u1 - ub), h0 = ub - p.Hq - p.Hkv;
    __syncthreads();
    for (int i = tid; i < nh * 16 * (D / N); i += 256) {
      const int c = i % (D / N), j = i / (D / N) % 16, h = i / (16 * (D / N));
      if (!s_live[j]) continue;
      Piece<T, ALIGNED> x;
      x.load(v + (r0 + j) * p.v_ld + (h0 + h) * D + c * N);
      ((Piece<T, true>&)x).store(s_v + (h * 16 + j) * VLD + c * N);
    }
    __syncthreads();
    T* dst = (T*)p.v_pool + ((size_t)page * p.Hkv + h0) * D * 16;   // (a page's heads lie side by side)
    for (int i = tid; i < nh * D * (16 / N); i += 256) {
      const int hd = i / (16 / N), j0 = i % (16 / N) * N, h = hd / D, d = hd - h * D;
      Piece<T, true> x;
      int live = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x.e[e] = s_v[(h * 16 + j0 + e) * VLD + d];
        live += s_live[j0 + e];
      }
      if (live == N) {
        x.store(dst + hd * 16 + j0);
      } else if (live) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (s_live[j0 + e]) dst[hd * 16 + j0 + e] = x.e[e];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// accept_commit_tree
//
// follow(p) = the lowest child of row p whose token is the verifier's top-1 at
// p; the accepted path is 0, follow(0), follow(follow(0)), ...  The committed
// tokens are the verifier's at the path's rows, which kv_commit's kernel
// commits with its pages; the path's cache slots then move from kv_len +
// path[i] to kv_len + i in every layer.  The commit may give pages of the
// window back before the move: the move goes by the page ids noted here, and
// nothing writes to a page that was given back in between.  A slot that cannot
// move, for a page outside the pool, is found here too, so that a commit that
// needs it changes nothing.  Small steps are accepted and committed by one launch
// (commit.hip); this kernel is for the others.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(256) tree_accept_kernel(TreeCommit t) {
  __shared__ int s_next[TREE_MAX_ROWS];
  __shared__ int s_path[TREE_MAX_ROWS];
  __shared__ int s_page[TREE_MAX_ROWS / DVS_PAGE_SIZE + 2];
  __shared__ int s_A, s_movable;
  const int s = blockIdx.x, tid = threadIdx.x, R = t.R;
  const size_t base = (size_t)s * R;
  const int32_t *parent = t.parent + base, *argmax = t.argmax + base;
  const int L = t.kv_len[s];
  const bool live = t.finished[s] == 0 && parent[0] == -1;
  for (int r = tid; r < R; r += 256) s_next[r] = R;
  for (int i = tid; i < t.n_window_pages; i += 256)
    t.pages[(size_t)s * t.n_window_pages + i] = s_page[i] = tree_window_page(t, s, L, i);
  __syncthreads();
  for (int r = tid; r < R; r += 256) {
    const int p = parent[r];
    if (p >= 0 && p < r && t.tokens[base + r] == argmax[p]) atomicMin(&s_next[p], r);
  }
  __syncthreads();
  if (tid == 0) {
    int A = -1;
    if (live)
      for (int r = 0; r < R; r = s_next[r]) s_path[++A] = r;
    s_A = A;
    s_movable = A + 1;
    t.accept[s] = max(A, 0);
    t.run_len[s] = A;
    t.old_len[s] = L;
  }
  __syncthreads();
  const int A = s_A, off = L & (DVS_PAGE_SIZE - 1);
  for (int i = tid; i < R; i += 256) {
    const int r = i <= A ? s_path[i] : -1;
    t.path[base + i] = r;
    t.run[base + i] = r >= 0 ? argmax[r] : 0;
    if (r > i && (s_page[(off + r) >> 4] < 0 || s_page[(off + i) >> 4] < 0)) atomicMin(&s_movable, i);
  }
  __syncthreads();
  if (tid == 0) t.movable[s] = s_movable;
}

constexpr int MOVE_LAYERS = 64;   // layers per launch (as kernel arguments)
struct MovePools {
  char* p[2 * MOVE_LAYERS];
};

// A wave a (sequence, layer, K or V, KV head).  path[i] >= i and rises, so a
// slot is read before a later step writes it: MOVE slots are read together, then
// written.  Their rows and pages are found 64 at a time, a lane each.  Latency: 8
// sequences, 16 layers, 4 heads of 96: 5.0 - 5.5 us, 0.6 more a slot at a time.
template <typename T>
__global__ void __launch_bounds__(256) tree_move_kernel(TreeCommit t, MovePools pools, int n_pools,
                                                        int Hkv, int D) {
  constexpr int MOVE = 8, WORDS = 128 * (int)sizeof(T) / 4 / 64;   // words a lane of a slot of K
  const long long task = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (task >= (long long)t.S * n_pools * Hkv) return;
  const int h = (int)(task % Hkv), pl = (int)(task / Hkv % n_pools), s = (int)(task / Hkv / n_pools);
  const int L = t.old_len[s], k = t.kv_len[s] - L;
  if (k <= 1) return;
  const int32_t* path = t.path + (size_t)s * t.R;
  const int32_t* pages = t.pages + (size_t)s * t.n_window_pages;
  const int off = L % DVS_PAGE_SIZE;
  char* pool = pools.p[pl];
  const size_t head = (size_t)16 * D * sizeof(T);
  for (int i0 = 1; i0 < k; i0 += 64) {
    const int i = min(i0 + lane, k - 1), r = path[i];
    const int pf = pages[(off + r) >> 4], pt = pages[(off + i) >> 4];
    const int slots = ((off + r) & 15) << 4 | ((off + i) & 15);
    uint64_t todo = __ballot(i0 + lane < k && r != i);   // (the commit saw to their pages)
    while (todo) {
      char *from[MOVE], *to[MOVE];
      int n = 0;
#pragma unroll
      for (int b = 0; b < MOVE; ++b) {
        const int at = todo ? __ffsll((unsigned long long)todo) - 1 : 0;
        if (todo) n = b + 1;
        todo &= todo - 1;
        const int ab = __builtin_amdgcn_readlane(slots, at);
        const size_t step = pl & 1 ? sizeof(T) : D * sizeof(T);
        from[b] = pool + ((size_t)__builtin_amdgcn_readlane(pf, at) * Hkv + h) * head + (ab >> 4) * step;
        to[b] = pool + ((size_t)__builtin_amdgcn_readlane(pt, at) * Hkv + h) * head + (ab & 15) * step;
      }
      if (pl & 1) {
        T x[MOVE][2];
#pragma unroll
        for (int b = 0; b < MOVE; ++b)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (b < n && e * 64 + lane < D) x[b][e] = *(const T*)(from[b] + (e * 64 + lane) * 16 * sizeof(T));
#pragma unroll
        for (int b = 0; b < MOVE; ++b)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (b < n && e * 64 + lane < D) *(T*)(to[b] + (e * 64 + lane) * 16 * sizeof(T)) = x[b][e];
      } else {
        const int words = D * (int)sizeof(T) / 4;
        uint32_t x[MOVE][WORDS];
#pragma unroll
        for (int b = 0; b < MOVE; ++b)
#pragma unroll
          for (int e = 0; e < WORDS; ++e)
            if (b < n && e * 64 + lane < words) x[b][e] = *(const uint32_t*)(from[b] + (e * 64 + lane) * 4);
#pragma unroll
        for (int b = 0; b < MOVE; ++b)
#pragma unroll
          for (int e = 0; e < WORDS; ++e)
            if (b < n && e * 64 + lane < words) *(uint32_t*)(to[b] + (e * 64 + lane) * 4) = x[b][e];
      }
    }
  }
}

static size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }

static int window_pages(int R) { return (int)((R + DVS_PAGE_SIZE - 2LL) / DVS_PAGE_SIZE) + 1; }

template <typename T, bool ALIGNED>
static void launch_append(const AppendParams& p, int D, unsigned grid, hipStream_t st) {
  if (D == 128) hipLaunchKernelGGL((append_rope_kernel<T, 128, ALIGNED>), dim3(grid), dim3(256), 0, st, p);
  else if (D == 96) hipLaunchKernelGGL((append_rope_kernel<T, 96, ALIGNED>), dim3(grid), dim3(256), 0, st, p);
  else hipLaunchKernelGGL((append_rope_kernel<T, 64, ALIGNED>), dim3(grid), dim3(256), 0, st, p);
}

}  // namespace dvs

using namespace dvs;

extern "C" int tree_masks(const int32_t* parent, int32_t S, int32_t R, int32_t* mask_out,
                          int32_t* depth_out, int32_t* err_word, void* stream) {
  clear_error();
  DVS_CHECK_ARG(parent && mask_out, "tree_masks: NULL parent or mask_out");
  DVS_CHECK_ARG(S >= 1 && R >= 1 && R <= TREE_MAX_ROWS, "tree_masks: need S >= 1, 1 <= R <= %d",
                TREE_MAX_ROWS);
  DVS_CHECK_ARG(R <= 32 || ((uintptr_t)mask_out & 7) == 0, "tree_masks: mask_out must start on 8 bytes");
  DVS_CHECK_SUPPORTED(S < (1 << 22), "tree_masks: more than 2^22 sequences");
  hipStream_t st = (hipStream_t)stream;
  if (R <= 64) {
    hipLaunchKernelGGL(tree_masks_small_kernel, dim3((S + 3) / 4), dim3(256), 0, st, parent, S, R,
                       mask_out, depth_out, err_word);
  } else {
    const int parts = (R + 255) / 256, W = (R + 31) / 32;
    const bool wide = W % 4 == 0 && ((uintptr_t)mask_out & 15) == 0;
    auto launch = [&](auto nb) {
      hipLaunchKernelGGL(tree_masks_kernel<decltype(nb)::value>, dim3((unsigned)(S * parts)), dim3(256), 0, st,
                         parent, R, parts, wide, mask_out, depth_out, err_word);
    };
    if (R <= 128) launch(IC<2>{});
    else if (R <= 256) launch(IC<4>{});
    else if (R <= 512) launch(IC<8>{});
    else launch(IC<16>{});
  }
  return launch_status("tree_masks");
}

extern "C" int kv_append_rope(const void* q, int64_t q_seq, int64_t q_ld, const void* k_new,
                              int64_t k_seq, int64_t k_ld, const void* v_new, int64_t v_seq,
                              int64_t v_ld, void* k_pool, void* v_pool, const int32_t* page_table,
                              const int32_t* kv_len, const int32_t* depth, int32_t S, int32_t R,
                              int32_t Hq, int32_t Hkv, int32_t D, int32_t rot_dim, float theta,
                              int32_t max_pages, int32_t num_pool_pages, int32_t dtype, void* q_out,
                              int32_t* err_word, void* stream) {
  clear_error();
  DVS_CHECK_ARG(k_new && v_new && k_pool && v_pool && page_table && kv_len,
                "kv_append_rope: NULL array argument");
  DVS_CHECK_ARG(!q == !q_out, "kv_append_rope: q and q_out go together");
  DVS_CHECK_ARG(S >= 1 && R >= 1, "kv_append_rope: need S >= 1 and R >= 1");
  DVS_CHECK_ARG(Hkv >= 1 && Hq >= (q ? 1 : 0), "kv_append_rope: need heads");
  DVS_CHECK_ARG(max_pages >= 1 && num_pool_pages >= 1, "kv_append_rope: empty page table/pool");
  DVS_CHECK_SUPPORTED(max_pages <= TREE_MAX_PAGES, "kv_append_rope: max_pages must be below 2^27 - 3");
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "kv_append_rope: dtype %d", dtype);
  DVS_CHECK_SUPPORTED(D == 64 || D == 96 || D == 128, "kv_append_rope: head_dim %d", D);
  DVS_CHECK_SUPPORTED(rot_dim >= 0 && rot_dim <= D && rot_dim % 16 == 0,
                      "kv_append_rope: rot_dim must be a multiple of 16 of at most head_dim");
  DVS_CHECK_ARG(theta > 0.f && isfinite(theta), "kv_append_rope: theta must be positive");
  const int64_t qrow = (int64_t)Hq * D, krow = (int64_t)Hkv * D;
  DVS_CHECK_ARG((!q || R == 1 || q_ld >= qrow) && (R == 1 || (k_ld >= krow && v_ld >= krow)),
                "kv_append_rope: rows overlap");
  DVS_CHECK_ARG(q != q_out || !q || ((R == 1 || q_ld == qrow) && (S == 1 || q_seq == R * qrow)),
                "kv_append_rope: q is rotated in place only where its rows are dense");
  const uintptr_t es = dtype == DVS_BF16 ? 2 : 4;
  DVS_CHECK_ARG((((uintptr_t)k_pool | (uintptr_t)v_pool) & 15) == 0,
                "kv_append_rope: the pools must start on 16 bytes");
  DVS_CHECK_ARG((((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)q_out) & (es - 1)) == 0,
                "kv_append_rope: rows must start on an element");
  AppendParams p{};
  p.q = q; p.k = k_new; p.v = v_new;
  p.q_seq = q_seq; p.q_ld = q_ld; p.k_seq = k_seq; p.k_ld = k_ld; p.v_seq = v_seq; p.v_ld = v_ld;
  p.k_pool = k_pool; p.v_pool = v_pool; p.q_out = q_out;
  p.table = page_table; p.kv_len = kv_len; p.depth = depth; p.err = err_word;
  p.S = S; p.R = R; p.Hq = q ? Hq : 0; p.Hkv = Hkv; p.max_pages = max_pages;
  p.pool_pages = num_pool_pages; p.half = rot_dim / 2;
  // (by products in 64-bit mantissas, which keep all of a double's bits: 64 pow()
  // take longer than the launch)
  if (p.half) {
    const long double ratio = powl((long double)theta, -1.0L / p.half);
    long double turn = 0.636619772367581343075535L;
    for (int i = 0; i < p.half; ++i, turn *= ratio) p.turns[i] = (double)turn;
  }
  p.n_pages = window_pages(R);
  // heads of a page over several workgroups where the pages alone do not fill
  // the chip a few times over; fewer where a page has few rows to write (64 single
  // tokens, four / eight workgroups a CU 6.2 / 7.2 us; prefills 18.9 / 17.4)
  const int heads = p.Hq + 2 * Hkv;
  const long long pages = (long long)S * p.n_pages;
  const int groups = (int)std::min<long long>(heads, std::max<long long>(1, (R < DVS_PAGE_SIZE ? 4LL : 8LL) * device_cus() / pages));
  p.per_group = (heads + groups - 1) / groups;
  p.n_groups = (heads + p.per_group - 1) / p.per_group;
  DVS_CHECK_SUPPORTED(pages * p.n_groups < (1LL << 24), "kv_append_rope: grid too large");
  const unsigned grid = (unsigned)(pages * p.n_groups);
  auto on16 = [&](const void* b, int64_t seq, int64_t ld) {
    return !b || ((((uintptr_t)b | (uintptr_t)(S > 1 ? seq : 0) * es | (uintptr_t)(R > 1 ? ld : 0) * es)) & 15) == 0;
  };
  const bool aligned = on16(q, q_seq, q_ld) && on16(k_new, k_seq, k_ld) && on16(v_new, v_seq, v_ld) &&
                       on16(q_out, 0, 0);
  hipStream_t st = (hipStream_t)stream;
  if (dtype == DVS_BF16) {
    if (aligned) launch_append<__bf16, true>(p, D, grid, st);
    else launch_append<__bf16, false>(p, D, grid, st);
  } else {
    if (aligned) launch_append<float, true>(p, D, grid, st);
    else launch_append<float, false>(p, D, grid, st);
  }
  return launch_status("kv_append_rope");
}

extern "C" size_t dvs_accept_tree_workspace_bytes(int32_t S, int32_t R) {
  if (S < 1 || S > 1024 || R < 1 || R > TREE_MAX_ROWS) return 0;
  return al256((size_t)S * 4 * (4 + window_pages(R) + 2 * (size_t)R));
}

extern "C" int accept_commit_tree(const dvs_state* st, const dvs_layer* layers, int32_t n_layers,
                                  int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t R,
                                  const int32_t* parent, const int32_t* tokens,
                                  const int32_t* argmax, int32_t* accept_out, int32_t* path_out,
                                  void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  DVS_CHECK_ARG(st && st->kv_len && st->page_table && st->num_pages && st->free_stack &&
                    st->free_top && st->boundary && st->out_tokens && st->out_count && st->finished,
                "accept_commit_tree: NULL state or state array");
  DVS_CHECK_ARG(parent && tokens && argmax, "accept_commit_tree: NULL parent, tokens or argmax");
  DVS_CHECK_ARG(R >= 1 && R <= TREE_MAX_ROWS, "accept_commit_tree: need 1 <= R <= %d", TREE_MAX_ROWS);
  DVS_CHECK_ARG(st->S >= 1 && st->S <= 1024, "accept_commit_tree: need 1 <= S <= 1024");
  DVS_CHECK_ARG(st->max_pages >= 1 && st->num_pool_pages >= 1 && st->max_new >= 1,
                "accept_commit_tree: need max_pages, num_pool_pages, max_new >= 1");
  DVS_CHECK_SUPPORTED(st->max_pages <= TREE_MAX_PAGES, "accept_commit_tree: max_pages must be below 2^27 - 3");
  DVS_CHECK_ARG(layers && n_layers >= 1 && n_kv_heads >= 1, "accept_commit_tree: need layers and heads");
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "accept_commit_tree: dtype %d", dtype);
  DVS_CHECK_SUPPORTED(head_dim == 64 || head_dim == 96 || head_dim == 128,
                      "accept_commit_tree: head_dim %d", head_dim);
  for (int l = 0; l < n_layers; ++l)
    DVS_CHECK_ARG(layers[l].k_pool && layers[l].v_pool &&
                      (((uintptr_t)layers[l].k_pool | (uintptr_t)layers[l].v_pool) & 15) == 0,
                  "accept_commit_tree: layer %d needs pools that start on 16 bytes", l);
  for (int l = 0; l < n_layers; ++l)
    for (int e = 0; e < l; ++e)
      DVS_CHECK_ARG((layers[e].k_pool == layers[l].k_pool) == (layers[e].v_pool == layers[l].v_pool),
                    "accept_commit_tree: layers %d and %d share one of their two pools", e, l);
  // (the move's grid: 2^32 threads are too many, and the state would be committed by then)
  DVS_CHECK_SUPPORTED((long long)st->S * 2 * std::min(n_layers, MOVE_LAYERS) * n_kv_heads < (1LL << 26) - 3,
                      "accept_commit_tree: sequences, layers and heads make too large a grid");
  const size_t need = dvs_accept_tree_workspace_bytes(st->S, R);
  if (!workspace || ws_bytes < need) {
    set_error("accept_commit_tree: workspace needs %zu bytes, got %zu", need, ws_bytes);
    return DVS_EWORKSPACE;
  }
  const int S = st->S;
  TreeCommit t{};
  t.S = S; t.R = R; t.max_pages = st->max_pages; t.pool_pages = st->num_pool_pages;
  t.n_window_pages = window_pages(R);
  t.parent = parent; t.tokens = tokens; t.argmax = argmax;
  t.kv_len = st->kv_len; t.table = st->page_table; t.finished = st->finished;
  int32_t* w = (int32_t*)workspace;
  t.run_len = w; t.old_len = w + S;
  t.accept = accept_out ? accept_out : w + 2 * S;
  t.movable = w + 3 * S;
  t.pages = w + 4 * S;
  t.run = t.pages + (size_t)S * t.n_window_pages;
  t.path = path_out ? path_out : t.run + (size_t)S * R;
  hipStream_t hs = (hipStream_t)stream;
  int rc;
  if (!tree_accept_in_commit(t)) {
    hipLaunchKernelGGL(tree_accept_kernel, dim3(S), dim3(256), 0, hs, t);
    if ((rc = launch_status("accept_commit_tree(accept)"))) return rc;
  }
  if ((rc = commit_tree_run(st, t, stream))) return rc;
  for (int l = 0; l < n_layers;) {
    MovePools pools{};
    int nl = 0;
    for (; l < n_layers && nl < MOVE_LAYERS; ++l) {
      // a cache that several layers share moves once: a second wave on the same
      // slots would read what the first has moved
      bool moved = false;
      for (int e = 0; e < l; ++e) moved |= layers[e].k_pool == layers[l].k_pool;
      if (moved) continue;
      pools.p[2 * nl] = (char*)layers[l].k_pool;
      pools.p[2 * nl++ + 1] = (char*)layers[l].v_pool;
    }
    if (!nl) break;
    const long long tasks = (long long)S * 2 * nl * n_kv_heads;
    const dim3 gr((unsigned)((tasks + 3) / 4));
    if (dtype == DVS_BF16)
      hipLaunchKernelGGL(tree_move_kernel<uint16_t>, gr, dim3(256), 0, hs, t, pools, 2 * nl, n_kv_heads, head_dim);
    else
      hipLaunchKernelGGL(tree_move_kernel<float>, gr, dim3(256), 0, hs, t, pools, 2 * nl, n_kv_heads, head_dim);
    if ((rc = launch_status("accept_commit_tree(move)"))) return rc;
  }
  return DVS_OK;
}
