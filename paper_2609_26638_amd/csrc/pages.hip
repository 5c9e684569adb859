// kv_fork, kv_release, kv_compact: the cache pages of sequences that are
// duplicated, dropped and moved together.
//
// Ownership.  A page that several sequences hold has page_refs[page] holders
// beyond the first (0 for a page of one holder and for a free page).  Only
// full committed pages (below floor(kv_len / 16)) are ever shared: a step
// appends at positions >= kv_len, and a commit neither pops a shared page
// (it is not on the stack) nor pushes one (it keeps every page below kv_len),
// so the attention and the commits need not know of the counts.
//
// kv_fork and kv_release give destination slots new page rows in one way:
//   plan    slot checks; per pair the shared, fresh and copied pages, their
//           exclusive scans (one workgroup, one thread per pair);
//   drop    every page of a destination loses a holder; one left without any
//           sets its bit in a bitmap (atomics: counts and bits do not depend
//           on their order);
//   settle  the bitmap's pages go on the stack, the highest id first (so the
//           lowest is popped first), then the fresh pages are popped, pairs in
//           order.  Feasibility is decided before anything is written;
//   apply   page rows, counts of shared pages, sequence fields; on an error
//           the dropped holders come back and nothing else has changed;
//   copy    the partly filled (or, unshared, every committed) page, all layers.
// A destination is never a source, so a page that is shared on keeps its
// source as a holder all the while and cannot be freed by the drop.
//
// kv_compact marks the free and the held pages in two bitmaps, checks that
// they make up the pool, and pairs the k-th held id past the number of held
// pages with the k-th free id below it; copies, tables, counts and the stack
// follow.  Sources and targets are disjoint, so the copies need no order.
//
// The copies are bound by HBM (fork of one sequence of 2000 rows to three slots
// of their own, 32 pools: 49 MB read and 147 written in 40 us; compaction of
// 209 MB read and written in 86 us); the rest by the latency of a few dependent
// loads.  Forks and compactions of up to SMALL_ENTRIES table entries, and
// releases of up to twice as many, over pools of up to SMALL_POOL pages do
// everything up to the settling (a release all of it) in one workgroup with its
// bitmaps in LDS; page rows and copies share a launch.  A release of one
// sequence: 9 us.
#include "dvs_common.h"

namespace dvs {

constexpr int PLAN_THREADS = 1024;
constexpr int COPY_THREADS = 256;
constexpr int SMALL_ENTRIES = 4096, SMALL_POOL = 32768;
constexpr int COPY_LAYERS = 64;    // pools per launch (as kernel arguments)
constexpr int MAX_POOL = 1 << 29;  // sums of two page counts, and ids by whole words, fit 31 bits

struct PageState {   // of dvs_state, as the kernels take it
  int S, max_pages, pool, draft_width, max_new;
  int32_t *kv_len, *table, *num_pages, *stack, *top, *boundary, *draft, *out_tokens, *out_count,
      *finished, *err, *refs;
};

struct PageWork {    // workspace
  int32_t* head;     // H_* words
  int32_t *full, *need, *pop_at, *copy_at;   // per pair
  uint32_t *bits, *free_bits;
  int32_t *from, *to;                        // page copies
  int32_t* pages;                            // fresh pages in order / new ids of moved pages
  int words;
};

enum { H_ERR, H_DROP_ERR, H_POPS, H_COPIES, H_USED, H_WORDS };

__device__ __forceinline__ int pages_for(long long rows) {
  return (int)((rows + DVS_PAGE_SIZE - 1) / DVS_PAGE_SIZE);
}

// Exclusive scan over the workgroup; total to every thread.
__device__ __forceinline__ int scan_excl(int v, int* sh, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  if (lane == 63) sh[w] = incl;
  __syncthreads();
  int base = 0, all = 0;
  for (int i = 0; i < (int)blockDim.x / 64; ++i) {
    if (i < w) base += sh[i];
    all += sh[i];
  }
  __syncthreads();
  total = all;
  return base + incl - v;
}

// Calls use(id, k) for the k-th set bit of `words` words, from the lowest id or,
// `down`, from the highest; a workgroup of PLAN_THREADS takes as many words at
// a time, and neighbouring threads neighbouring ids, so that their stores join.
template <typename G, typename U>
__device__ __forceinline__ void each_bit(int words, bool down, G word, U use) {
  __shared__ uint32_t part[PLAN_THREADS];
  __shared__ int before[PLAN_THREADS];
  __shared__ int sh[PLAN_THREADS / 64];
  const int t = threadIdx.x;
  for (int w0 = 0, k0 = 0, found; w0 < words; w0 += PLAN_THREADS, k0 += found) {
    const int w = w0 + t;
    part[t] = w < words ? word(down ? words - 1 - w : w) : 0;
    if (down) part[t] = __brev(part[t]);
    before[t] = k0 + scan_excl(__popc(part[t]), sh, found);
    __syncthreads();
    if (found)
      for (int e = t; e < min(PLAN_THREADS, words - w0) * 32; e += PLAN_THREADS) {
        const uint32_t b = part[e >> 5], bit = 1u << (e & 31);
        if (b & bit)
          use(down ? (words - w0) * 32 - 1 - e : w0 * 32 + e,
              before[e >> 5] + __popc(b & (bit - 1)));
      }
    __syncthreads();
  }
}

struct Assign {      // one call's pairs
  const int32_t *src, *dst;   // src NULL: the slots become empty
  int n, window, share;
};

// Thread t's pair: its slots (src -1: none), committed pages of the source,
// pages the destination had, shared and needed pages, places of its fresh and
// its copied pages in their lists.
struct Pair {
  int src, dst, have, old, full, need, pop_at, copy_at;
};

struct Totals {
  int err, top, pops, copies;
};

// The plan, by a workgroup of PLAN_THREADS; the totals go to every thread.
__device__ __forceinline__ Pair assign_plan(const PageState& st, const PageWork& wk,
                                            const Assign& as, Totals& all) {
  __shared__ int role[PLAN_THREADS];
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  const int top = *st.top;
  Pair pr{-1, -1, 0, 0, 0, 0, 0, 0};
  role[t] = 0;
  if (t == 0) s_err = 0;
  __syncthreads();
  bool ok = false;
  if (t < as.n) {
    pr.dst = as.dst[t];
    if (as.src) pr.src = as.src[t];
    ok = pr.dst >= 0 && pr.dst < st.S && (!as.src || (pr.src >= 0 && pr.src < st.S));
    if (ok) {
      ok = !(atomicOr(&role[pr.dst], 1) & 1);
      if (as.src) atomicOr(&role[pr.src], 2);
    }
    if (!ok) atomicOr(&s_err, DVS_ERR_BAD_SLOT);
  }
  __syncthreads();
  if (role[t] == 3) atomicOr(&s_err, DVS_ERR_BAD_SLOT);
  if (ok) {
    const int L = as.src ? st.kv_len[pr.src] : 0;
    const int held = as.src ? st.num_pages[pr.src] : 0;
    const int old = st.num_pages[pr.dst];
    const int need = L < 0 ? 0 : pages_for((long long)L + as.window);
    if (L < 0 || need > st.max_pages || old < 0 || old > st.max_pages) {
      atomicOr(&s_err, DVS_ERR_MAX_PAGES);
    } else {
      pr.old = old;
      pr.need = need;
      pr.have = pages_for(L);
      pr.full = as.share ? L / DVS_PAGE_SIZE : 0;
      if (as.src && (held < pr.have || held > st.max_pages)) atomicOr(&s_err, DVS_ERR_BAD_PAGE);
    }
  }
  pr.pop_at = scan_excl(pr.need - pr.full, sh, all.pops);
  pr.copy_at = scan_excl(pr.have - pr.full, sh, all.copies);
  all.top = top;
  all.err = s_err | (top < 0 || top > st.pool ? DVS_ERR_POOL_EXHAUSTED : 0);
  if (t < as.n) {
    wk.full[t] = pr.full;
    wk.need[t] = pr.need;
    wk.pop_at[t] = pr.pop_at;
    wk.copy_at[t] = pr.copy_at;
  }
  if (t == 0) {
    wk.head[H_ERR] = all.err;
    wk.head[H_DROP_ERR] = 0;
    wk.head[H_POPS] = all.pops;
    wk.head[H_COPIES] = all.copies;
  }
  return pr;
}

// Page p of a destination loses a holder; true if its id or its count is bad.
__device__ __forceinline__ bool drop_page(const PageState& st, uint32_t* bits, int p) {
  if (p < 0 || p >= st.pool) return true;
  const int holders = st.refs ? atomicSub(&st.refs[p], 1) : 0;
  const uint32_t bit = 1u << (p & 31);
  return holders < 0 || (holders == 0 && (atomicOr(&bits[p >> 5], bit) & bit));
}

// The stack, and the fresh pages in wk.pages, by a workgroup of PLAN_THREADS:
// the freed pages come on top of the stack's `top`, `pops` ids leave it.  err:
// the errors so far; false if there are any.
__device__ __forceinline__ bool assign_settle(const PageState& st, const PageWork& wk,
                                              const uint32_t* bits, int err, int top, int pops) {
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  if (t == 0) s_err = err;
  int mine = 0, freed = 0;
  if (!err)
    for (int w = t; w < wk.words; w += PLAN_THREADS) mine += __popc(bits[w]);
  scan_excl(mine, sh, freed);
  const int full = top + freed, left = full - pops;    // pop k takes entry full - 1 - k
  if (!err) {
    if (t == 0 && (left < 0 || full > st.pool)) atomicOr(&s_err, DVS_ERR_POOL_EXHAUSTED);
    for (int i = max(0, left) + t; i < top; i += PLAN_THREADS) {
      const int p = st.stack[i];
      if (p < 0 || p >= st.pool) atomicOr(&s_err, DVS_ERR_BAD_PAGE);
      if (full <= st.pool) wk.pages[full - 1 - i] = p;
    }
  }
  __syncthreads();
  if (s_err) {
    if (t == 0) {
      wk.head[H_DROP_ERR] = s_err;       // H_ERR still says whether pages were dropped
      set_err(st.err, s_err);
    }
    return false;
  }
  each_bit(wk.words, true, [&](int w) { return bits[w]; },
           [&](int p, int k) {
             const int at = top + k;
             st.stack[at] = at < left ? p : -1;
             if (at >= left) wk.pages[full - 1 - at] = p;
             if (st.refs) st.refs[p] = 0;
           });
  for (int i = left + t; i < top; i += PLAN_THREADS) st.stack[i] = -1;
  if (t == 0) *st.top = left;
  __threadfence_block();
  __syncthreads();
  return true;
}

// Runs load(i, j) and then use(i, j, loaded) for j < width of pairs i < n, a
// few a thread at a time, so that their loads are in flight together.  There
// are at most 2^20 of them, for which e / width is exact by the reciprocal:
// (e + 1/2) / width is 1 / (2 width) away from an integer, its error below
// e / width * 2^-22.
template <typename L, typename U>
__device__ __forceinline__ void each_entry(int n, int width, L load, U use) {
  constexpr int K = 4;
  const int all = n * width;
  const float inv = 1.f / width;
  for (int e0 = threadIdx.x; e0 < all; e0 += K * PLAN_THREADS) {
    int2 v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = min(e0 + k * PLAN_THREADS, all - 1), i = (int)((e + 0.5f) * inv);
      v[k] = load(i, e - i * width);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int e = e0 + k * PLAN_THREADS, i = (int)((e + 0.5f) * inv);
      if (e < all) use(i, e - i * width, v[k]);
    }
  }
}

// Entry j of a pair's new page row; with an error the dropped holder comes back.
__device__ __forceinline__ void apply_entry(const PageState& st, const PageWork& wk, bool failed,
                                            const Pair& pr, int j) {
  int32_t* row = st.table + (size_t)pr.dst * st.max_pages;
  if (failed) {
    if (st.refs && j < pr.old && row[j] >= 0 && row[j] < st.pool) atomicAdd(&st.refs[row[j]], 1);
    return;
  }
  int p = -1;
  if (j < pr.full) {
    p = st.table[(size_t)pr.src * st.max_pages + j];
    atomicAdd(&st.refs[p], 1);
  } else if (j < pr.need) {
    p = wk.pages[pr.pop_at + j - pr.full];
  }
  row[j] = p;
}

// A pair's sequence fields, by threads t, t + step, ...
__device__ __forceinline__ void apply_fields(const PageState& st, const Pair& pr, int t, int step) {
  const int a = pr.src, b = pr.dst;
  if (a >= 0) {
    for (int k = t; k < st.draft_width; k += step)
      st.draft[(size_t)b * st.draft_width + k] = st.draft[(size_t)a * st.draft_width + k];
    for (int k = t; k < st.max_new; k += step)
      st.out_tokens[(size_t)b * st.max_new + k] = st.out_tokens[(size_t)a * st.max_new + k];
  }
  if (t == 0) {
    st.num_pages[b] = pr.need;
    st.kv_len[b] = a >= 0 ? st.kv_len[a] : 0;
    st.boundary[b] = a >= 0 ? st.boundary[a] : 0;
    st.out_count[b] = a >= 0 ? st.out_count[a] : 0;
    st.finished[b] = a >= 0 ? st.finished[a] : 1;
  }
}

// Everything up to the settling in one workgroup, a release whole.  The
// holders that a page loses are counted in LDS, in 16 bits (a call has at most
// 2 * SMALL_ENTRIES of them): 16 us for 56 forks of 8 prefixes, where seven
// destinations give up the same pages, 19.5 with an atomic on page_refs for
// each.
__global__ void __launch_bounds__(PLAN_THREADS) assign_small_kernel(PageState st, PageWork wk,
                                                                    Assign as) {
  __shared__ uint32_t bits[SMALL_POOL / 32];
  __shared__ uint32_t lost[SMALL_POOL / 2];
  __shared__ Pair pairs[PLAN_THREADS];
  __shared__ int s_bad, s_pages, s_copies;
  const int t = threadIdx.x;
  for (int i = t; i < wk.words * 16; i += PLAN_THREADS) lost[i] = 0;
  for (int i = t; i < wk.words; i += PLAN_THREADS) bits[i] = 0;
  if (t == 0) s_bad = s_pages = s_copies = 0;
  Totals all;
  pairs[t] = assign_plan(st, wk, as, all);
  if (t < as.n) {
    atomicMax(&s_pages, max(pairs[t].old, pairs[t].have));
    atomicMax(&s_copies, pairs[t].have - pairs[t].full);
  }
  __syncthreads();
  const bool go = all.err == 0;
  if (go) {
    bool bad = false;
    each_entry(
        as.n, s_pages,
        [&](int i, int j) {
          const int a = as.src ? pairs[i].src : pairs[i].dst;
          return make_int2(st.table[(size_t)pairs[i].dst * st.max_pages + j],
                           st.table[(size_t)a * st.max_pages + j]);
        },
        [&](int i, int j, int2 v) {
          const bool in = v.x >= 0 && v.x < st.pool;
          if (j < pairs[i].old) {
            if (in) atomicAdd(&lost[v.x >> 1], 1u << (v.x & 1) * 16);
            bad |= !in;
          }
          if (j < pairs[i].have) bad |= v.y < 0 || v.y >= st.pool;
        });
    __syncthreads();
    each_entry(
        st.pool, 1, [&](int p, int) { return make_int2(st.refs ? st.refs[p] : 0, 0); },
        [&](int p, int, int2 v) {
          const int gone = lost[p >> 1] >> (p & 1) * 16 & 0xffff, left = v.x - gone;
          if (!gone) return;
          bad |= left < -1;
          if (left == -1) atomicOr(&bits[p >> 5], 1u << (p & 31));
          if (st.refs) st.refs[p] = left;
        });
    if (bad) s_bad = DVS_ERR_BAD_PAGE;
  }
  __syncthreads();
  const bool fine = assign_settle(st, wk, bits, all.err | s_bad, all.top, all.pops);
  if (as.src) {
    if (fine)
      each_entry(
          as.n, s_copies,
          [&](int i, int j) {
            const int from = min(pairs[i].full + j, st.max_pages - 1);
            return make_int2(st.table[(size_t)pairs[i].src * st.max_pages + from],
                             wk.pages[min(pairs[i].pop_at + j, st.pool - 1)]);
          },
          [&](int i, int j, int2 v) {
            if (j < pairs[i].have - pairs[i].full) {
              wk.from[pairs[i].copy_at + j] = v.x;
              wk.to[pairs[i].copy_at + j] = v.y;
            }
          });
  } else if (go) {
    for (int e = t, i = 0; e < as.n * st.max_pages; e += PLAN_THREADS) {
      i = e / st.max_pages;
      apply_entry(st, wk, !fine, pairs[i], e - i * st.max_pages);
    }
    if (fine && t < as.n) apply_fields(st, pairs[t], 0, 1);
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) assign_plan_kernel(PageState st, PageWork wk,
                                                                   Assign as) {
  for (int i = threadIdx.x; i < wk.words; i += PLAN_THREADS) wk.bits[i] = 0;
  Totals all;
  assign_plan(st, wk, as, all);
}

__global__ void __launch_bounds__(256) assign_drop_kernel(PageState st, PageWork wk, Assign as) {
  if (wk.head[H_ERR]) return;
  const int i = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x, b = as.dst[i];
  bool bad = false;
  if (j < st.num_pages[b]) bad = drop_page(st, wk.bits, st.table[(size_t)b * st.max_pages + j]);
  if (as.src && j < pages_for(st.kv_len[as.src[i]])) {
    const int p = st.table[(size_t)as.src[i] * st.max_pages + j];
    bad |= p < 0 || p >= st.pool;
  }
  if (bad) atomicOr(&wk.head[H_DROP_ERR], DVS_ERR_BAD_PAGE);
}

// Pair i as the plan left it.
__device__ __forceinline__ Pair planned(const PageState& st, const PageWork& wk, const Assign& as,
                                        int i) {
  const int a = as.src ? as.src[i] : -1, b = as.dst[i];
  return {a, b, a >= 0 ? pages_for(st.kv_len[a]) : 0, st.num_pages[b], wk.full[i], wk.need[i],
          wk.pop_at[i], wk.copy_at[i]};
}

__global__ void __launch_bounds__(PLAN_THREADS) assign_settle_kernel(PageState st, PageWork wk,
                                                                     Assign as) {
  const int err = wk.head[H_ERR] | wk.head[H_DROP_ERR];
  if (!assign_settle(st, wk, wk.bits, err, *st.top, wk.head[H_POPS]) || !as.src) return;
  auto list = [&](const Pair& pr, int j) {
    wk.from[pr.copy_at + j] = st.table[(size_t)pr.src * st.max_pages + pr.full + j];
    wk.to[pr.copy_at + j] = wk.pages[pr.pop_at + j];
  };
  const int t = threadIdx.x;
  if (as.share) {                        // at most a page each
    if (t >= as.n) return;
    const Pair pr = planned(st, wk, as, t);
    if (pr.have > pr.full) list(pr, 0);
  } else {
    for (int i = t >> 6; i < as.n; i += PLAN_THREADS / 64) {
      const Pair pr = planned(st, wk, as, i);
      for (int j = t & 63; j < pr.have; j += 64) list(pr, j);
    }
  }
}

// ---------------------------------------------------------------------------
// page copies
// ---------------------------------------------------------------------------

struct Pools {
  char* p[2 * COPY_LAYERS];              // K and V pool of each layer
};

// Copies page from[c] to page to[c] in every pool, c < head[H_COPIES], by
// workgroups `first`, first + step, ...: a page of a pool at a time.
__device__ __forceinline__ void copy_pages(const PageWork& wk, const Pools& pools, int n_pools,
                                           int page_bytes, int first, int step) {
  const long long tasks = (long long)wk.head[H_COPIES] * n_pools;
  const int vecs = page_bytes / 16;
  for (long long t = first; t < tasks; t += step) {
    const int c = (int)(t / n_pools), k = (int)(t - (long long)c * n_pools);
    const u32x4* from = (const u32x4*)(pools.p[k] + (size_t)wk.from[c] * page_bytes);
    u32x4* to = (u32x4*)(pools.p[k] + (size_t)wk.to[c] * page_bytes);
    for (int v0 = threadIdx.x; v0 < vecs; v0 += 4 * COPY_THREADS) {
      u32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = from[min(v0 + i * COPY_THREADS, vecs - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (v0 + i * COPY_THREADS < vecs)
          __builtin_nontemporal_store(x[i], &to[v0 + i * COPY_THREADS]);
    }
  }
}

// The first row_blocks workgroups write the pairs' page rows and fields, the
// others copy pages: sources are no destinations, so neither waits.
__global__ void __launch_bounds__(COPY_THREADS) assign_apply_kernel(PageState st, PageWork wk,
                                                                    Assign as, int per_row,
                                                                    int row_blocks, Pools pools,
                                                                    int n_pools, int page_bytes) {
  if (wk.head[H_ERR]) return;
  const bool failed = wk.head[H_DROP_ERR] != 0;
  if ((int)blockIdx.x >= row_blocks) {
    if (!failed)
      copy_pages(wk, pools, n_pools, page_bytes, blockIdx.x - row_blocks, gridDim.x - row_blocks);
    return;
  }
  const int i = blockIdx.x / per_row, x = blockIdx.x - i * per_row;
  const int j = x * COPY_THREADS + threadIdx.x;
  const Pair pr = planned(st, wk, as, i);   // (its `old` counts after an error only)
  if (j < st.max_pages) apply_entry(st, wk, failed, pr, j);
  if (x == 0 && !failed) apply_fields(st, pr, threadIdx.x, COPY_THREADS);
}

// Copies alone (the pools of further layers).
__global__ void __launch_bounds__(COPY_THREADS) copy_pages_kernel(PageWork wk, Pools pools,
                                                                  int n_pools, int page_bytes) {
  if (wk.head[H_ERR] | wk.head[H_DROP_ERR]) return;
  copy_pages(wk, pools, n_pools, page_bytes, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------

__global__ void __launch_bounds__(256) compact_clear_kernel(PageWork wk) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < wk.words) wk.bits[i] = wk.free_bits[i] = 0;
  if (i < H_WORDS) wk.head[i] = 0;
}

// Marks page p; true if the id is bad or, where it may be there once only,
// marked already.
__device__ __forceinline__ bool mark_page(const PageState& st, uint32_t* bits, int p, bool once) {
  if (p < 0 || p >= st.pool) return true;
  const uint32_t bit = 1u << (p & 31);
  const bool again = atomicOr(&bits[p >> 5], bit) & bit;
  return again && once;
}

// Moves, counts and stack from the two bitmaps, by a workgroup of PLAN_THREADS.
__device__ __forceinline__ void compact_plan(const PageState& st, const PageWork& wk,
                                             const uint32_t* bits, const uint32_t* free_bits,
                                             int err, int32_t* moved_out) {
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  if (t == 0) s_err = err;
  __syncthreads();
  int held = 0, used = 0;
  for (int w = t; w < wk.words; w += PLAN_THREADS) {
    const uint32_t all = (w + 1) * 32 <= st.pool ? ~0u : (1u << (st.pool & 31)) - 1;
    if ((bits[w] ^ free_bits[w]) != all || (bits[w] & free_bits[w]))
      atomicOr(&s_err, DVS_ERR_BAD_PAGE);
    held += __popc(bits[w]);
  }
  scan_excl(held, sh, used);
  if (s_err) {
    if (t == 0) {
      wk.head[H_ERR] = s_err;
      set_err(st.err, s_err);
      if (moved_out) *moved_out = 0;
    }
    return;
  }
  // bits of word w below the id `used`
  auto low = [&](int w) { return w * 32 >= used ? 0u : used - w * 32 >= 32 ? ~0u : (1u << (used - w * 32)) - 1; };
  int holes = 0, moved = 0;
  for (int w = t; w < wk.words; w += PLAN_THREADS) holes += __popc(free_bits[w] & low(w));
  scan_excl(holes, sh, moved);
  each_bit(wk.words, false, [&](int w) { return free_bits[w] & low(w); },
           [&](int p, int k) { wk.to[k] = p; });
  each_bit(wk.words, false, [&](int w) { return bits[w] & ~low(w); },
           [&](int p, int k) { wk.from[k] = p; });
  __threadfence_block();
  __syncthreads();
  for (int k = t; k < moved; k += PLAN_THREADS) {
    const int a = wk.from[k], b = wk.to[k];
    wk.pages[a] = b;
    if (st.refs) { st.refs[b] = st.refs[a]; st.refs[a] = 0; }
  }
  for (int i = t; i < st.pool; i += PLAN_THREADS)
    st.stack[i] = i < st.pool - used ? st.pool - 1 - i : -1;
  if (t == 0) {
    wk.head[H_ERR] = wk.head[H_DROP_ERR] = 0;
    wk.head[H_USED] = used;
    wk.head[H_COPIES] = moved;
    if (moved_out) *moved_out = moved;
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_small_kernel(PageState st, PageWork wk,
                                                                     int32_t* moved_out) {
  __shared__ uint32_t bits[SMALL_POOL / 32], free_bits[SMALL_POOL / 32];
  __shared__ int counts[PLAN_THREADS];
  __shared__ int s_err, s_pages;
  const int t = threadIdx.x;
  const int top = *st.top;
  for (int i = t; i < wk.words; i += PLAN_THREADS) bits[i] = free_bits[i] = 0;
  if (t == 0) {
    s_err = top < 0 || top > st.pool ? DVS_ERR_MAX_PAGES : 0;
    s_pages = 0;
  }
  __syncthreads();
  if (t < st.S) {
    const int c = counts[t] = st.num_pages[t];
    if (c < 0 || c > st.max_pages) atomicOr(&s_err, DVS_ERR_MAX_PAGES);
    else atomicMax(&s_pages, c);
  }
  __syncthreads();
  if (!s_err) {
    bool bad = false;
    each_entry(
        1, top, [&](int, int j) { return make_int2(st.stack[j], 0); },
        [&](int, int, int2 v) { bad |= mark_page(st, free_bits, v.x, true); });
    each_entry(
        st.S, s_pages,
        [&](int i, int j) { return make_int2(st.table[(size_t)i * st.max_pages + j], 0); },
        [&](int i, int j, int2 v) {
          if (j < counts[i]) bad |= mark_page(st, bits, v.x, !st.refs);
        });
    if (bad) atomicOr(&s_err, DVS_ERR_BAD_PAGE);
  }
  __syncthreads();
  compact_plan(st, wk, bits, free_bits, s_err, moved_out);
}

// Workgroups of per_row a sequence, then those of the free stack.
__global__ void __launch_bounds__(256) compact_mark_kernel(PageState st, PageWork wk,
                                                           int per_row) {
  const int s = min((int)blockIdx.x / per_row, st.S);
  const bool is_free = s == st.S;
  const int count = is_free ? *st.top : st.num_pages[s];
  const int j = (blockIdx.x - s * per_row) * 256 + threadIdx.x;
  if (count < 0 || count > (is_free ? st.pool : st.max_pages)) {
    atomicOr(&wk.head[H_ERR], DVS_ERR_MAX_PAGES);
  } else if (j < count) {
    const int p = is_free ? st.stack[j] : st.table[(size_t)s * st.max_pages + j];
    if (mark_page(st, is_free ? wk.free_bits : wk.bits, p, is_free || !st.refs))
      atomicOr(&wk.head[H_ERR], DVS_ERR_BAD_PAGE);
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(PageState st, PageWork wk,
                                                                    int32_t* moved_out) {
  compact_plan(st, wk, wk.bits, wk.free_bits, wk.head[H_ERR], moved_out);
}

// The first row_blocks workgroups follow the moves in the page tables, the
// others copy pages.
__global__ void __launch_bounds__(COPY_THREADS) compact_apply_kernel(PageState st, PageWork wk,
                                                                     int per_row, int row_blocks,
                                                                     Pools pools, int n_pools,
                                                                     int page_bytes) {
  if (wk.head[H_ERR]) return;
  if ((int)blockIdx.x >= row_blocks) {
    copy_pages(wk, pools, n_pools, page_bytes, blockIdx.x - row_blocks, gridDim.x - row_blocks);
    return;
  }
  const int s = blockIdx.x / per_row, j = (blockIdx.x - s * per_row) * COPY_THREADS + threadIdx.x;
  if (j >= st.num_pages[s]) return;
  int32_t* id = st.table + (size_t)s * st.max_pages + j;
  if (*id >= wk.head[H_USED]) *id = wk.pages[*id];
}

}  // namespace dvs

using namespace dvs;

static size_t al(size_t v) { return (v + 255) & ~(size_t)255; }

extern "C" size_t dvs_kv_workspace_bytes(int32_t S, int32_t num_pool_pages) {
  if (S < 1 || S > PLAN_THREADS || num_pool_pages < 1 || num_pool_pages > MAX_POOL) return 0;
  const size_t words = ((size_t)num_pool_pages + 31) / 32;
  return 256 + 4 * al((size_t)S * 4) + 2 * al(words * 4) + 3 * al((size_t)num_pool_pages * 4);
}

static PageWork work_layout(char* ws, int S, int pool) {
  PageWork w;
  w.words = (pool + 31) / 32;
  const size_t per_pair = al((size_t)S * 4), bits = al((size_t)w.words * 4), list = al((size_t)pool * 4);
  w.head = (int32_t*)ws; ws += 256;
  w.full = (int32_t*)ws; ws += per_pair;
  w.need = (int32_t*)ws; ws += per_pair;
  w.pop_at = (int32_t*)ws; ws += per_pair;
  w.copy_at = (int32_t*)ws; ws += per_pair;
  w.bits = (uint32_t*)ws; ws += bits;
  w.free_bits = (uint32_t*)ws; ws += bits;
  w.from = (int32_t*)ws; ws += list;
  w.to = (int32_t*)ws; ws += list;
  w.pages = (int32_t*)ws;
  return w;
}

static int check_state(const char* who, const dvs_state* st, PageState& p, int32_t* refs,
                       void* workspace, size_t ws_bytes) {
  DVS_CHECK_ARG(st && st->kv_len && st->page_table && st->num_pages && st->free_stack &&
                    st->free_top && st->boundary && st->out_tokens && st->out_count && st->finished,
                "%s: invalid state description", who);
  DVS_CHECK_ARG(st->S >= 1 && st->S <= PLAN_THREADS, "%s: need 1 <= S <= %d", who, PLAN_THREADS);
  DVS_CHECK_ARG(st->max_pages >= 1 && st->num_pool_pages >= 1 && st->max_new >= 1,
                "%s: need max_pages, num_pool_pages, max_new >= 1", who);
  DVS_CHECK_ARG(st->max_pages <= (1 << 20), "%s: max_pages over 2^20", who);
  DVS_CHECK_ARG(st->num_pool_pages <= MAX_POOL, "%s: num_pool_pages over 2^29", who);
  DVS_CHECK_ARG(st->draft_width >= 0 && (st->draft || st->draft_width == 0), "%s: bad draft", who);
  const size_t need = dvs_kv_workspace_bytes(st->S, st->num_pool_pages);
  if (!workspace || ws_bytes < need) {
    set_error("%s: workspace needs %zu bytes, got %zu", who, need, ws_bytes);
    return DVS_EWORKSPACE;
  }
  p = PageState{st->S, st->max_pages, st->num_pool_pages, st->draft_width, st->max_new,
                st->kv_len, st->page_table, st->num_pages, st->free_stack, st->free_top,
                st->boundary, st->draft, st->out_tokens, st->out_count, st->finished,
                st->err_word, refs};
  return DVS_OK;
}

static int check_pools(const char* who, const dvs_layer* layers, int n_layers, int n_kv_heads,
                       int head_dim, int dtype) {
  DVS_CHECK_SUPPORTED(dtype == DVS_F32 || dtype == DVS_BF16, "%s: dtype %d", who, dtype);
  DVS_CHECK_ARG(layers && n_layers >= 1 && n_kv_heads >= 1 && head_dim >= 1,
                "%s: need layers, n_layers, n_kv_heads, head_dim >= 1", who);
  DVS_CHECK_ARG((int64_t)n_kv_heads * head_dim <= (1 << 20), "%s: pages too large", who);
  for (int l = 0; l < n_layers; ++l)
    DVS_CHECK_ARG(layers[l].k_pool && layers[l].v_pool &&
                      (((uintptr_t)layers[l].k_pool | (uintptr_t)layers[l].v_pool) & 15) == 0,
                  "%s: layer %d needs pools that start on 16 bytes", who, l);
  return DVS_OK;
}

// Calls f(first, pools, n_pools, workgroups) for the layers, COPY_LAYERS at a
// time; workgroups: enough for `most` pages or to fill the chip.
template <typename F>
static int by_layers(const char* who, const dvs_layer* layers, int n_layers, long long most, F f) {
  for (int l0 = 0; l0 < n_layers; l0 += COPY_LAYERS) {
    const int nl = n_layers - l0 < COPY_LAYERS ? n_layers - l0 : COPY_LAYERS;
    Pools pools{};
    for (int l = 0; l < nl; ++l) {
      pools.p[2 * l] = (char*)layers[l0 + l].k_pool;
      pools.p[2 * l + 1] = (char*)layers[l0 + l].v_pool;
    }
    const long long tasks = most * 2 * nl, cap = 8LL * device_cus();
    f(l0 == 0, pools, 2 * nl, (int)(tasks < cap ? tasks : cap));
    const int rc = launch_status(who);
    if (rc) return rc;
  }
  return DVS_OK;
}

static int page_bytes(int n_kv_heads, int head_dim, int dtype) {
  return n_kv_heads * DVS_PAGE_SIZE * head_dim * (dtype == DVS_BF16 ? 2 : 4);
}

// One workgroup and its LDS for the plan: two launches instead of four.  A fork
// of 7/8 of the slots, pages shared, in a graph and called one by one, us:
//   slots x pages     one workgroup    four launches
//      4 x 252          12.9 / 14.9      14.6 / 20.9
//     32 x 134          15.9 / 16.7      15.9 / 20.1
//     64 x 252          23.1 / 23.4      17.9 / 20.3
// A release is one launch instead of four, for up to twice the entries: 48 slots
// of 134 pages, called one by one, 19.2 / 22.8.
static bool one_workgroup(const PageState& st, int rows, int entries) {
  return (long long)rows * st.max_pages <= entries && st.pool <= SMALL_POOL;
}

// true: in one workgroup, a release to its end.
static bool launch_assign(const PageState& st, const PageWork& wk, const Assign& as,
                          hipStream_t s) {
  if (one_workgroup(st, as.n, as.src ? SMALL_ENTRIES : 2 * SMALL_ENTRIES)) {
    hipLaunchKernelGGL(assign_small_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, st, wk, as);
    return true;
  }
  hipLaunchKernelGGL(assign_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, st, wk, as);
  hipLaunchKernelGGL(assign_drop_kernel, dim3((st.max_pages + 255) / 256, as.n), dim3(256), 0, s,
                     st, wk, as);
  hipLaunchKernelGGL(assign_settle_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, st, wk, as);
  return false;
}

extern "C" int kv_fork(const dvs_state* st, int32_t* page_refs, const dvs_layer* layers,
                       int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                       int32_t n, const int32_t* src, const int32_t* dst, int32_t window,
                       int32_t share, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  PageState p;
  int rc = check_state("kv_fork", st, p, page_refs, workspace, ws_bytes);
  if (rc) return rc;
  if ((rc = check_pools("kv_fork", layers, n_layers, n_kv_heads, head_dim, dtype))) return rc;
  DVS_CHECK_ARG(src && dst, "kv_fork: NULL src or dst");
  DVS_CHECK_ARG(n >= 1 && n < st->S, "kv_fork: need 1 <= n < S (n = %d, S = %d)", n, st->S);
  DVS_CHECK_ARG(window >= 1, "kv_fork: need window >= 1");
  DVS_CHECK_ARG(page_refs || !share, "kv_fork: sharing pages needs page_refs");
  const PageWork wk = work_layout((char*)workspace, st->S, st->num_pool_pages);
  hipStream_t s = (hipStream_t)stream;
  const Assign as{src, dst, n, window, share};
  launch_assign(p, wk, as, s);
  const int per_row = (p.max_pages + COPY_THREADS - 1) / COPY_THREADS, rows = n * per_row;
  const int bytes = page_bytes(n_kv_heads, head_dim, dtype);
  return by_layers("kv_fork", layers, n_layers, share ? n : p.pool,
                   [&](bool first, const Pools& pools, int n_pools, int groups) {
                     if (first)
                       hipLaunchKernelGGL(assign_apply_kernel, dim3(rows + groups),
                                          dim3(COPY_THREADS), 0, s, p, wk, as, per_row, rows,
                                          pools, n_pools, bytes);
                     else
                       hipLaunchKernelGGL(copy_pages_kernel, dim3(groups), dim3(COPY_THREADS), 0, s,
                                          wk, pools, n_pools, bytes);
                   });
}

extern "C" int kv_release(const dvs_state* st, int32_t* page_refs, int32_t n, const int32_t* slots,
                          int32_t window, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  PageState p;
  const int rc = check_state("kv_release", st, p, page_refs, workspace, ws_bytes);
  if (rc) return rc;
  DVS_CHECK_ARG(slots, "kv_release: NULL slots");
  DVS_CHECK_ARG(n >= 1 && n <= st->S, "kv_release: need 1 <= n <= S (n = %d, S = %d)", n, st->S);
  DVS_CHECK_ARG(window >= 1, "kv_release: need window >= 1");
  const PageWork wk = work_layout((char*)workspace, st->S, st->num_pool_pages);
  const Assign as{nullptr, slots, n, window, 0};
  if (!launch_assign(p, wk, as, (hipStream_t)stream)) {
    const int per_row = (p.max_pages + COPY_THREADS - 1) / COPY_THREADS;
    hipLaunchKernelGGL(assign_apply_kernel, dim3(n * per_row), dim3(COPY_THREADS), 0,
                       (hipStream_t)stream, p, wk, as, per_row, n * per_row, Pools{}, 0, 0);
  }
  return launch_status("kv_release");
}

extern "C" int kv_compact(const dvs_state* st, int32_t* page_refs, const dvs_layer* layers,
                          int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                          int32_t* moved_out, void* workspace, size_t ws_bytes, void* stream) {
  clear_error();
  PageState p;
  int rc = check_state("kv_compact", st, p, page_refs, workspace, ws_bytes);
  if (rc) return rc;
  if ((rc = check_pools("kv_compact", layers, n_layers, n_kv_heads, head_dim, dtype))) return rc;
  const PageWork wk = work_layout((char*)workspace, st->S, st->num_pool_pages);
  hipStream_t s = (hipStream_t)stream;
  if (one_workgroup(p, st->S, SMALL_ENTRIES)) {
    hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, p, wk, moved_out);
  } else {
    hipLaunchKernelGGL(compact_clear_kernel, dim3((wk.words + 255) / 256), dim3(256), 0, s, wk);
    const int per_row = (p.max_pages + 255) / 256;
    hipLaunchKernelGGL(compact_mark_kernel, dim3(st->S * per_row + (p.pool + 255) / 256), dim3(256),
                       0, s, p, wk, per_row);
    hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, p, wk, moved_out);
  }
  const int per_row = (p.max_pages + COPY_THREADS - 1) / COPY_THREADS, rows = st->S * per_row;
  const int bytes = page_bytes(n_kv_heads, head_dim, dtype);
  return by_layers("kv_compact", layers, n_layers, p.pool,
                   [&](bool first, const Pools& pools, int n_pools, int groups) {
                     if (first)
                       hipLaunchKernelGGL(compact_apply_kernel, dim3(rows + groups),
                                          dim3(COPY_THREADS), 0, s, p, wk, per_row, rows, pools,
                                          n_pools, bytes);
                     else
                       hipLaunchKernelGGL(copy_pages_kernel, dim3(groups), dim3(COPY_THREADS), 0, s,
                                          wk, pools, n_pools, bytes);
                   });
}
