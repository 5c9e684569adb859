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
#include "dvs_common.h"

namespace dvs {

constexpr int PLAN_THREADS = 1024;
constexpr int COPY_THREADS = 256;
constexpr int COPY_LAYERS = 64;    // pools per launch (as kernel arguments)

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

__global__ void __launch_bounds__(PLAN_THREADS) assign_plan_kernel(
    PageState st, PageWork wk, int n, const int32_t* __restrict__ src,
    const int32_t* __restrict__ dst, int window, int share) {
  __shared__ int role[PLAN_THREADS];
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  role[t] = 0;
  if (t == 0) s_err = 0;
  __syncthreads();
  int a = -1, b = -1;
  bool ok = false;
  if (t < n) {
    b = dst[t];
    if (src) a = src[t];
    ok = b >= 0 && b < st.S && (!src || (a >= 0 && a < st.S));
    if (ok) {
      ok = !(atomicOr(&role[b], 1) & 1);
      if (src) atomicOr(&role[a], 2);
    }
    if (!ok) atomicOr(&s_err, DVS_ERR_BAD_SLOT);
  }
  __syncthreads();
  if (role[t] == 3) atomicOr(&s_err, DVS_ERR_BAD_SLOT);
  int full = 0, need = 0, have = 0;
  if (ok) {
    const int L = src ? st.kv_len[a] : 0;
    const int old = st.num_pages[b];
    need = L < 0 ? 0 : pages_for((long long)L + window);
    if (L < 0 || need > st.max_pages || old < 0 || old > st.max_pages) {
      atomicOr(&s_err, DVS_ERR_MAX_PAGES);
      need = 0;
    } else {
      have = pages_for(L);
      full = share ? L / DVS_PAGE_SIZE : 0;
      if (src && (st.num_pages[a] < have || st.num_pages[a] > st.max_pages))
        atomicOr(&s_err, DVS_ERR_BAD_PAGE);
    }
  }
  int pops = 0, copies = 0;
  const int pop_at = scan_excl(need - full, sh, pops);
  const int copy_at = scan_excl(have - full, sh, copies);
  if (t < n) {
    wk.full[t] = full;
    wk.need[t] = need;
    wk.pop_at[t] = pop_at;
    wk.copy_at[t] = copy_at;
  }
  for (int i = t; i < wk.words; i += PLAN_THREADS) wk.bits[i] = 0;
  if (t == 0) {
    const int top = *st.top;
    int e = s_err;
    if (top < 0 || top > st.pool) e |= DVS_ERR_POOL_EXHAUSTED;
    wk.head[H_ERR] = e;
    wk.head[H_DROP_ERR] = 0;
    wk.head[H_POPS] = pops;
    wk.head[H_COPIES] = copies;
  }
}

// Pages of destination blockIdx.y, and the ids that its source passes on.
__global__ void __launch_bounds__(256) assign_drop_kernel(PageState st, PageWork wk,
                                                          const int32_t* __restrict__ src,
                                                          const int32_t* __restrict__ dst) {
  if (wk.head[H_ERR]) return;
  const int i = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x, b = dst[i];
  bool bad = false;
  if (j < st.num_pages[b]) {
    const int p = st.table[(size_t)b * st.max_pages + j];
    if (p < 0 || p >= st.pool) {
      bad = true;
    } else {
      const int holders = st.refs ? atomicSub(&st.refs[p], 1) : 0;
      const uint32_t bit = 1u << (p & 31);
      if (holders < 0) bad = true;
      if (holders == 0 && (atomicOr(&wk.bits[p >> 5], bit) & bit)) bad = true;
    }
  }
  if (src && j < pages_for(st.kv_len[src[i]])) {
    const int p = st.table[(size_t)src[i] * st.max_pages + j];
    bad |= p < 0 || p >= st.pool;
  }
  if (bad) atomicOr(&wk.head[H_DROP_ERR], DVS_ERR_BAD_PAGE);
}

__global__ void __launch_bounds__(PLAN_THREADS) assign_settle_kernel(PageState st, PageWork wk) {
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  if (t == 0) s_err = wk.head[H_ERR] | wk.head[H_DROP_ERR];
  __syncthreads();
  const int per = (wk.words + PLAN_THREADS - 1) / PLAN_THREADS;
  const int top0 = *st.top, pops = wk.head[H_POPS];
  int mine = 0, freed = 0;
  if (!s_err)
    for (int i = 0; i < per; ++i) {      // thread 0 has the highest words
      const int w = wk.words - 1 - (t * per + i);
      if (w >= 0) mine += __popc(wk.bits[w]);
    }
  int at = scan_excl(mine, sh, freed);
  const int top1 = top0 + freed;
  if (!s_err) {
    if (t == 0 && (pops > top1 || top1 > st.pool)) atomicOr(&s_err, DVS_ERR_POOL_EXHAUSTED);
    for (int i = max(0, top1 - pops) + t; i < top0; i += PLAN_THREADS)
      if (st.stack[i] < 0 || st.stack[i] >= st.pool) atomicOr(&s_err, DVS_ERR_BAD_PAGE);
  }
  __syncthreads();
  if (s_err) {
    if (t == 0) {
      wk.head[H_DROP_ERR] |= s_err;      // H_ERR still says whether pages were dropped
      set_err(st.err, s_err);
    }
    return;
  }
  for (int i = 0; i < per; ++i) {
    const int w = wk.words - 1 - (t * per + i);
    uint32_t b = w >= 0 ? wk.bits[w] : 0;
    while (b) {
      const int k = 31 - __clz(b), p = w * 32 + k;
      b ^= 1u << k;
      st.stack[top0 + at++] = p;
      if (st.refs) st.refs[p] = 0;
    }
  }
  __threadfence_block();
  __syncthreads();
  for (int k = t; k < pops; k += PLAN_THREADS) {
    wk.pages[k] = st.stack[top1 - 1 - k];
    st.stack[top1 - 1 - k] = -1;
  }
  if (t == 0) *st.top = top1 - pops;
}

__global__ void __launch_bounds__(256) assign_apply_kernel(PageState st, PageWork wk,
                                                           const int32_t* __restrict__ src,
                                                           const int32_t* __restrict__ dst) {
  if (wk.head[H_ERR]) return;
  const int i = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  const int b = dst[i];
  int32_t* row = st.table + (size_t)b * st.max_pages;
  if (wk.head[H_DROP_ERR]) {             // the dropped holders come back
    if (st.refs && j < st.num_pages[b] && row[j] >= 0 && row[j] < st.pool)
      atomicAdd(&st.refs[row[j]], 1);
    return;
  }
  const int a = src ? src[i] : -1;
  const int full = wk.full[i], need = wk.need[i];
  if (j < st.max_pages) {
    int p = -1;
    if (j < full) {
      p = st.table[(size_t)a * st.max_pages + j];
      atomicAdd(&st.refs[p], 1);
    } else if (j < need) {
      p = wk.pages[wk.pop_at[i] + j - full];
      if (src && j < pages_for(st.kv_len[a])) {
        const int c = wk.copy_at[i] + j - full;
        wk.from[c] = st.table[(size_t)a * st.max_pages + j];
        wk.to[c] = p;
      }
    }
    row[j] = p;
  }
  if (blockIdx.x) return;
  const int t = threadIdx.x;
  if (src) {
    for (int k = t; k < st.draft_width; k += 256)
      st.draft[(size_t)b * st.draft_width + k] = st.draft[(size_t)a * st.draft_width + k];
    for (int k = t; k < st.max_new; k += 256)
      st.out_tokens[(size_t)b * st.max_new + k] = st.out_tokens[(size_t)a * st.max_new + k];
  }
  if (t == 0) {
    st.num_pages[b] = need;
    st.kv_len[b] = src ? st.kv_len[a] : 0;
    st.boundary[b] = src ? st.boundary[a] : 0;
    st.out_count[b] = src ? st.out_count[a] : 0;
    st.finished[b] = src ? st.finished[a] : 1;
  }
}

// ---------------------------------------------------------------------------
// page copies
// ---------------------------------------------------------------------------

struct Pools {
  char* p[2 * COPY_LAYERS];              // K and V pool of each layer
};

// Copies page from[c] to page to[c] in every pool, c < head[H_COPIES]; one
// workgroup per page and pool at a time.
__global__ void __launch_bounds__(COPY_THREADS) copy_pages_kernel(PageWork wk, Pools pools,
                                                                  int n_pools, int page_bytes) {
  if (wk.head[H_ERR] | wk.head[H_DROP_ERR]) return;
  const long long tasks = (long long)wk.head[H_COPIES] * n_pools;
  const int vecs = page_bytes / 16;
  for (long long t = blockIdx.x; t < tasks; t += gridDim.x) {
    const int c = (int)(t / n_pools), k = (int)(t - (long long)c * n_pools);
    const u32x4* from = (const u32x4*)(pools.p[k] + (size_t)wk.from[c] * page_bytes);
    u32x4* to = (u32x4*)(pools.p[k] + (size_t)wk.to[c] * page_bytes);
    for (int v = threadIdx.x; v < vecs; v += COPY_THREADS) to[v] = from[v];
  }
}

// ---------------------------------------------------------------------------
// compaction
// ---------------------------------------------------------------------------

__global__ void __launch_bounds__(256) compact_clear_kernel(PageWork wk) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < wk.words) wk.bits[i] = wk.free_bits[i] = 0;
  if (i < H_WORDS) wk.head[i] = 0;
}

// blockIdx.y < S: the pages of sequence blockIdx.y; S: the free stack.
__global__ void __launch_bounds__(256) compact_mark_kernel(PageState st, PageWork wk) {
  const int s = blockIdx.y;
  const bool is_free = s == st.S;
  const int count = is_free ? *st.top : st.num_pages[s];
  const int most = is_free ? st.pool : st.max_pages;
  if (count < 0 || count > most) {
    if (threadIdx.x == 0) atomicOr(&wk.head[H_ERR], DVS_ERR_MAX_PAGES);
    return;
  }
  const int32_t* ids = is_free ? st.stack : st.table + (size_t)s * st.max_pages;
  uint32_t* bits = is_free ? wk.free_bits : wk.bits;
  for (int j = blockIdx.x * 256 + threadIdx.x; j < count; j += gridDim.x * 256) {
    const int p = ids[j];
    bool bad = p < 0 || p >= st.pool;
    if (!bad) {
      const uint32_t bit = 1u << (p & 31);
      const bool again = atomicOr(&bits[p >> 5], bit) & bit;
      bad = again && (is_free || !st.refs);
    }
    if (bad) atomicOr(&wk.head[H_ERR], DVS_ERR_BAD_PAGE);
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(PageState st, PageWork wk,
                                                                    int32_t* moved_out) {
  __shared__ int sh[PLAN_THREADS / 64];
  __shared__ int s_err;
  const int t = threadIdx.x;
  if (t == 0) s_err = wk.head[H_ERR];
  __syncthreads();
  const int per = (wk.words + PLAN_THREADS - 1) / PLAN_THREADS;
  const int w0 = min(wk.words, t * per), w1 = min(wk.words, w0 + per);
  int held = 0, used = 0;
  for (int w = w0; w < w1; ++w) {
    const uint32_t all = (w + 1) * 32 <= st.pool ? ~0u : (1u << (st.pool & 31)) - 1;
    if ((wk.bits[w] ^ wk.free_bits[w]) != all || (wk.bits[w] & wk.free_bits[w]))
      atomicOr(&s_err, DVS_ERR_BAD_PAGE);
    held += __popc(wk.bits[w]);
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
  int holes = 0, movers = 0, n_holes = 0, moved = 0;
  for (int w = w0; w < w1; ++w) {
    holes += __popc(wk.free_bits[w] & low(w));
    movers += __popc(wk.bits[w] & ~low(w));
  }
  int hole_at = scan_excl(holes, sh, n_holes), mover_at = scan_excl(movers, sh, moved);
  for (int w = w0; w < w1; ++w) {
    for (uint32_t b = wk.free_bits[w] & low(w); b; b &= b - 1)
      wk.to[hole_at++] = w * 32 + __ffs(b) - 1;
    for (uint32_t b = wk.bits[w] & ~low(w); b; b &= b - 1)
      wk.from[mover_at++] = w * 32 + __ffs(b) - 1;
  }
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
    wk.head[H_USED] = used;
    wk.head[H_COPIES] = moved;
    if (moved_out) *moved_out = moved;
  }
}

__global__ void __launch_bounds__(256) compact_apply_kernel(PageState st, PageWork wk) {
  if (wk.head[H_ERR]) return;
  const int s = blockIdx.y, j = blockIdx.x * 256 + threadIdx.x;
  if (j >= st.num_pages[s]) return;
  int32_t* id = st.table + (size_t)s * st.max_pages + j;
  if (*id >= wk.head[H_USED]) *id = wk.pages[*id];
}

}  // namespace dvs

using namespace dvs;

static size_t al(size_t v) { return (v + 255) & ~(size_t)255; }

extern "C" size_t dvs_kv_workspace_bytes(int32_t S, int32_t num_pool_pages) {
  if (S < 1 || S > PLAN_THREADS || num_pool_pages < 1) return 0;
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

static int launch_copies(const char* who, const PageWork& wk, const dvs_layer* layers, int n_layers,
                         int n_kv_heads, int head_dim, int dtype, long long most, hipStream_t s) {
  const int page = n_kv_heads * DVS_PAGE_SIZE * head_dim * (dtype == DVS_BF16 ? 2 : 4);
  for (int l0 = 0; l0 < n_layers; l0 += COPY_LAYERS) {
    const int nl = n_layers - l0 < COPY_LAYERS ? n_layers - l0 : COPY_LAYERS;
    Pools pools{};
    for (int l = 0; l < nl; ++l) {
      pools.p[2 * l] = (char*)layers[l0 + l].k_pool;
      pools.p[2 * l + 1] = (char*)layers[l0 + l].v_pool;
    }
    const long long tasks = most * 2 * nl, cap = 8LL * device_cus();
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(tasks < cap ? tasks : cap)),
                       dim3(COPY_THREADS), 0, s, wk, pools, 2 * nl, page);
    const int rc = launch_status(who);
    if (rc) return rc;
  }
  return DVS_OK;
}

static int assign(const char* who, const PageState& st, const PageWork& wk, int n,
                  const int32_t* src, const int32_t* dst, int window, int share, hipStream_t s) {
  const dim3 rows((st.max_pages + 255) / 256, n);
  hipLaunchKernelGGL(assign_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, st, wk, n, src, dst,
                     window, share);
  hipLaunchKernelGGL(assign_drop_kernel, rows, dim3(256), 0, s, st, wk, src, dst);
  hipLaunchKernelGGL(assign_settle_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, st, wk);
  hipLaunchKernelGGL(assign_apply_kernel, rows, dim3(256), 0, s, st, wk, src, dst);
  return launch_status(who);
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
  if ((rc = assign("kv_fork", p, wk, n, src, dst, window, share, s))) return rc;
  const long long most = share ? n : st->num_pool_pages;
  return launch_copies("kv_fork", wk, layers, n_layers, n_kv_heads, head_dim, dtype, most, s);
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
  return assign("kv_release", p, wk, n, nullptr, slots, window, 0, (hipStream_t)stream);
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
  hipLaunchKernelGGL(compact_clear_kernel, dim3((wk.words + 255) / 256), dim3(256), 0, s, wk);
  hipLaunchKernelGGL(compact_mark_kernel, dim3((st->max_pages + 255) / 256, st->S + 1), dim3(256),
                     0, s, p, wk);
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, p, wk, moved_out);
  hipLaunchKernelGGL(compact_apply_kernel, dim3((st->max_pages + 255) / 256, st->S), dim3(256), 0,
                     s, p, wk);
  if ((rc = launch_status("kv_compact"))) return rc;
  return launch_copies("kv_compact", wk, layers, n_layers, n_kv_heads, head_dim, dtype,
                       st->num_pool_pages, s);
}
