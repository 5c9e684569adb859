// attn_tree: attention of a window of drafted rows, whose keys and values are
// in the paged cache already, over the cache and each row's ancestors.
#include <math.h>

#include "dvs_common.h"

namespace dvs {

struct TreeAttn {
  const void *q, *k_pool, *v_pool;
  const int32_t *table, *kv_len, *mask;
  void* out;
  int32_t* err;
  int S, R, W, Hq, Hkv, G, max_pages, pool_pages;
  float scale;
};

// A workgroup a (sequence, row, query head); 256 keys at a time, a thread a
// key, then a thread an element of the head.
template <typename T, int D>
__global__ void __launch_bounds__(256) tree_attn_plain_kernel(TreeAttn p) {
  __shared__ float s_q[D], s_p[256], s_red[8];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int h = blockIdx.x % p.Hq, r = blockIdx.x / p.Hq % p.R, s = blockIdx.x / p.Hq / p.R;
  const int kvh = h / p.G, L = p.kv_len[s];
  if (L < 0 || (long long)L + p.R > (long long)p.max_pages * 16) {
    if (tid == 0) set_err(p.err, DVS_ERR_MAX_PAGES);
    return;
  }
  const size_t row = ((size_t)s * p.R + r) * p.Hq + h;
  const uint32_t* bits = p.mask ? (const uint32_t*)p.mask + ((size_t)s * p.R + r) * p.W : nullptr;
  bool any = !bits;
  if (bits)
    for (int i = 0; i < p.W; ++i) any |= bits[i] != 0;
  const int T1 = any ? L + p.R : 0;
  if (tid < D) s_q[tid] = (float)((const T*)p.q)[row * D + tid];
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc = 0.f;
  const int d = tid % 128, part = tid / 128;
  for (int t0 = 0; t0 < T1; t0 += 256) {
    const int k = t0 + tid;
    float sc = -INFINITY;
    if (k < T1 && (k < L || (bits ? bits[(k - L) >> 5] >> ((k - L) & 31) & 1 : k - L <= r))) {
      const int pg = p.table[(size_t)s * p.max_pages + (k >> 4)];
      if (pg >= 0 && pg < p.pool_pages) {
        const T* kr = (const T*)p.k_pool + (((size_t)pg * p.Hkv + kvh) * 16 + (k & 15)) * D;
        float dot = 0.f;
        for (int e = 0; e < D; ++e) dot = fmaf(s_q[e], (float)kr[e], dot);
        sc = dot * p.scale;
      } else {
        set_err(p.err, DVS_ERR_BAD_PAGE);
      }
    }
    float v = sc;
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    if (lane == 0) s_red[w] = v;
    __syncthreads();
    const float mn = fmaxf(fmaxf(m, fmaxf(s_red[0], s_red[1])), fmaxf(s_red[2], s_red[3]));
    const float al = m == -INFINITY ? 0.f : expf(m - mn);
    const float e = sc == -INFINITY ? 0.f : expf(sc - mn);
    s_p[tid] = sc == -INFINITY ? -1.f : e;
    float sum = e;
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if (lane == 0) s_red[4 + w] = sum;
    __syncthreads();
    l = l * al + ((s_red[4] + s_red[5]) + (s_red[6] + s_red[7]));
    m = mn;
    acc *= al;
    if (d < D)
      for (int j = part; j < 256; j += 2) {
        if (s_p[j] < 0.f) continue;
        const int kk = t0 + j, pg = p.table[(size_t)s * p.max_pages + (kk >> 4)];
        acc = fmaf(s_p[j], (float)((const T*)p.v_pool)[(((size_t)pg * p.Hkv + kvh) * D + d) * 16 + (kk & 15)], acc);
      }
    __syncthreads();
  }
  s_p[tid] = acc;
  __syncthreads();
  if (tid < D) ((T*)p.out)[row * D + tid] = (T)(l > 0.f ? (s_p[tid] + s_p[tid + 128]) / l : 0.f);
}

}  // namespace dvs

using namespace dvs;

extern "C" size_t dvs_tree_workspace_bytes(int32_t S, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                                           int32_t max_pages, int32_t dtype) {
  if (S < 1 || R < 1 || R > 1024 || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 ||
      (D != 64 && D != 96 && D != 128) || max_pages < 1 || (dtype != DVS_F32 && dtype != DVS_BF16))
    return 0;
  return 256;
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
  const size_t need = dvs_tree_workspace_bytes(S, R, Hq, Hkv, D, max_pages, dtype);
  if (!workspace || ws_bytes < need) {
    set_error("attn_tree: workspace needs %zu bytes, got %zu", need, ws_bytes);
    return DVS_EWORKSPACE;
  }
  TreeAttn p{};
  p.q = q; p.k_pool = k_pool; p.v_pool = v_pool; p.table = page_table; p.kv_len = kv_len;
  p.mask = tree_mask; p.out = out; p.err = err_word;
  p.S = S; p.R = R; p.W = (R + 31) / 32; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
  p.max_pages = max_pages; p.pool_pages = num_pool_pages; p.scale = softmax_scale;
  const long long grid = (long long)S * R * Hq;
  DVS_CHECK_SUPPORTED(grid < (1LL << 31), "attn_tree: grid too large");
  hipStream_t st = (hipStream_t)stream;
#define PLAIN(T)                                                                                      \
  if (D == 128) hipLaunchKernelGGL((tree_attn_plain_kernel<T, 128>), dim3(grid), dim3(256), 0, st, p); \
  else if (D == 96) hipLaunchKernelGGL((tree_attn_plain_kernel<T, 96>), dim3(grid), dim3(256), 0, st, p); \
  else hipLaunchKernelGGL((tree_attn_plain_kernel<T, 64>), dim3(grid), dim3(256), 0, st, p);
  if (dtype == DVS_BF16) { PLAIN(__bf16) } else { PLAIN(float) }
#undef PLAIN
  return launch_status("attn_tree");
}
