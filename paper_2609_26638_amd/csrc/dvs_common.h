// Internal helpers shared by the HIP translation units of libdvs.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dvs.h"

namespace dvs {

// Per-thread error message for dvs_last_error().
void set_error(const char* fmt, ...);
void clear_error();

#define DVS_CHECK_ARG(cond, ...)                  \
  do {                                            \
    if (!(cond)) {                                \
      ::dvs::set_error(__VA_ARGS__);              \
      return DVS_EINVAL;                          \
    }                                             \
  } while (0)

#define DVS_CHECK_SUPPORTED(cond, ...)            \
  do {                                            \
    if (!(cond)) {                                \
      ::dvs::set_error(__VA_ARGS__);              \
      return DVS_EUNSUPPORTED;                    \
    }                                             \
  } while (0)

// Launch status after hipLaunchKernelGGL.
int launch_status(const char* what);

// Sampled two-forward round (sample.hip).
int launch_row_stats(const float* logits, int rows, int V, float invT, float2* stats,
                     int32_t* err, hipStream_t st);
int launch_sample_rows(const float* logits, const float2* stats, int V, float invT,
                       const float* u, int u_stride, int S, int R, int32_t* tok, hipStream_t st);
int launch_accept_final(int S, int B, int V, float invT, const float* zv, const float2* sv,
                        const float* zd, const float2* sd, const int32_t* draft, int draft_width,
                        const float* u, int u_stride, int32_t* accept_len, int32_t* am,
                        hipStream_t st);

// Filtered sampling (filter.hip).  Parameters of a request each, device
// arrays; NULL: temperature 1, filter off.
struct RowParams {
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
};

// Row r = s * rows_per_param + i takes the parameters s and u[s * u_stride + i].
int launch_sample_filtered(const void* logits, int dtype, int rows, int V, long long ld,
                           const RowParams& par, int rows_per_param, const float* u, int u_stride,
                           int32_t* token_out, float* prob_out, int32_t* err, hipStream_t st);
// vs, vld, ds, dld: elements from a sequence's (a row's) logits to the next's.
// The final token of sequence s goes to token_out[s * token_stride], or to
// slot accept_len[s] of that row (at_accepted).  ws: filter_cuts_bytes.
size_t filter_cuts_bytes(int S, int B);
int launch_accept_sampled(const void* zv, long long vs, long long vld, const void* zd,
                          long long ds, long long dld, int dtype, int S, int B, int V,
                          const RowParams& par, const int32_t* draft, int draft_width,
                          const float* u, int u_stride, int32_t* accept_len, int32_t* token_out,
                          int token_stride, int at_accepted, int32_t* err, void* ws,
                          hipStream_t st);

// Whether an attention call takes this chunk_keys (what plans its shape needs it).
bool attn_chunk_ok(int chunk_keys);
// Bytes at the start of an attention workspace that hold the split-merge
// counters (zero between calls) for the given call shape.
size_t attn_counter_bytes(int S, int R, int Hq, int Hkv, int D, int max_pages, int chunk_keys,
                          int dtype);

// Widest page table of the tree calls: positions, and the keys of a tile behind
// the last one, stay within 31 bits.
constexpr int TREE_MAX_PAGES = (1 << 27) - 4;

// accept_commit_tree: a step's trees and what its launches hand on.
struct TreeCommit {
  int S, R, max_pages, pool_pages, n_window_pages;
  const int32_t *parent, *tokens, *argmax, *kv_len, *table, *finished;
  int32_t *accept, *path;                      // outputs (or workspace)
  int32_t *run_len, *old_len, *movable, *pages, *run;    // workspace
};
// Page i of a sequence's window, -1 for an id outside the pool.  (No slot behind
// the table or of a negative length is moved: the commit refuses such a sequence.)
__device__ __forceinline__ int tree_window_page(const TreeCommit& t, int s, int L, int i) {
  const int pg = L / DVS_PAGE_SIZE + i;
  if (L < 0 || pg >= t.max_pages) return 0;
  const int id = t.table[(size_t)s * t.max_pages + pg];
  return id >= 0 && id < t.pool_pages ? id : -1;
}
// Whether the commit's launch accepts as well; the commit (commit.hip).
bool tree_accept_in_commit(const TreeCommit& t);
int commit_tree_run(const dvs_state* st, const TreeCommit& t, void* stream);

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_bits_to_f32(uint32_t b16) {
  return __uint_as_float(b16 << 16);
}

// The value of lane ^ 32 and this lane's, in lane order: (v[l & 31], v[l | 32]).
// gfx950's v_permlane32_swap exchanges the upper half of its first operand
// with the lower half of its second; with both equal to v, lane l ends up
// holding v[l & 31] in the first result and v[l | 32] in the second (a VALU
// exchange, not the LDS round trip of a general shuffle).  Both halves see the
// pair in the same order, so a sum of the two is identical on all 64 lanes.
__device__ __forceinline__ f32x2 halves_pair(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

__device__ __forceinline__ void set_err(int32_t* err, int32_t bit) {
  if (err) atomicOr(err, bit);
}

// Compile-time loop: f(IC<I>{}) for I = B .. E-1, so that an index can select
// registers (ring slots, fragment arrays) without dynamic indexing.
template <int N>
struct IC {
  static constexpr int value = N;
};

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(IC<I>{});
    static_for<I + 1, N>(f);
  }
}

// Compute units of the current device (queried once; 256 if the query fails).
inline int device_cus() {
  static int cus = 0;
  if (cus == 0) {
    int dev = 0, v = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0)
      cus = v;
    else
      cus = 256;
  }
  return cus;
}

}  // namespace dvs
