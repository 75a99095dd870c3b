// Attention of a tree's nodes, a prompt's chunk or single tokens over the paged cache.  See include/c2t.h.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cache_internal.h"

namespace c2t {
namespace {

constexpr int kRowWarps = 8;

// What the rows of a sequence see.
struct Sight {
  int prefix, n, keys;                      // cached tokens, new tokens, positions with a held page
  int window, sinks;
  const uint64_t *bits;                     // of the sequence, or null: causal
  const int32_t *positions;                 // of the sequence, or null
  int words;

  __device__ __forceinline__ int position(int j) const {
    return positions ? max(positions[j], prefix) : prefix + j;
  }
  // does the new token i, at position `own`, see key p < keys?
  __device__ __forceinline__ bool sees(int i, int own, int p) const {
    int at = p;
    if (p >= prefix) {
      const int j = p - prefix;
      if (bits ? j >= 64 * words || !(bits[(long long)i * words + (j >> 6)] >> (j & 63) & 1) : j > i) return false;
      if (window > 0) at = position(j);
    }
    return window == 0 || own - at < window || at < sinks;
  }
};

__device__ __forceinline__ Sight sight_of(const c2t_cache &c, const c2t_attention &a, int b) {
  Sight s;
  s.prefix = max(a.prefix_len_dev[b], 0);
  s.n = min(max(a.n_queries_dev[b], 0), a.max_queries);
  const long long held = (long long)held_pages(c, b) * c.page_size, want = (long long)s.prefix + s.n;
  s.keys = (int)min(held, want);
  s.window = a.window;
  s.sinks = a.sinks;
  s.words = a.mask_words;
  s.bits = a.mask_bits_dev ? a.mask_bits_dev + (long long)b * a.max_queries * a.mask_words : nullptr;
  s.positions = a.position_ids_dev ? a.position_ids_dev + (long long)b * a.max_queries : nullptr;
  return s;
}

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }

// One warp, one row (b, i, h): the keys in [lo, hi) one after the other, with the running maximum m (in units of the exponent, base 2), the sum l of
// the weights and their sum over the values, D / 32 elements a lane.
template <typename T, int D>
__device__ void attend_row(const c2t_cache &c, const c2t_attention &a, const Sight &see, int b, int i, int h, int lo, int hi, float &m, float &l,
                           float *o) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const T *q = static_cast<const T *>(a.q_dev) + b * a.q_seq_stride + i * a.q_token_stride + h * a.q_head_stride + lane * E;
  float qe[E];
#pragma unroll
  for (int e = 0; e < E; ++e) qe[e] = to_float(q[e]);
  const long long head = a.layer * c.layer_stride + (h / (a.q_heads / c.kv_heads)) * c.head_stride + lane * E;
  const int own = see.position(i);
  const float unit = a.scale * 1.4426950408889634f;
  for (int p = lo; p < hi; ++p) {
    if (!see.sees(i, own, p)) continue;
    const int page = c.table_dev[(long long)b * c.max_pages + p / c.page_size];
    if (page < 0 || page >= c.n_pages) {
      cache_fault(c, b, C2T_ST_BAD_PAGE);
      continue;
    }
    const long long at = head + page * c.page_stride + (p & (c.page_size - 1)) * c.token_stride;
    const T *k = static_cast<const T *>(c.k_dev) + at, *v = static_cast<const T *>(c.v_dev) + at;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += qe[e] * to_float(k[e]);
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    s *= unit;
    const float top = fmaxf(m, s), keep = m == top ? 1.f : exp2f(m - top), w = s == -INFINITY ? 0.f : exp2f(s - top);
    l = l * keep + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * keep + w * to_float(v[e]);
    m = top;
  }
}

template <typename T, int D>
__device__ __forceinline__ void store_row(const c2t_attention &a, int b, int i, int h, float m, float l, const float *o) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  T *out = static_cast<T *>(a.out_dev) + b * a.out_seq_stride + i * a.out_token_stride + h * a.out_head_stride + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = from_float<T>(l == 0.f ? 0.f : o[e] / l);
  if (a.lse_dev && lane == 0)
    a.lse_dev[((long long)b * a.max_queries + i) * a.q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <typename T, int D>
__global__ void __launch_bounds__(kRowWarps * 32) attend_rows_kernel(c2t_cache c, c2t_attention a) {
  chain_enter();
  const int b = blockIdx.y;
  const long long row = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  const int i = (int)(row / a.q_heads), h = (int)(row % a.q_heads);
  const Sight see = sight_of(c, a, b);
  if (i >= see.n) return;
  if (row == 0 && see.keys < see.prefix + see.n && (threadIdx.x & 31) == 0) cache_fault(c, b, C2T_ST_BAD_PAGE);
  float m = -INFINITY, l = 0.f, o[D / 32];
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  attend_row<T, D>(c, a, see, b, i, h, 0, see.keys, m, l, o);
  store_row<T, D>(a, b, i, h, m, l, o);
}

int check_attention(const c2t_cache *c, const c2t_attention *a) {
  const int rc = check_cache(c);
  if (rc != C2T_OK) return rc;
  if (!a || !a->q_dev || !a->out_dev || !a->n_queries_dev || !a->prefix_len_dev) return C2T_EINVAL;
  if (a->layer < 0 || a->layer >= c->layers || a->q_heads < 1 || a->q_heads % c->kv_heads || a->max_queries < 1) return C2T_EINVAL;
  if (a->window < 0 || a->sinks < 0 || (a->mask_bits_dev && a->mask_words < 1)) return C2T_EINVAL;
  if (!(a->scale > 0.f) || a->scale > 3e38f) return C2T_EINVAL;
  const int64_t strides[] = {a->q_seq_stride, a->q_token_stride, a->q_head_stride, a->out_seq_stride, a->out_token_stride, a->out_head_stride};
  for (int64_t s : strides)
    if (s < 0) return C2T_EINVAL;
  if (a->max_queries > 0x1000000 || a->q_heads > 65536) return C2T_ERANGE;
  if (!vector_aligned(a->q_dev) || !vector_aligned(a->out_dev)) return C2T_EALIGN;
  for (int64_t s : strides)
    if (!vector_stride(s)) return C2T_EALIGN;
  return C2T_OK;
}

}  // namespace
}  // namespace c2t

using namespace c2t;

extern "C" {

size_t c2t_verify_attention_workspace_bytes(const c2t_cache *cache, int32_t q_heads, int32_t max_queries) {
  if (check_cache(cache) != C2T_OK || q_heads < 1 || q_heads % cache->kv_heads || max_queries < 1) return 0;
  return 256;
}

int c2t_verify_attention(const c2t_cache *cache, const c2t_attention *attention, void *workspace_dev, size_t workspace_bytes, void *stream) {
  const int rc = check_attention(cache, attention);
  if (rc != C2T_OK) return rc;
  const c2t_attention &a = *attention;
  if (!workspace_dev) return C2T_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace_dev) & 255) return C2T_EALIGN;
  if (workspace_bytes < c2t_verify_attention_workspace_bytes(cache, a.q_heads, a.max_queries)) return C2T_ERANGE;
  const long long rows = (long long)a.max_queries * a.q_heads;
  const dim3 grid((unsigned)((rows + kRowWarps - 1) / kRowWarps), cache->batch);
  const bool bf16 = cache->dtype == C2T_BF16;
  auto kernel = cache->head_dim == 64 ? (bf16 ? attend_rows_kernel<__nv_bfloat16, 64> : attend_rows_kernel<__half, 64>)
                                      : (bf16 ? attend_rows_kernel<__nv_bfloat16, 128> : attend_rows_kernel<__half, 128>);
  if (launch_chained(kernel, grid, dim3(kRowWarps * 32), 0, (cudaStream_t)stream, *cache, a) != cudaSuccess) {
    cudaGetLastError();
    return C2T_ECUDA;
  }
  return C2T_OK;
}

}  // extern "C"
