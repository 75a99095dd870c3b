// Penalties, biases and grammar masks on logits rows, and the history's counts.  See include/c2t.h.
//
// A row is read once and written once; the arithmetic is a handful of operations on the few tokens that the text has, so the
// pass is bound by the memory.  A thread keeps one 16-byte vector position and goes down the rows of its sequence with it: the
// history's counts and the biases of its tokens, which all rows share, are read once and stay in registers.  What differs from row to
// row besides the logits is the grammar's bits and the few tokens on the row's own root path; of those the block lists, once, the ones
// that lie in its tile of the vocabulary.
#include <cuda_bf16.h>

#include "c2t_internal.h"

namespace c2t {
namespace {

constexpr int kRuleThreads = 256;
constexpr int kRuleRows = 32;               // rows of a block, at most
constexpr int kPathMax = C2T_MAX_DEPTH + 1;
constexpr int kRowsAtOnce = 4;

struct RuleShared {
  int listed[kRuleRows];                    // path tokens of the row that lie in the tile
  int token[kRuleRows][kPathMax];
};

template <typename T> struct Lanes;         // elements of 16 bytes
template <> struct Lanes<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void open(const uint4 &v, float *x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 close(const float *x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Lanes<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void open(const uint4 &v, float *x) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ uint4 close(const float *x) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const unsigned *>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// 16 bytes of a row; at the row's end, where a vector would reach behind it, element by element
template <typename T>
__device__ __forceinline__ uint4 load_vector(const T *row, int v0, int V) {
  if (v0 + Lanes<T>::n <= V) return *reinterpret_cast<const uint4 *>(row + v0);
  uint4 x = make_uint4(0, 0, 0, 0);
  T *e = reinterpret_cast<T *>(&x);
#pragma unroll
  for (int i = 0; i < Lanes<T>::n; ++i)
    if (v0 + i < V) e[i] = row[v0 + i];
  return x;
}

template <typename T>
__device__ __forceinline__ void store_vector(T *row, int v0, int V, uint4 x) {
  if (v0 + Lanes<T>::n <= V) {
    *reinterpret_cast<uint4 *>(row + v0) = x;
    return;
  }
  const T *e = reinterpret_cast<const T *>(&x);
#pragma unroll
  for (int i = 0; i < Lanes<T>::n; ++i)
    if (v0 + i < V) row[v0 + i] = e[i];
}

// Grid (tiles of kRuleThreads vectors, groups of rows, B).  Dynamic shared memory: 2 N ints for the sequence's nodes.
template <typename T>
__global__ void __launch_bounds__(kRuleThreads) penalize_kernel(c2t_logit_rules a, int rows_per_block) {
  chain_enter();
  constexpr int n = Lanes<T>::n;
  __shared__ RuleShared sh;
  extern __shared__ int nodes[];
  const int b = blockIdx.z, V = a.vocab;
  const int r0 = blockIdx.y * rows_per_block;
  int r1 = min(r0 + rows_per_block, a.rows);
  if (a.n_rows_dev) r1 = min(r1, a.n_rows_dev[b]);
  if (r0 >= r1) return;
  const int tile0 = blockIdx.x * kRuleThreads * n, v0 = tile0 + threadIdx.x * n;
  const bool live = v0 < V;

  // what the rows share
  float count[n], bias[n];
  bool seen = false;
#pragma unroll
  for (int i = 0; i < n; ++i) count[i] = bias[i] = 0.f;
  if (live && a.counts_dev) {
    const int32_t *c = a.counts_dev + b * a.counts_stride + v0;
#pragma unroll
    for (int i = 0; i < n; ++i)
      if (v0 + i < V) { count[i] = (float)max(c[i], 0); seen |= count[i] > 0.f; }
  }
  if (live && a.bias_dev) {
    const float *s = a.bias_dev + b * a.bias_stride + v0;
#pragma unroll
    for (int i = 0; i < n; ++i)
      if (v0 + i < V) bias[i] = s[i];
  }
  const float rep = a.repetition_dev ? a.repetition_dev[b] : 1.f, freq = a.frequency_dev ? a.frequency_dev[b] : 0.f,
              pres = a.presence_dev ? a.presence_dev[b] : 0.f;

  // the rows' own tokens
  const int rows = r1 - r0;
  if (threadIdx.x < rows) sh.listed[threadIdx.x] = 0;
  if (a.node_token_dev) {
    int *token = nodes, *parent = nodes + a.nodes;
    for (int i = threadIdx.x; i < a.nodes; i += kRuleThreads) {
      token[i] = a.node_token_dev[(long long)b * a.nodes + i];
      parent[i] = a.node_parent_dev[(long long)b * a.nodes + i];
    }
    __syncthreads();
    if (threadIdx.x < rows) {
      const int r = r0 + threadIdx.x;
      int node = a.row_node_dev ? a.row_node_dev[(long long)b * a.rows + r] : r, found = 0;
      for (int d = 0; d < kPathMax && node >= 0 && node < a.nodes; ++d) {
        const int t = token[node];
        if (t >= tile0 && t < tile0 + kRuleThreads * n && t < V) sh.token[threadIdx.x][found++] = t;
        node = parent[node];
      }
      sh.listed[threadIdx.x] = found;
    }
  }
  __syncthreads();
  if (!live) return;

  const T *in = static_cast<const T *>(a.in_dev) + b * a.in_seq_stride;
  T *out = static_cast<T *>(a.out_dev) + b * a.out_seq_stride;
  const uint32_t *allowed = a.allowed_dev ? a.allowed_dev + b * a.allowed_seq_stride + (v0 >> 5) : nullptr;
  for (int r = r0; r < r1; r += kRowsAtOnce) {
    uint4 raw[kRowsAtOnce];
    unsigned on[kRowsAtOnce];
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      if (r + u >= r1) break;
      raw[u] = load_vector(in + (r + u) * a.in_row_stride, v0, V);
      on[u] = allowed ? allowed[(r + u) * a.allowed_row_stride] >> (v0 & 31) : ~0u;
    }
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      if (r + u >= r1) break;
      float x[n];
      Lanes<T>::open(raw[u], x);
      const int listed = sh.listed[r + u - r0];
      if (seen || listed) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
          float c = count[i];
          for (int e = 0; e < listed; ++e) c += sh.token[r + u - r0][e] == v0 + i ? 1.f : 0.f;
          if (c > 0.f) x[i] = (x[i] > 0.f ? x[i] / rep : x[i] * rep) - freq * c - pres;
        }
      }
#pragma unroll
      for (int i = 0; i < n; ++i) x[i] = on[u] >> i & 1 ? x[i] + bias[i] : -INFINITY;
      store_vector(out + (r + u) * a.out_row_stride, v0, V, Lanes<T>::close(x));
    }
  }
}

__global__ void __launch_bounds__(kRuleThreads) count_tokens_kernel(int32_t *counts, int64_t counts_stride, int vocab, const int32_t *tokens,
                                                                    int token_width, const int32_t *index, int index_stride, const int32_t *n,
                                                                    int plus_one, int width, int delta) {
  chain_enter();
  const int b = blockIdx.y, k = blockIdx.x * kRuleThreads + threadIdx.x;
  if (k >= width || k >= (long long)n[b] + plus_one) return;
  const int at = index ? index[(long long)b * index_stride + k] : k;
  if (at < 0 || at >= token_width) return;
  const int t = tokens[(long long)b * token_width + at];
  if (t >= 0 && t < vocab) atomicAdd(counts + b * counts_stride + t, delta);
}

int launched(cudaError_t e) {
  if (e == cudaSuccess) return C2T_OK;
  cudaGetLastError();
  return C2T_ECUDA;
}

}  // namespace
}  // namespace c2t

using namespace c2t;

extern "C" {

int c2t_penalize_logits(const c2t_logit_rules *rules, void *stream) {
  if (!rules || !rules->in_dev || !rules->out_dev) return C2T_EINVAL;
  const c2t_logit_rules &a = *rules;
  if (a.dtype != C2T_F32 && a.dtype != C2T_BF16) return C2T_EINVAL;
  if (a.batch < 1 || a.rows < 1 || a.vocab < 1) return C2T_EINVAL;
  if (a.in_seq_stride < 0 || a.out_seq_stride < 0 || a.in_row_stride < a.vocab || a.out_row_stride < a.vocab) return C2T_EINVAL;
  if (a.counts_dev && a.counts_stride < a.vocab) return C2T_EINVAL;
  if (a.bias_dev && a.bias_stride != 0 && a.bias_stride < a.vocab) return C2T_EINVAL;
  if (a.allowed_dev && (a.allowed_seq_stride < 0 || a.allowed_row_stride < 0)) return C2T_EINVAL;
  if ((a.node_token_dev != nullptr) != (a.node_parent_dev != nullptr) || (a.node_token_dev && a.nodes < 1)) return C2T_EINVAL;
  if (a.in_dev == a.out_dev && (a.in_seq_stride != a.out_seq_stride || a.in_row_stride != a.out_row_stride)) return C2T_EINVAL;
  if (a.batch > C2T_MAX_BATCH || (a.node_token_dev && a.nodes > C2T_MAX_TREE) || a.vocab > (1 << 30)) return C2T_ERANGE;
  const int esz = a.dtype == C2T_BF16 ? 2 : 4;
  auto odd = [&](const void *p, int64_t seq, int64_t row) {
    return (reinterpret_cast<uintptr_t>(p) & 15) || (seq * esz) % 16 || (row * esz) % 16;
  };
  if (odd(a.in_dev, a.in_seq_stride, a.in_row_stride) || odd(a.out_dev, a.out_seq_stride, a.out_row_stride)) return C2T_EALIGN;

  const int tiles = (a.vocab + kRuleThreads * (16 / esz) - 1) / (kRuleThreads * (16 / esz));
  const int rows_per_block = a.rows < kRuleRows ? a.rows : kRuleRows;
  const int groups = (a.rows + rows_per_block - 1) / rows_per_block;
  if (groups > 65535) return C2T_ERANGE;
  const size_t smem = a.node_token_dev ? 2 * sizeof(int) * (size_t)a.nodes : 0;
  void (*kernel)(c2t_logit_rules, int) = a.dtype == C2T_BF16 ? penalize_kernel<__nv_bfloat16> : penalize_kernel<float>;
  if (smem > 32768 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * sizeof(int) * C2T_MAX_TREE) != cudaSuccess)
    return launched(cudaErrorUnknown);
  return launched(launch_chained(kernel, dim3(tiles, groups, a.batch), dim3(kRuleThreads), smem, (cudaStream_t)stream, a, rows_per_block));
}

int c2t_count_tokens(int32_t *counts_dev, int64_t counts_stride, int32_t batch, int32_t vocab, const int32_t *tokens_dev,
                     int32_t token_width, const int32_t *index_dev, int32_t index_stride, const int32_t *n_dev, int32_t plus_one,
                     int32_t width, int32_t delta, void *stream) {
  if (!counts_dev || !tokens_dev || !n_dev || batch < 1 || vocab < 1 || token_width < 1 || width < 1 || counts_stride < vocab) return C2T_EINVAL;
  if (plus_one != 0 && plus_one != 1) return C2T_EINVAL;
  if (width > (index_dev ? index_stride : token_width)) return C2T_EINVAL;
  if (batch > C2T_MAX_BATCH) return C2T_ERANGE;
  return launched(launch_chained(count_tokens_kernel, dim3((width + kRuleThreads - 1) / kRuleThreads, batch), dim3(kRuleThreads), 0,
                                 (cudaStream_t)stream, counts_dev, counts_stride, vocab, tokens_dev, token_width, index_dev, index_stride, n_dev,
                                 plus_one, width, delta));
}

}  // extern "C"
