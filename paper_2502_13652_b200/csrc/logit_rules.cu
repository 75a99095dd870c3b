// Penalties, biases and grammar masks on logits rows, and the history's counts.  See include/c2t.h.
//
// A row is read once and written once; the arithmetic touches only the few tokens that the text or the bias table has, and the rest of a row is
// a copy under the grammar's mask, bound by the memory.  So a block, which has a tile of the vocabulary and some rows of a sequence, first lists the
// tile's tokens that need more than the mask, computes their logits one by one, a thread each, and keeps them in shared memory; then it copies its
// rows, 16 bytes a thread; then it puts the computed logits over them.  (Computing before copying allows in place.  With the arithmetic in the
// copying loop, under a branch per vector, 64 x 60 rows of 128256 bf16 took 583 us: a warp nearly always has a lane that takes it.)
#include <cuda_bf16.h>

#include "c2t_internal.h"

namespace c2t {
namespace {

constexpr int kRuleThreads = 256;
constexpr int kRuleRows = 32;               // rows of a block, at most
constexpr int kRuleBlocks = 6;              // of a multiprocessor
constexpr int kPathMax = C2T_MAX_DEPTH + 1;
constexpr int kRowsAtOnce = 4;
constexpr int kTileTokens = kRuleThreads * 8;                   // of a tile, at most
constexpr int kKept = 4096;                 // computed logits that a block keeps: at least a tile's of one row

struct RuleShared {
  float kept[kKept], path_kept[kRuleRows][kPathMax];
  int marks;                                // tokens of the tile with a count or a bias
  uint16_t mark[kTileTokens];               // which, from the tile's first
  int listed[kRuleRows];                    // path tokens of the row that lie in the tile
  int token[kRuleRows][kPathMax];
  bool path_own[kRuleRows][kPathMax];       // is it a logit that the marks do not have, here for the first time?
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
  static __device__ __forceinline__ uint4 choose(const uint4 &v, unsigned on) {          // -inf where a token is not allowed
    return make_uint4(on & 1 ? v.x : 0xFF800000u, on & 2 ? v.y : 0xFF800000u, on & 4 ? v.z : 0xFF800000u, on & 8 ? v.w : 0xFF800000u);
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
  static __device__ __forceinline__ uint4 choose(const uint4 &v, unsigned on) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    unsigned y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned lo = on >> (2 * i) & 1 ? w[i] : 0xFF80u, hi = on >> (2 * i + 1) & 1 ? w[i] : 0xFF800000u;
      y[i] = __byte_perm(lo, hi, 0x7610);
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
  }
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float *to, float x) { *to = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 *to, float x) { *to = __float2bfloat16_rn(x); }

// Grid (B, groups of rows, tiles of kRuleThreads vectors): the first tiles, with the frequent tokens and the most arithmetic, of all sequences
// begin first.  Dynamic shared memory: 2 N ints for the sequence's nodes.
template <typename T>
__global__ void __launch_bounds__(kRuleThreads, kRuleBlocks) penalize_kernel(const __grid_constant__ c2t_logit_rules a, int rows_per_block) {
  chain_enter();
  constexpr int n = Lanes<T>::n;
  __shared__ RuleShared sh;
  extern __shared__ int nodes[];
  const int b = blockIdx.x, V = a.vocab, r0 = blockIdx.y * rows_per_block;
  int r1 = min(r0 + rows_per_block, a.rows);
  if (a.n_rows_dev) r1 = min(r1, a.n_rows_dev[b]);
  if (r0 >= r1) return;
  const int rows = r1 - r0, tile0 = blockIdx.z * kRuleThreads * n, tile1 = min(tile0 + kRuleThreads * n, V), v0 = tile0 + threadIdx.x * n;
  const int32_t *counts = a.counts_dev ? a.counts_dev + b * a.counts_stride : nullptr;
  const float *bias = a.bias_dev ? a.bias_dev + b * a.bias_stride : nullptr;
  const T *in = static_cast<const T *>(a.in_dev) + b * a.in_seq_stride;
  T *out = static_cast<T *>(a.out_dev) + b * a.out_seq_stride;
  const uint32_t *allowed = a.allowed_dev ? a.allowed_dev + b * a.allowed_seq_stride : nullptr;
  auto count_of = [&](int v) { return counts ? max(counts[v], 0) : 0; };
  auto bias_of = [&](int v) { return bias ? bias[v] : 0.f; };

  // ---- the tile's tokens in the history or the bias table, and the rows' own
  if (threadIdx.x == 0) sh.marks = 0;
  if (threadIdx.x < rows) sh.listed[threadIdx.x] = 0;
  if (a.node_token_dev) {
    for (int i = threadIdx.x; i < a.nodes; i += kRuleThreads) {
      nodes[i] = a.node_token_dev[(long long)b * a.nodes + i];
      nodes[a.nodes + i] = a.node_parent_dev[(long long)b * a.nodes + i];
    }
  }
  unsigned marked = 0;
  if (counts || bias) {
#pragma unroll
    for (int i = 0; i < n; ++i) {           // (side by side in a warp: whole sectors)
      const int v = tile0 + i * kRuleThreads + threadIdx.x;
      if (v < tile1) marked |= (count_of(v) > 0 || bias_of(v) != 0.f ? 1u : 0u) << i;
    }
  }
  __syncthreads();
  if (marked) {
    int at = atomicAdd(&sh.marks, __popc(marked));
    for (; marked; marked &= marked - 1) sh.mark[at++] = (uint16_t)((__ffs(marked) - 1) * kRuleThreads + threadIdx.x);
  }
  if (a.node_token_dev && threadIdx.x < rows) {
    const int r = r0 + threadIdx.x;
    int node = a.row_node_dev ? a.row_node_dev[(long long)b * a.rows + r] : r, found = 0;
    for (int d = 0; d < kPathMax && node >= 0 && node < a.nodes; ++d) {
      const int t = nodes[node];
      if (t >= tile0 && t < tile1) sh.token[threadIdx.x][found++] = t;
      node = nodes[a.nodes + node];
    }
    sh.listed[threadIdx.x] = found;
  }
  __syncthreads();

  // ---- their logits
  const float rep = a.repetition_dev ? a.repetition_dev[b] : 1.f, freq = a.frequency_dev ? a.frequency_dev[b] : 0.f,
              pres = a.presence_dev ? a.presence_dev[b] : 0.f;
  auto is_on = [&](int row, int v) { return !allowed || (allowed[(r0 + row) * a.allowed_row_stride + (v >> 5)] >> (v & 31) & 1); };
  auto ruled = [&](int row, int v, int c, float y, float x, bool on) {          // of row r0 + row, token v: its count and bias; its logit
#pragma unroll 1
    for (int e = 0; e < sh.listed[row]; ++e) c += sh.token[row][e] == v;
    if (c > 0) x = (x > 0.f ? x / rep : x * rep) - freq * (float)c - pres;
    if (y != 0.f) x += y;
    return on ? x : -INFINITY;
  };
  if (a.node_token_dev) {
#pragma unroll 1
    for (int i = threadIdx.x; i < rows * kPathMax; i += kRuleThreads) {
      const int row = i / kPathMax, e = i - row * kPathMax;
      if (e >= sh.listed[row]) continue;
      const int v = sh.token[row][e];
      bool own = count_of(v) == 0 && bias_of(v) == 0.f;
      for (int f = 0; f < e; ++f) own &= sh.token[row][f] != v;
      sh.path_own[row][e] = own;
      if (own) sh.path_kept[row][e] = ruled(row, v, 0, 0.f, to_float(in[(r0 + row) * a.in_row_stride + v]), is_on(row, v));
    }
  }
  const int marks = sh.marks, batch = marks == 0 ? rows : min(rows, kKept / marks);
#pragma unroll 1
  for (int first = 0; first < rows; first += batch) {
    const int size = min(batch, rows - first);
    // a thread has a mark, and every so many-th row: what it loads for its rows goes out together
    const int groups = marks > 0 ? max(kRuleThreads / marks, 1) : 1, group = marks > 0 ? threadIdx.x / marks : 0;
#pragma unroll 1
    for (int k = groups > 1 ? threadIdx.x - group * marks : threadIdx.x; k < marks && (groups == 1 || group < groups); k += kRuleThreads) {
      const int v = tile0 + sh.mark[k], c = count_of(v);
      const float y = bias_of(v);
#pragma unroll 1
      for (int row = groups > 1 ? group : 0; row < size; row += kRowsAtOnce * groups) {
        float x[kRowsAtOnce];
        bool on[kRowsAtOnce];
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
          const int r = first + min(row + u * groups, size - 1);
          x[u] = to_float(in[(r0 + r) * a.in_row_stride + v]);
          on[u] = is_on(r, v);
        }
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u)
          if (row + u * groups < size) sh.kept[(row + u * groups) * marks + k] = ruled(first + row + u * groups, v, c, y, x[u], on[u]);
      }
    }
    __syncthreads();                        // (the rows' path logits are kept too by now: nothing has been written yet)

    // ---- the rows, under the grammar's mask
    const int last = r0 + first + size;
    if (v0 + n <= V) {
#pragma unroll 1
      for (int r = r0 + first; r < last; r += kRowsAtOnce) {
        uint4 raw[kRowsAtOnce];
        unsigned on[kRowsAtOnce];
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) {
          const int row = min(r + u, last - 1);
          raw[u] = *reinterpret_cast<const uint4 *>(in + row * a.in_row_stride + v0);
          on[u] = allowed ? allowed[row * a.allowed_row_stride + (v0 >> 5)] >> (v0 & 31) : ~0u;
        }
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u)
          if (r + u < last) __stcs(reinterpret_cast<uint4 *>(out + (r + u) * a.out_row_stride + v0), Lanes<T>::choose(raw[u], on[u]));
      }
    } else {                                // the vector that reaches over the rows' end
#pragma unroll 1
      for (int i = 0; i < size * (V - v0); ++i) {
        const int r = r0 + first + i / (V - v0), v = v0 + i % (V - v0);
        const bool on = !allowed || (allowed[r * a.allowed_row_stride + (v >> 5)] >> (v & 31) & 1);
        from_float(out + r * a.out_row_stride + v, on ? to_float(in[r * a.in_row_stride + v]) : -INFINITY);
      }
    }
    __syncthreads();

    // ---- and over them what was computed
#pragma unroll 1
    for (int i = threadIdx.x; i < size * marks; i += kRuleThreads) {
      const int row = i / marks;
      from_float(out + (r0 + first + row) * a.out_row_stride + tile0 + sh.mark[i - row * marks], sh.kept[i]);
    }
    if (a.node_token_dev)
#pragma unroll 1
      for (int i = threadIdx.x; i < size * kPathMax; i += kRuleThreads) {
        const int row = first + i / kPathMax, e = i % kPathMax;
        if (e < sh.listed[row] && sh.path_own[row][e]) from_float(out + (r0 + row) * a.out_row_stride + sh.token[row][e], sh.path_kept[row][e]);
      }
    __syncthreads();
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
  if (a.batch > 1 && a.out_seq_stride < a.vocab) return C2T_EINVAL;             // (rows of two sequences in one place)
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
  // As many rows a block as leave the chip several rounds of blocks: 64 x 60 rows of 128256 bf16 take 374 us with 32 rows a block, 389 with 16, 504 with 8;
  // 8 x 60 rows of 32000 take 59, 36, 24.
  int sms = 0, device = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return launched(cudaErrorUnknown);
  int rows_per_block = kRuleRows;
  while (rows_per_block > 8 && (int64_t)tiles * ((a.rows + rows_per_block - 1) / rows_per_block) * a.batch < 4ll * kRuleBlocks * sms) rows_per_block /= 2;
  const int groups = (a.rows + rows_per_block - 1) / rows_per_block;
  if (groups > 65535 || tiles > 65535) return C2T_ERANGE;
  const size_t smem = a.node_token_dev ? 2 * sizeof(int) * (size_t)a.nodes : 0;
  void (*kernel)(c2t_logit_rules, int) = a.dtype == C2T_BF16 ? penalize_kernel<__nv_bfloat16> : penalize_kernel<float>;
  if (smem + sizeof(RuleShared) > 48 * 1024 &&                  // what a block has of both kinds without being asked for
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * sizeof(int) * C2T_MAX_TREE) != cudaSuccess)
    return launched(cudaErrorUnknown);
  return launched(launch_chained(kernel, dim3(a.batch, groups, tiles), dim3(kRuleThreads), smem, (cudaStream_t)stream, a, rows_per_block));
}

int c2t_count_tokens(int32_t *counts_dev, int64_t counts_stride, int32_t batch, int32_t vocab, const int32_t *tokens_dev,
                     int32_t token_width, const int32_t *index_dev, int32_t index_stride, const int32_t *n_dev, int32_t plus_one,
                     int32_t width, int32_t delta, void *stream) {
  if (!counts_dev || !tokens_dev || !n_dev || batch < 1 || vocab < 1 || token_width < 1 || width < 1 || counts_stride < vocab) return C2T_EINVAL;
  if (plus_one != 0 && plus_one != 1) return C2T_EINVAL;
  if (width > (index_dev ? index_stride : token_width)) return C2T_EINVAL;
  if (batch > C2T_MAX_BATCH || width > (1 << 30)) return C2T_ERANGE;
  return launched(launch_chained(count_tokens_kernel, dim3((width + kRuleThreads - 1) / kRuleThreads, batch), dim3(kRuleThreads), 0,
                                 (cudaStream_t)stream, counts_dev, counts_stride, vocab, tokens_dev, token_width, index_dev, index_stride, n_dev,
                                 plus_one, width, delta));
}

}  // extern "C"
