// The paged key/value cache's own operations: room, release, forks, new tokens, the accepted path.  See include/c2t.h.
//
// All of them move bytes and count pages; none computes.  The bookkeeping keeps one count per page and no list of free pages:
// a release is then a decrement whose order does not matter, and an allocation takes the lowest free pages, so that equal calls leave
// equal tables however their threads are timed.
#include "cache_internal.h"

namespace c2t {

int check_cache(const c2t_cache *c) {
  if (!c || !c->k_dev || !c->v_dev || !c->table_dev || !c->held_dev || !c->refs_dev) return C2T_EINVAL;
  if (c->dtype != C2T_BF16 && c->dtype != C2T_F16) return C2T_EINVAL;
  if (c->batch < 1 || c->layers < 1 || c->kv_heads < 1 || c->n_pages < 1 || c->max_pages < 1 || c->page_size < 1) return C2T_EINVAL;
  if (c->layer_stride < 0 || c->page_stride < 0 || c->token_stride < c->head_dim || c->head_stride < c->head_dim) return C2T_EINVAL;
  if (c->batch > C2T_MAX_BATCH || (c->head_dim != 64 && c->head_dim != 128)) return C2T_ERANGE;
  if (c->page_size < 8 || c->page_size > C2T_MAX_PAGE_SIZE || (c->page_size & (c->page_size - 1))) return C2T_ERANGE;
  // positions, and all slots' pages together, are 32-bit numbers
  if ((int64_t)c->max_pages * c->page_size > 0x40000000 || (int64_t)c->max_pages * c->batch > 0x7FFFFFFF) return C2T_ERANGE;
  if (!vector_aligned(c->k_dev) || !vector_aligned(c->v_dev) || !vector_stride(c->layer_stride) || !vector_stride(c->page_stride) ||
      !vector_stride(c->token_stride) || !vector_stride(c->head_stride))
    return C2T_EALIGN;
  return C2T_OK;
}

namespace {

// The planning kernels are one block each and wait for memory and for one another's warps, round by round.  A first round of 2048 counts, then of 8192, by
// 512 threads: a fork of 8 slots and its three other launches take 19.4 us, with 16384 counts a round by 1024 threads 29.3 (64 slots' room given and taken back:
// 5.9, 9.8); where the 256 free pages are the last of 131072, 36.1 and 33.2, with 256 threads 49.8.
constexpr int kPlanThreads = 512;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kFirstScan = 4, kScan = 16;   // counts per lane and round of the search for free pages
constexpr int kCopyThreads = 256;

// the page that holds a position of slot b, -1 where it has none
__device__ __forceinline__ int page_of(const c2t_cache &c, int b, int held, long long position, int page_shift) {
  const long long index = position >> page_shift;
  if (position < 0 || index >= held) return -1;
  const int page = c.table_dev[(long long)b * c.max_pages + index];
  return page < 0 || page >= c.n_pages ? -1 : page;
}

// the element offset of a position in that page, without layer and head
__device__ __forceinline__ long long place_in(const c2t_cache &c, int page, long long position) {
  return page * c.page_stride + (position & (c.page_size - 1)) * c.token_stride;
}

// Does another slot hold the page?  Then nothing is written to it: a slot that was trimmed into a page which it shares with a fork would write over
// that one's tokens.  (Asked of every position that is written: 64 sequences' 60 tokens take 6.8 us with and without it, their paths in 32 layers 16.0 and 15.5.)
__device__ __forceinline__ bool is_shared(const c2t_cache &c, int page) { return c.refs_dev[page] > 1; }

__device__ __forceinline__ int pages_for(const c2t_cache &c, int tokens) { return (tokens + c.page_size - 1) / c.page_size; }

// ---------------------------------------------------------------- pages for the slots' needs

struct PlanShared {
  int offset[C2T_MAX_BATCH + 1];            // slots' needs, summed up
  int warp_sum[kPlanWarps];
  int total;
};

// Exclusive sums of sh.offset[0 .. B), which holds the needs; the total behind them.  All threads.
__device__ void sum_needs(PlanShared &sh, int B) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int carry = 0;
  for (int base = 0; base < B; base += kPlanThreads) {
    const int b = base + threadIdx.x;
    const int need = b < B ? sh.offset[b] : 0;
    int x = need;
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(~0u, x, d);
      if (lane >= d) x += y;
    }
    if (lane == 31) sh.warp_sum[warp] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kPlanWarps; ++w) {
      const int s = sh.warp_sum[w];
      before += w < warp ? s : 0;
      all += s;
    }
    if (b < B) sh.offset[b] = carry + before + x - need;
    carry += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) sh.offset[B] = carry;
  __syncthreads();
}

// One round of take_pages: the counts [base, base + kPlanThreads * n), each warp over a part of its own in ascending order.
template <int n, typename First>
__device__ int take_round(const c2t_cache &c, PlanShared &sh, long long base, int total, int taken, First first) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long at = base + warp * (32 * n) + lane;
  int ref[n];
#pragma unroll
  for (int i = 0; i < n; ++i) ref[i] = at + 32 * i < c.n_pages ? c.refs_dev[at + 32 * i] : 1;
  unsigned free_mask[n];
  int mine = 0;
#pragma unroll
  for (int i = 0; i < n; ++i) {
    free_mask[i] = __ballot_sync(~0u, ref[i] == 0);
    mine += __popc(free_mask[i]);
  }
  if (lane == 0) sh.warp_sum[warp] = mine;
  __syncthreads();
  int rank = taken, all = 0;
  for (int w = 0; w < kPlanWarps; ++w) {
    const int s = sh.warp_sum[w];
    rank += w < warp ? s : 0;
    all += s;
  }
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const int r = rank + __popc(free_mask[i] & ((1u << lane) - 1));
    rank += __popc(free_mask[i]);
    if (ref[i] != 0 || r >= total) continue;
    int lo = 0, hi = c.batch;                          // the last slot whose offset is <= r: later ones with the same offset need nothing
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sh.offset[mid] <= r) lo = mid; else hi = mid;
    }
    c.refs_dev[at + 32 * i] = 1;
    c.table_dev[(long long)lo * c.max_pages + first(lo) + r - sh.offset[lo]] = (int)(at + 32 * i);
  }
  __syncthreads();
  return all;
}

// Gives free pages, in ascending order, to the needs in sh.offset (summed up): the r-th page to entry r - offset[b] of the slot b with
// offset[b] <= r < offset[b + 1], behind the first[b] pages that it has.  Returns how many there were, at most the total.  One read of the
// counts, in rounds, until the needs are met: a short one first, since the free pages are often the first ones, then longer ones, which a
// full pool asks for.
template <typename First>
__device__ int take_pages(const c2t_cache &c, PlanShared &sh, First first) {
  const int total = sh.offset[c.batch];
  int taken = 0;
  long long base = 0;
  if (total > 0) {
    taken = take_round<kFirstScan>(c, sh, base, total, taken, first);
    base += kPlanThreads * kFirstScan;
  }
  for (; base < c.n_pages && taken < total; base += kPlanThreads * kScan) taken += take_round<kScan>(c, sh, base, total, taken, first);
  return taken < total ? taken : total;
}

// The slot whose need is met in part gives its pages back: at most one, since pages go to the slots in order.
template <typename First>
__device__ void undo_part(const c2t_cache &c, const PlanShared &sh, int b, int taken, First first) {
  for (int r = sh.offset[b]; r < taken; ++r) {
    int32_t *entry = c.table_dev + (long long)b * c.max_pages + first(b) + r - sh.offset[b];
    c.refs_dev[*entry] = 0;
    *entry = -1;
  }
}

__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(c2t_cache c, const int32_t *len) {
  chain_enter();
  __shared__ PlanShared sh;
  for (int b = threadIdx.x; b < c.batch; b += kPlanThreads) {
    const int n = len[b], held = held_pages(c, b);
    const bool bad = n < 0 || n > (long long)c.max_pages * c.page_size;
    if (bad) cache_fault(c, b, C2T_ST_BAD_PAGE);
    const int want = bad ? 0 : pages_for(c, n);
    sh.offset[b] = want > held ? want - held : 0;
  }
  __syncthreads();
  sum_needs(sh, c.batch);
  auto first = [&](int b) { return held_pages(c, b); };
  const int taken = take_pages(c, sh, first);
  __syncthreads();
  for (int b = threadIdx.x; b < c.batch; b += kPlanThreads) {
    const int need = sh.offset[b + 1] - sh.offset[b];
    if (need == 0) continue;
    if (sh.offset[b + 1] <= taken) {
      c.held_dev[b] = first(b) + need;
    } else {
      undo_part(c, sh, b, taken, first);
      cache_fault(c, b, C2T_ST_NO_PAGE);
    }
  }
}

__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(c2t_cache c, const int32_t *src, const int32_t *len, int32_t *forked) {
  chain_enter();
  __shared__ PlanShared sh;
  auto valid = [&](int b) {
    const int s = src[b], n = len[b];
    return s < c.batch && s != b && src[s] < 0 && c.held_dev[b] == 0 && n >= 0 && n <= (long long)held_pages(c, s) * c.page_size;
  };
  for (int b = threadIdx.x; b < c.batch; b += kPlanThreads) {
    const bool asked = src[b] >= 0, ok = asked && valid(b);
    if (asked && !ok) cache_fault(c, b, C2T_ST_BAD_PAGE);
    forked[b] = ok;
    sh.offset[b] = ok && len[b] % c.page_size > 0;
  }
  __syncthreads();
  sum_needs(sh, c.batch);
  auto first = [&](int b) { return len[b] / c.page_size; };
  const int taken = take_pages(c, sh, first);
  __syncthreads();
  for (int b = threadIdx.x; b < c.batch; b += kPlanThreads) {
    if (!forked[b]) continue;
    if (sh.offset[b + 1] <= taken || sh.offset[b + 1] == sh.offset[b]) {
      c.held_dev[b] = pages_for(c, len[b]);             // (read by valid() of other slots for their sources only, and b is none)
    } else {
      forked[b] = 0;
      cache_fault(c, b, C2T_ST_NO_PAGE);
    }
  }
}

// Grid (parts, B): the table entries that are shared, and the begun page's tokens in all layers, 16 bytes a thread and turn.
__global__ void __launch_bounds__(kCopyThreads) fork_copy_kernel(c2t_cache c, const int32_t *src, const int32_t *len, const int32_t *forked) {
  chain_enter();
  const int b = blockIdx.y;
  if (!forked[b]) return;
  const int s = src[b], n = len[b], full = n / c.page_size, rest = n % c.page_size;
  const int32_t *from = c.table_dev + (long long)s * c.max_pages;
  int32_t *to = c.table_dev + (long long)b * c.max_pages;
  const int step = gridDim.x * kCopyThreads, me = blockIdx.x * kCopyThreads + threadIdx.x;
  for (int i = me; i < full; i += step) {
    const int page = from[i];
    to[i] = page;
    if (page >= 0 && page < c.n_pages) atomicAdd(c.refs_dev + page, 1);
    else cache_fault(c, b, C2T_ST_BAD_PAGE);
  }
  if (rest == 0) return;
  const int old_page = from[full], new_page = to[full];
  if (old_page < 0 || old_page >= c.n_pages) {
    if (me == 0) cache_fault(c, b, C2T_ST_BAD_PAGE);
    return;
  }
  const int vecs = c.head_dim / 8;
  const int per_layer = rest * c.kv_heads * vecs;
  const long long old_at = old_page * c.page_stride, new_at = new_page * c.page_stride;
  for (long long i = me; i < 2ll * c.layers * per_layer; i += step) {
    const long long slab = i / per_layer;               // layer * 2 + (0: keys, 1: values)
    int r = (int)(i - slab * per_layer);
    const int vec = r % vecs;
    r /= vecs;
    const int h = r % c.kv_heads, t = r / c.kv_heads;
    uint16_t *pool = reinterpret_cast<uint16_t *>(slab & 1 ? c.v_dev : c.k_dev);
    const long long in_page = (slab >> 1) * c.layer_stride + t * c.token_stride + h * c.head_stride + vec * 8;
    *reinterpret_cast<uint4 *>(pool + new_at + in_page) = *reinterpret_cast<const uint4 *>(pool + old_at + in_page);
  }
}

__global__ void __launch_bounds__(kCopyThreads) release_kernel(c2t_cache c, const int32_t *keep_len) {
  chain_enter();
  const int b = blockIdx.x;
  const int held = held_pages(c, b), n = keep_len[b];
  if (n < 0) {
    if (threadIdx.x == 0) cache_fault(c, b, C2T_ST_BAD_PAGE);
    return;
  }
  const long long want = ((long long)n + c.page_size - 1) / c.page_size;
  const int kept = want < held ? (int)want : held;
  int32_t *row = c.table_dev + (long long)b * c.max_pages;
  for (int i = kept + threadIdx.x; i < held; i += kCopyThreads) {
    const int page = row[i];
    row[i] = -1;
    bool bad = page < 0 || page >= c.n_pages;
    if (!bad && atomicSub(c.refs_dev + page, 1) <= 0) {  // a page that nobody holds
      atomicAdd(c.refs_dev + page, 1);
      bad = true;
    }
    if (bad) cache_fault(c, b, C2T_ST_BAD_PAGE);
  }
  __syncthreads();
  if (threadIdx.x == 0) c.held_dev[b] = kept;
}

// ---------------------------------------------------------------- tokens

struct NewTokens {
  const uint16_t *k, *v;
  int64_t seq_stride, token_stride, head_stride;
  int max_new, page_shift;
};

// Grid (parts, B).  A thread moves 16 bytes of a key and of its value; consecutive threads go along a head, then along the heads.
__global__ void __launch_bounds__(kCopyThreads) append_kernel(c2t_cache c, int layer, NewTokens in, const int32_t *start, const int32_t *count) {
  chain_enter();
  const int b = blockIdx.y;
  const int held = held_pages(c, b), first = start[b];
  const int n = min(count[b], in.max_new);
  const int vecs = c.head_dim / 8, per_token = c.kv_heads * vecs;
  uint16_t *k = reinterpret_cast<uint16_t *>(c.k_dev) + layer * c.layer_stride, *v = reinterpret_cast<uint16_t *>(c.v_dev) + layer * c.layer_stride;
  for (long long i = blockIdx.x * kCopyThreads + threadIdx.x; i < (long long)n * per_token; i += gridDim.x * kCopyThreads) {
    const int j = (int)(i / per_token), r = (int)(i - (long long)j * per_token), h = r / vecs, vec = r - h * vecs;
    const long long from = b * in.seq_stride + j * in.token_stride + h * in.head_stride + vec * 8;
    const uint4 key = *reinterpret_cast<const uint4 *>(in.k + from), value = *reinterpret_cast<const uint4 *>(in.v + from);
    const int page = page_of(c, b, held, (long long)first + j, in.page_shift);
    if (page < 0 || is_shared(c, page)) {
      cache_fault(c, b, C2T_ST_BAD_PAGE);
      continue;
    }
    const long long to = place_in(c, page, (long long)first + j) + h * c.head_stride + vec * 8;
    *reinterpret_cast<uint4 *>(k + to) = key;
    *reinterpret_cast<uint4 *>(v + to) = value;
  }
}

constexpr int kPathMax = C2T_MAX_DEPTH + 1;
constexpr int kPathBatch = 8;               // tokens of a path that a thread holds at once

// Grid (parts, B).  A thread owns 16 bytes of every token of (layer, keys or values, head) and goes along the path in order: since
// path[d] >= d ascends, place d is written after every read of it, and a batch is read before any of it is written.
__global__ void __launch_bounds__(kCopyThreads) compact_kernel(c2t_cache c, const int32_t *prefix_len, const int32_t *accept_len, const int32_t *path,
                                                               int path_width, int32_t *new_len, int page_shift) {
  chain_enter();
  __shared__ long long from[kPathMax], to[kPathMax];
  __shared__ int faults;
  const int b = blockIdx.y, n = accept_len[b] + 1, prefix = prefix_len[b];
  if (threadIdx.x == 0) faults = n < 1 || n > path_width || prefix < 0;
  __syncthreads();
  if (!faults && threadIdx.x < n) {
    const int d = threadIdx.x, held = held_pages(c, b);
    const int32_t *p = path + (long long)b * path_width;
    const long long source = (long long)prefix + p[d], target = (long long)prefix + d;
    const int from_page = page_of(c, b, held, source, page_shift), to_page = page_of(c, b, held, target, page_shift);
    if (from_page < 0 || to_page < 0 || p[d] < d || (d > 0 && p[d] <= p[d - 1]) || (p[d] != d && is_shared(c, to_page))) atomicOr(&faults, 1);
    from[d] = place_in(c, from_page, source);
    to[d] = place_in(c, to_page, target);
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (faults) cache_fault(c, b, C2T_ST_BAD_PAGE);
    if (new_len) new_len[b] = faults ? prefix : prefix + n;
  }
  if (faults) return;
  int d0 = 0;
  while (d0 < n && from[d0] == to[d0]) ++d0;            // the path's head stays where it is
  if (d0 == n) return;
  const int vecs = c.head_dim / 8, per_layer = c.kv_heads * vecs;
  for (int i = blockIdx.x * kCopyThreads + threadIdx.x; i < 2 * c.layers * per_layer; i += gridDim.x * kCopyThreads) {
    const int slab = i / per_layer, r = i - slab * per_layer, h = r / vecs, vec = r - h * vecs;
    uint16_t *pool = reinterpret_cast<uint16_t *>(slab & 1 ? c.v_dev : c.k_dev) + (slab >> 1) * c.layer_stride + h * c.head_stride + vec * 8;
    for (int d = d0; d < n; d += kPathBatch) {
      uint4 x[kPathBatch];
#pragma unroll
      for (int u = 0; u < kPathBatch; ++u)
        if (d + u < n) x[u] = *reinterpret_cast<const uint4 *>(pool + from[d + u]);
#pragma unroll
      for (int u = 0; u < kPathBatch; ++u)
        if (d + u < n) *reinterpret_cast<uint4 *>(pool + to[d + u]) = x[u];
    }
  }
}

int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

unsigned parts_for(long long threads, int most) {
  const long long n = (threads + kCopyThreads - 1) / kCopyThreads;
  return (unsigned)(n < 1 ? 1 : n > most ? most : n);
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

int c2t_cache_reserve(const c2t_cache *cache, const int32_t *len_dev, void *stream) {
  const int rc = check_cache(cache);
  if (rc != C2T_OK) return rc;
  if (!len_dev) return C2T_EINVAL;
  return launched(launch_chained(reserve_kernel, dim3(1), dim3(kPlanThreads), 0, (cudaStream_t)stream, *cache, len_dev));
}

int c2t_cache_release(const c2t_cache *cache, const int32_t *keep_len_dev, void *stream) {
  const int rc = check_cache(cache);
  if (rc != C2T_OK) return rc;
  if (!keep_len_dev) return C2T_EINVAL;
  return launched(launch_chained(release_kernel, dim3(cache->batch), dim3(kCopyThreads), 0, (cudaStream_t)stream, *cache, keep_len_dev));
}

int c2t_cache_fork(const c2t_cache *cache, const int32_t *src_dev, const int32_t *len_dev, int32_t *forked_dev, void *stream) {
  int rc = check_cache(cache);
  if (rc != C2T_OK) return rc;
  if (!src_dev || !len_dev || !forked_dev || forked_dev == src_dev || forked_dev == len_dev) return C2T_EINVAL;
  const cudaStream_t s = (cudaStream_t)stream;
  rc = launched(launch_chained(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, *cache, src_dev, len_dev, forked_dev));
  if (rc != C2T_OK) return rc;
  const long long most = 2ll * cache->layers * cache->page_size * cache->kv_heads * (cache->head_dim / 8);
  return launched(launch_chained(fork_copy_kernel, dim3(parts_for(most / 4, 64), cache->batch), dim3(kCopyThreads), 0, s, *cache, src_dev, len_dev,
                                 static_cast<const int32_t *>(forked_dev)));
}

int c2t_cache_append(const c2t_cache *cache, int32_t layer, const void *k_new_dev, const void *v_new_dev, int32_t max_new,
                     int64_t seq_stride, int64_t token_stride, int64_t head_stride, const int32_t *start_dev,
                     const int32_t *count_dev, void *stream) {
  const int rc = check_cache(cache);
  if (rc != C2T_OK) return rc;
  if (!k_new_dev || !v_new_dev || !start_dev || !count_dev || layer < 0 || layer >= cache->layers || max_new < 1) return C2T_EINVAL;
  if (seq_stride < 0 || token_stride < 0 || head_stride < 0) return C2T_EINVAL;
  if (!vector_aligned(k_new_dev) || !vector_aligned(v_new_dev) || !vector_stride(seq_stride) || !vector_stride(token_stride) ||
      !vector_stride(head_stride))
    return C2T_EALIGN;
  const NewTokens in = {static_cast<const uint16_t *>(k_new_dev), static_cast<const uint16_t *>(v_new_dev), seq_stride, token_stride, head_stride,
                        max_new, log2_of(cache->page_size)};
  const long long threads = (long long)max_new * cache->kv_heads * (cache->head_dim / 8);
  return launched(launch_chained(append_kernel, dim3(parts_for(threads, 4096), cache->batch), dim3(kCopyThreads), 0, (cudaStream_t)stream, *cache,
                                 layer, in, start_dev, count_dev));
}

int c2t_cache_compact(const c2t_cache *cache, const int32_t *prefix_len_dev, const int32_t *accept_len_dev, const int32_t *path_dev,
                      int32_t path_width, int32_t *new_len_dev, void *stream) {
  const int rc = check_cache(cache);
  if (rc != C2T_OK) return rc;
  if (!prefix_len_dev || !accept_len_dev || !path_dev || path_width < 1) return C2T_EINVAL;
  if (new_len_dev == prefix_len_dev || new_len_dev == accept_len_dev) return C2T_EINVAL;       // (other blocks still read those)
  if (path_width > kPathMax) return C2T_ERANGE;
  const long long threads = 2ll * cache->layers * cache->kv_heads * (cache->head_dim / 8);
  if (threads > 0x40000000) return C2T_ERANGE;
  return launched(launch_chained(compact_kernel, dim3(parts_for(threads, 4096), cache->batch), dim3(kCopyThreads), 0, (cudaStream_t)stream, *cache,
                                 prefix_len_dev, accept_len_dev, path_dev, path_width, new_len_dev, log2_of(cache->page_size)));
}

}  // extern "C"
