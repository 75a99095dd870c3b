// Attention of a tree's nodes, a prompt's chunk or single tokens over the paged cache.  See include/c2t.h.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include <cuda.h>

#include "cache_internal.h"
#include "tensor_core.cuh"

namespace c2t {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
  const float unit = a.scale * kLog2e;
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

// ---------------------------------------------------------------- the blocks of work
// The rows of a sequence and a key head are (new token, query head of the group), token-major; 256 of them, or what is left of a
// sequence, form a block of rows.  Its keys are cut into tiles of 128: those that hold the sinks, then those from the first key that a
// row's window can reach.  All of it follows from the lengths on the device.

constexpr int kTile = 128;                  // keys of a tile
constexpr int kRows = 128;                  // rows of one accumulator
constexpr int kBlockRows = 2 * kRows;

struct Params {
  c2t_cache c;
  c2t_attention a;
  int group, blocks_per_seq;                // query heads of a key head; blocks of max_queries * group rows
  int box_rows;                             // tokens of one copy: a page's, at most a tile's
  int split;                                // 1: tiles are dealt out evenly, blocks of rows may be cut; 0: whole blocks
  float *part_o;                            // [2 G][kBlockRows][D]: unfinished sums over the values, two per thread block
  float2 *part_ml;                          // [2 G][kBlockRows]: their maximum (scaled, base 2) and sum of weights
  int4 *cut;                                // [G]: {pair, key head, first thread block, last} of a cut block of rows
};

struct Maps { TensorMap k, v; };

struct Block {
  Sight see;
  int b, row0, rows;                        // first row; rows that are there
  int sink_tiles, first_tile, tiles;
  __device__ __forceinline__ int key0(int t) const { return (t < sink_tiles ? t : first_tile + t - sink_tiles) * kTile; }
};

__device__ __forceinline__ Block block_of(const Params &p, int pair) {
  Block w;
  w.b = pair / p.blocks_per_seq;
  w.row0 = (pair - w.b * p.blocks_per_seq) * kBlockRows;
  w.see = sight_of(p.c, p.a, w.b);
  const Sight &s = w.see;
  const long long all = (long long)s.n * p.group;
  w.rows = (int)min(max(all - w.row0, 0ll), (long long)kBlockRows);
  w.sink_tiles = w.first_tile = w.tiles = 0;
  if (w.rows == 0) return w;
  const int first = w.row0 / p.group, last = (w.row0 + w.rows - 1) / p.group;
  const int end = s.bits ? s.keys : min(s.keys, s.prefix + last + 1);
  const int end_tile = (end + kTile - 1) / kTile;
  if (s.window > 0) {
    const int lowest = s.prefix + (s.positions ? 0 : first);                    // the lowest position of a row
    w.first_tile = min(max(lowest - s.window + 1, 0) / kTile, max(end_tile - 1, 0));
    w.sink_tiles = min((min(s.sinks, end) + kTile - 1) / kTile, w.first_tile);
  }
  w.tiles = max(w.sink_tiles + end_tile - w.first_tile, 1);                     // (rows that see nothing are written too)
  return w;
}

// The thread block's share: a walk over (pair, key head, tiles).  Every role of the block makes the same one.
struct Walk {
  long long left;                           // tiles to go (dealt out) or pairs-and-heads (whole blocks)
  int pair, head, k0, k1;
  Block w;
};

__device__ __forceinline__ bool walk_load(const Params &p, Walk &x, int n_pairs) {        // to the next pair that has rows
  while (x.pair < n_pairs) {
    x.w = block_of(p, x.pair);
    if (x.w.tiles > 0) return true;
    ++x.pair;
  }
  return false;
}

// Makes [k0, k1) the next tiles; false at the end.
__device__ __forceinline__ bool walk_next(const Params &p, Walk &x, int n_pairs, bool first) {
  if (p.split) {
    if (!first) {
      x.left -= x.k1 - x.k0;
      if (x.left <= 0) return false;
      x.k0 = 0;
      if (++x.head == p.c.kv_heads) {
        x.head = 0;
        ++x.pair;
        if (!walk_load(p, x, n_pairs)) return false;
      }
    } else if (x.left <= 0) {
      return false;
    }
    x.k1 = (int)min((long long)x.w.tiles, x.k0 + x.left);
    return true;
  }
  long long item = first ? blockIdx.x : x.left + gridDim.x;
  for (; item < (long long)n_pairs * p.c.kv_heads; item += gridDim.x) {
    const int pair = (int)(item / p.c.kv_heads);
    if (first || pair != x.pair) x.w = block_of(p, pair);
    x.pair = pair;
    x.head = (int)(item - (long long)pair * p.c.kv_heads);
    first = false;
    if (x.w.tiles > 0) {
      x.left = item;
      x.k0 = 0;
      x.k1 = x.w.tiles;
      return true;
    }
  }
  return false;
}

// ---------------------------------------------------------------- the kernel
// Two accumulators of 128 rows, each with a group of four warps that takes its logits through the softmax.  A block of more than 128
// rows has its halves in them, which read the same tiles; a smaller one goes over its tiles with both, the even ones and the odd ones, and
// adds up at the end.  Either way one group's exponentials run while the tensor cores work for the other.
//   warp 8   issues the products: logits S = Q K^T (both from shared memory), and O += P V with P, the weights, in tensor memory in S's place
//   warp 9   copies the tiles of keys and values, a box per page and 64 elements of a head, into a ring of buffers
//   warps 0-3, 4-7   a thread per row: S from tensor memory, its maximum, the weights back as 16-bit numbers
// The running maximum is only raised when a row's new one is more than 2^8 in weight above it: then O and the sum are rescaled.  Weights
// are so at most 2^8, which both types hold.

constexpr int kSoftmaxThreads = 256, kThreads = 320;
constexpr int kMathColumns = 512;           // of tensor memory: S 2 x 128, O 2 x 128 at most
constexpr float kRaise = 8.f;
constexpr int kTries = 1 << 22;             // of a wait, after which the block gives up

template <int D> struct Ring { static constexpr int bytes = kTile * D * 2, n = D == 128 ? 5 : 10; };

template <int D>
struct alignas(1024) Shared {
  unsigned char q[2][kRows * D * 2];        // 64 elements of all rows after the other 64
  union {
    unsigned char ring[Ring<D>::n][Ring<D>::bytes];
    long long before[C2T_MAX_BATCH + 1];    // while the work is dealt out: tiles of the pairs before
  };
  float2 ml[2][kRows];
  uint64_t full[Ring<D>::n], empty[Ring<D>::n];
  uint64_t logits[2], weights[2], done, queries, halves;
  uint32_t tmem;
  int gave_up;
  long long warp_sum[kThreads / 32];
  long long left;
  int pair, head, k0;
};

constexpr int kMaxPairs = C2T_MAX_BATCH;    // for an even deal

template <int D>
__device__ __forceinline__ bool wait(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
  for (int i = 0; i < kTries; ++i) {
    if (barrier_try(bar, parity)) return true;
    if ((i & 63) == 63 && *(volatile int *)&sh.gave_up) return false;
  }
  sh.gave_up = 1;
  return false;
}

// place of a tile's keys or values in the order of the copies: K_0 .. K_{ahead-1}, then V_t, K_{t+ahead}
__device__ __forceinline__ int place_of_keys(int t, int ahead) { return t < ahead ? t : 2 * t - ahead + 1; }
__device__ __forceinline__ int place_of_values(int t, int n, int ahead) { return min(n, ahead + t) + t; }

// bits 0..31: columns c < n
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// which of the 32 keys from `key` row i sees
__device__ __forceinline__ uint32_t sight_bits(const Sight &s, int i, int own, int key) {
  uint32_t on = low_bits(s.keys - key);
  const int node = key - s.prefix;          // of the first of them
  const uint32_t cached = low_bits(-node);
  uint32_t tree = ~0u;
  if (node + 31 >= 0) {
    if (s.bits) {
      const uint64_t *row = s.bits + (long long)i * s.words;
      const int from = max(node, 0), word = from >> 6, bit = from & 63;
      uint64_t x = word < s.words ? row[word] >> bit : 0;
      if (bit && word + 1 < s.words) x |= row[word + 1] << (64 - bit);
      tree = (uint32_t)x << (from - node);
    } else {
      tree = low_bits(i + 1 - node);
    }
  }
  if (s.window > 0) {
    const uint32_t sink = low_bits(s.sinks - key);
    uint32_t near = ~low_bits(own - s.window + 1 - key);
    if (node + 31 >= 0 && s.positions && own - s.prefix >= s.window) {          // nodes' positions are their levels': one by one
      uint32_t nodes = tree & ~cached & on;
      tree &= ~nodes;
      while (nodes) {
        const int c = __ffs(nodes) - 1;
        nodes &= nodes - 1;
        const int at = s.position(node + c);
        if (own - at < s.window || at < s.sinks) tree |= 1u << c;
      }
      near |= ~cached;
    } else if (s.positions) {
      near |= ~cached;                      // no node is further away than the prefix's end
    }
    on &= near | (sink & cached) | (s.positions ? 0u : sink);
  }
  return on & (cached | tree);
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&x);
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  const __half2 x = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&x);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) attend_tiles_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  constexpr int kRing = Ring<D>::n;
  constexpr bool kBf16 = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ __align__(1024) unsigned char raw[];       // (the tiles' swizzle goes by the address)
  Shared<D> &sh = *reinterpret_cast<Shared<D> *>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_pairs = p.c.batch * p.blocks_per_seq, G = gridDim.x;

  chain_release();
  if (warp == 8) tmem_alloc(&sh.tmem, kMathColumns);
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) { barrier_init(sh.full + i, 1); barrier_init(sh.empty + i, 1); }
    for (int s = 0; s < 2; ++s) { barrier_init(sh.logits + s, 1); barrier_init(sh.weights + s, kRows); }
    barrier_init(&sh.done, 1);
    barrier_init(&sh.queries, kSoftmaxThreads);
    barrier_init(&sh.halves, kSoftmaxThreads);
    barrier_init_fence();
    sh.gave_up = 0;
    tensor_map_prefetch(&maps.k);
    tensor_map_prefetch(&maps.v);
  }
  chain_wait();

  // ---- the block's share of the tiles
  if (p.split) {
    long long carry = 0;
    for (int base = 0; base < n_pairs; base += kThreads) {
      const int pair = base + tid;
      const long long mine = pair < n_pairs ? block_of(p, pair).tiles : 0;
      long long x = mine;
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
      }
      if (lane == 31) sh.warp_sum[warp] = x;
      __syncthreads();
      long long earlier = 0, all = 0;
      for (int w = 0; w < kThreads / 32; ++w) {
        const long long s = sh.warp_sum[w];
        earlier += w < warp ? s : 0;
        all += s;
      }
      if (pair < n_pairs) sh.before[pair] = carry + earlier + x - mine;
      carry += all;
      __syncthreads();
    }
    if (tid == 0) {
      const long long total = carry * p.c.kv_heads, used = total < G ? max(total, 1ll) : G;        // (no block without a tile)
      const long long begin = blockIdx.x < used ? blockIdx.x * total / used : total, end = blockIdx.x < used ? (blockIdx.x + 1) * total / used : total;
      sh.left = end - begin;
      int4 cut = make_int4(-1, 0, 0, 0);
      if (end > begin) {
        int lo = 0, hi = n_pairs;           // the last pair whose tiles begin at or before `begin` and that has any
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sh.before[mid] * p.c.kv_heads <= begin) lo = mid; else hi = mid;
        }
        const long long tiles = (lo + 1 < n_pairs ? sh.before[lo + 1] : carry) - sh.before[lo];
        const long long in_pair = begin - sh.before[lo] * p.c.kv_heads;
        sh.pair = lo;
        sh.head = (int)(in_pair / tiles);
        sh.k0 = (int)(in_pair % tiles);
        if (sh.k0 > 0) {                    // a block of rows that an earlier thread block began
          const long long item = begin - sh.k0, item_last = item + tiles - 1;
          const int c0 = (int)(((item + 1) * used - 1) / total), c1 = (int)(((item_last + 1) * used - 1) / total);
          if (c0 == (int)blockIdx.x - 1) cut = make_int4(lo, sh.head, c0, c1);
        }
      }
      p.cut[blockIdx.x] = cut;
    }
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = sh.tmem;
  Walk x;
  x.left = sh.left;
  x.pair = sh.pair; x.head = sh.head; x.k0 = sh.k0; x.k1 = 0;
  __syncthreads();                          // (the ring's memory is free from here on)
  bool more = p.split ? x.left > 0 : true;
  if (p.split && more) x.w = block_of(p, x.pair);
  more = more && walk_next(p, x, n_pairs, true);

  if (warp == 9) {
    // ------------------------------------------------------------ copies
    const int box_bytes = p.box_rows * 128, boxes = kTile / p.box_rows * (D / 64);
    const int half = lane / (kTile / p.box_rows), part = lane % (kTile / p.box_rows);
    const int page_shift = __ffs(p.c.page_size) - 1;
    int turn = 0;                           // buffers filled so far
    bool ok = true;
    for (; more && ok; more = walk_next(p, x, n_pairs, false)) {
      const Block &w = x.w;
      const int n = x.k1 - x.k0, ahead = w.rows > kRows ? 1 : 2;
      if (x.head == 0 && x.k0 == 0 && w.row0 == 0 && lane == 0 && w.see.keys < w.see.prefix + w.see.n) cache_fault(p.c, w.b, C2T_ST_BAD_PAGE);
      const int32_t *table = p.c.table_dev + (long long)w.b * p.c.max_pages;
      for (int i = 0; i < 2 * n && ok; ++i, ++turn) {
        // the i-th copy of the walk's order: keys or values of which tile
        const bool values = i < min(n, ahead) ? false : i >= 2 * n - min(n, ahead) ? true : ((i - ahead) & 1) == 0;
        const int t = !values ? (i < ahead ? i : (i + ahead - 1) / 2) : i >= 2 * n - min(n, ahead) ? i - n : (i - ahead) / 2;
        const int key = w.key0(x.k0 + t) + part * p.box_rows;
        int page = p.c.n_pages;             // behind the pool: zeros
        if (lane < boxes && key < w.see.keys) {
          page = table[key >> page_shift];
          if (page < 0 || page >= p.c.n_pages) {
            page = p.c.n_pages;
            cache_fault(p.c, w.b, C2T_ST_BAD_PAGE);
          }
        }
        const int at = turn % kRing;
        ok = wait(sh, sh.empty + at, (turn / kRing & 1) ^ 1);
        ok = __all_sync(~0u, ok);
        if (!ok) break;
        if (lane == 0) barrier_expect(sh.full + at, Ring<D>::bytes);
        __syncwarp();
        if (lane < boxes)
          copy_box(shared_address(sh.ring[at]) + half * (kTile * 128) + part * box_bytes, values ? &maps.v : &maps.k, sh.full + at, half * 64, x.head,
                   key & (p.c.page_size - 1), page, p.a.layer);
      }
      if (!ok && lane == 0) cache_fault(p.c, w.b, C2T_ST_INTERNAL);
    }
    if (*(volatile int *)&sh.gave_up && lane == 0)             // nothing may arrive in a block's memory that has ended
      for (int i = max(turn - kRing, 0); i < turn; ++i)
        for (int tries = 0; tries < kTries && !barrier_try(sh.full + i % kRing, i / kRing & 1); ++tries) {}
    __syncwarp();
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    if (lane == 0) {
      constexpr uint32_t kLogits = product_descriptor(kBf16, kTile, false), kMix = product_descriptor(kBf16, D, true);
      const uint32_t q0 = shared_address(sh.q[0]), q1 = shared_address(sh.q[1]);
      int turn = 0, items = 0, weights_turn[2] = {0, 0};
      bool ok = true;
      auto buffer = [&](int i) { return shared_address(sh.ring[(turn + i) % kRing]); };
      auto filled = [&](int i) { return wait(sh, sh.full + (turn + i) % kRing, (turn + i) / kRing & 1); };
      auto release = [&](int i) { products_commit(sh.empty + (turn + i) % kRing); };
      auto logits = [&](int s, uint32_t q, uint32_t k) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const uint32_t off = (d >> 2) * (kTile * 128) + (d & 3) * 32;         // 64 elements, then the other 64; 16 of them a step
          product_shared(tmem + s * kTile, tile_descriptor(q + off, 1024, 16), tile_descriptor(k + off, 1024, 16), kLogits, d > 0);
        }
        products_commit(sh.logits + s);
      };
      auto mix = [&](int s, uint32_t v, bool add) {
        ok = ok && wait(sh, sh.weights + s, weights_turn[s]++ & 1);
        if (!ok) return;
        tmem_fence_after();
#pragma unroll
        for (int d = 0; d < kTile / 16; ++d)
          product_tensor(tmem + 256 + s * 128, tmem + s * kTile + d * 8, tile_descriptor(v + d * 2048, 1024, kTile * 128), kMix, add || d > 0);
      };
      for (; more && ok; more = walk_next(p, x, n_pairs, false), ++items) {
        const int n = x.k1 - x.k0;
        ok = wait(sh, &sh.queries, items & 1);
        if (!ok) break;
        tmem_fence_after();
        if (x.w.rows > kRows) {             // both halves of the rows over every tile
          if (!(ok = filled(0))) break;
          logits(0, q0, buffer(0));
          logits(1, q1, buffer(0));
          release(0);
          for (int t = 0; t < n && ok; ++t) {
            const int v = place_of_values(t, n, 1), k = place_of_keys(t + 1, 1);
            if (!(ok = filled(v))) break;
            mix(0, buffer(v), t > 0);
            if (!ok) break;
            if (t + 1 < n) {
              if (!(ok = filled(k))) break;
              logits(0, q0, buffer(k));
            }
            mix(1, buffer(v), t > 0);
            if (!ok) break;
            release(v);
            if (t + 1 < n) {
              logits(1, q1, buffer(k));
              release(k);
            }
          }
        } else {                            // all rows, every other tile
          for (int t = 0; t < min(n, 2) && ok; ++t) {
            if (!(ok = filled(t))) break;
            logits(t, q0, buffer(t));
            release(t);
          }
          for (int t = 0; t < n && ok; ++t) {
            const int v = place_of_values(t, n, 2), k = place_of_keys(t + 2, 2);
            if (!(ok = filled(v))) break;
            mix(t & 1, buffer(v), t > 1);
            if (!ok) break;
            release(v);
            if (t + 2 < n) {
              if (!(ok = filled(k))) break;
              logits(t & 1, q0, buffer(k));
              release(k);
            }
          }
        }
        if (!ok) break;
        products_commit(&sh.done);
        turn += 2 * n;
      }
      if (!ok) {                            // what is in flight must not outlive its tensor memory
        products_commit(&sh.done);
        for (int tries = 0; tries < kTries && !barrier_try(&sh.done, items & 1); ++tries) {}
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int s = warp >> 2, row = tid & 127;                   // the accumulator; the row in it = the lane of tensor memory
    const uint32_t my_s = tmem + s * kTile + ((uint32_t)(warp & 3) << 21), my_o = my_s + 256 + s * (128 - kTile);
    const float unit = p.a.scale * kLog2e;
    int turn = 0, items = 0, logits_turn = 0, both_turn = 0;
    bool ok = true;
    for (; more && ok; more = walk_next(p, x, n_pairs, false), ++items) {
      const Block &w = x.w;
      const Sight &see = w.see;
      const bool two = w.rows > kRows;
      const int n = x.k1 - x.k0, ahead = two ? 1 : 2;
      // the rows' queries, swizzled
      {
        constexpr int kPieces = D / 8;
        const int halves = two ? 2 : 1;
        for (int i = tid; i < halves * kRows * kPieces; i += kSoftmaxThreads) {
          const int r = i / kPieces, piece = i % kPieces, place = r & 127;
          uint4 q = make_uint4(0, 0, 0, 0);
          if (r < w.rows) {
            const int at = w.row0 + r, node = at / p.group, h = x.head * p.group + at - node * p.group;
            q = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.a.q_dev) + w.b * p.a.q_seq_stride + node * p.a.q_token_stride +
                                                 h * p.a.q_head_stride + piece * 8);
          }
          *reinterpret_cast<uint4 *>(sh.q[r >> 7] + (piece >> 3) * (kRows * 128) + place * 128 + (((piece & 7) ^ (place & 7)) << 4)) = q;
        }
        shared_writes_fence();
        tmem_fence_before();
        barrier_arrive(&sh.queries);
      }
      const int my_row = two ? s * kRows + row : row;            // in the block
      const bool live = my_row < w.rows;
      const bool warp_live = (my_row & ~31) < w.rows;
      const int at = w.row0 + (live ? my_row : w.rows - 1), node = at / p.group, head = x.head * p.group + at - node * p.group;
      const int own = see.position(node);
      float m = -INFINITY, l = 0.f;
      for (int t = two ? 0 : s; t < n; t += ahead) {
        const int key = w.key0(x.k0 + t);
        const bool all = key + kTile <= see.prefix && key + kTile <= see.keys && (see.window == 0 || key > own - see.window || key + kTile <= see.sinks);
        const bool masked = !__all_sync(~0u, all);
        uint32_t on0 = ~0u, on1 = ~0u, on2 = ~0u, on3 = ~0u;
        if (masked && warp_live) {          // (while the logits are on their way)
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            on0 = on1; on1 = on2; on2 = on3;
            on3 = sight_bits(see, node, own, key + 32 * i);
          }
        }
        if (!(ok = wait(sh, sh.logits + s, logits_turn++ & 1))) break;
        tmem_fence_after();
        if (key + kTile > see.keys) {       // rows of the values that nobody wrote: their weights are 0, they must be numbers
          const int at_v = turn + place_of_values(t, n, ahead);
          if (!(ok = wait(sh, sh.full + at_v % kRing, at_v / kRing & 1))) break;
          if (key + row >= see.keys && !(two && s == 1)) {       // (the first group's are in time for both)
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
              *reinterpret_cast<uint4 *>(sh.ring[at_v % kRing] + (i >> 3) * (kTile * 128) + row * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
          shared_writes_fence();
        }
        __syncwarp();
        if (warp_live) {
          // 32 logits at a time, and once more for the weights: to read tensor memory twice is cheaper than 128 registers
          uint32_t r[2][32];
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          tmem_load32(my_s, r[0]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            tmem_wait_loads();
            if (i < 3) tmem_load32(my_s + 32 * (i + 1), r[(i + 1) & 1]);
            const uint32_t on = i == 0 ? on0 : i == 1 ? on1 : i == 2 ? on2 : on3;
            uint32_t *y = r[i & 1];
            if (masked) {
#pragma unroll
              for (int j = 0; j < 32; ++j) y[j] = on >> j & 1 ? y[j] : 0xFF800000u;
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) top[j & 3] = fmaxf(top[j & 3], __uint_as_float(y[j]));
          }
          tmem_load32(my_s, r[0]);
          const float highest = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          // (m = -inf: nothing seen so far, the sums are 0 or not there yet)
          const bool raise = highest > m && (m == -INFINITY || (highest - m) * unit > kRaise);
          const float factor = raise ? exp2_fast((m - highest) * unit) : 1.f;
          if (raise) { l *= factor; m = highest; }
          if (__any_sync(~0u, raise) && t >= ahead) {
#pragma unroll
            for (int i = 0; i < D; i += 16) {
              uint32_t o[16];
              tmem_load16(my_o + i, o);
              tmem_wait_loads();
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * factor);
              tmem_store16(my_o + i, o);
            }
          }
          const float shift = m == -INFINITY ? 0.f : m * unit;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            tmem_wait_loads();
            if (i < 3) tmem_load32(my_s + 32 * (i + 1), r[(i + 1) & 1]);
            const uint32_t on = i == 0 ? on0 : i == 1 ? on1 : i == 2 ? on2 : on3;
            uint32_t *y = r[i & 1];
            if (masked) {
#pragma unroll
              for (int j = 0; j < 32; ++j) y[j] = on >> j & 1 ? y[j] : 0xFF800000u;
            }
            uint32_t packed[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float lo = exp2_fast(fmaf(__uint_as_float(y[j]), unit, -shift)), hi = exp2_fast(fmaf(__uint_as_float(y[j + 1]), unit, -shift));
              sum[j & 2] += lo;
              sum[(j & 2) + 1] += hi;
              packed[j / 2] = pack<T>(lo, hi);
            }
            tmem_store16(my_s + 16 * i, packed);                // over logits that have been read
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_wait_stores();
        }
        tmem_fence_before();
        barrier_arrive(sh.weights + s);
      }
      if (!ok || !(ok = wait(sh, &sh.done, items & 1))) {
        if (tid == 0) cache_fault(p.c, w.b, C2T_ST_INTERNAL);
        ok = false;
        break;
      }
      tmem_fence_after();
      turn += 2 * n;

      // what the block has of its rows: finished, or a part for the other launch to add up
      m = m == -INFINITY ? m : m * unit;
      float factor0 = 1.f, factor1 = 0.f;
      int column0 = 0, columns = D;
      if (!two) {
        sh.ml[s][row] = make_float2(m, l);
        barrier_arrive(&sh.halves);
        if (!(ok = wait(sh, &sh.halves, both_turn++ & 1))) {
          if (tid == 0) cache_fault(p.c, w.b, C2T_ST_INTERNAL);
          break;
        }
        const float2 e = sh.ml[0][row], o = sh.ml[1][row];          // (written again only after all threads' next queries)
        m = fmaxf(e.x, o.x);
        factor0 = e.x == -INFINITY ? 0.f : exp2_fast(e.x - m);
        factor1 = o.x == -INFINITY ? 0.f : exp2_fast(o.x - m);
        l = e.y * factor0 + o.y * factor1;
        columns = D / 2;
        column0 = s * columns;
      }
      const bool whole = x.k0 == 0 && x.k1 == w.tiles;
      __syncwarp();
      if (warp_live) {
        const float share = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        factor0 *= share;
        factor1 *= share;
        T *out = static_cast<T *>(p.a.out_dev) + w.b * p.a.out_seq_stride + node * p.a.out_token_stride + head * p.a.out_head_stride + column0;
        const long long part = (2ll * blockIdx.x + (x.k0 == 0 ? 1 : 0)) * kBlockRows + my_row;
        float *part_o = p.part_o + part * D + column0;
        bool odd = false;
        for (int i = 0; i < columns; i += 32) {
          uint32_t o[32], o1[32];
          tmem_load32((two ? my_o : tmem + 256 + ((uint32_t)(warp & 3) << 21)) + column0 + i, o);
          if (!two) tmem_load32(tmem + 384 + ((uint32_t)(warp & 3) << 21) + column0 + i, o1);
          tmem_wait_loads();
          float *v = reinterpret_cast<float *>(o);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            v[j] = factor0 == 0.f ? 0.f : v[j] * factor0;
            if (!two && factor1 != 0.f) v[j] += __uint_as_float(o1[j]) * factor1;
            odd |= !(fabsf(v[j]) < INFINITY);
          }
          if (live && whole) {
#pragma unroll
            for (int j = 0; j < 32; j += 8)
              *reinterpret_cast<uint4 *>(out + i + j) = make_uint4(pack<T>(v[j], v[j + 1]), pack<T>(v[j + 2], v[j + 3]), pack<T>(v[j + 4], v[j + 5]),
                                                                   pack<T>(v[j + 6], v[j + 7]));
          } else if (live) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4 *>(part_o + i + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          }
          __syncwarp();
        }
        if (live && (two || s == 0)) {
          if (!whole) p.part_ml[part] = make_float2(m, l);
          else if (p.a.lse_dev) p.a.lse_dev[((long long)w.b * p.a.max_queries + node) * p.a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
        // A row with a NaN or an infinity: from a value that the row does not see (0 times it is NaN), or its own.  Once more, key by key.
        for (uint32_t again = __ballot_sync(~0u, live && odd); again; again &= again - 1) {
          const int from = __ffs(again) - 1;
          const int i_ = __shfl_sync(~0u, node, from), h_ = __shfl_sync(~0u, head, from);
          const float m_ = __shfl_sync(~0u, m, from), share_ = __shfl_sync(~0u, share, from);
          constexpr int E = D / 32;
          float m2 = -INFINITY, l2 = 0.f, o2[E];
#pragma unroll
          for (int e = 0; e < E; ++e) o2[e] = 0.f;
          for (int t = x.k0; t < x.k1; ++t)
            attend_row<T, D>(p.c, p.a, see, w.b, i_, h_, w.key0(t), min(w.key0(t) + kTile, see.keys), m2, l2, o2);
          const float to = l2 == 0.f ? 0.f : exp2f(m2 - m_) * share_;
          const bool mine = two || (lane * E >= column0 && lane * E < column0 + columns);
          T *out_ = static_cast<T *>(p.a.out_dev) + w.b * p.a.out_seq_stride + i_ * p.a.out_token_stride + h_ * p.a.out_head_stride + lane * E;
          float *part_ = p.part_o + ((2ll * blockIdx.x + (x.k0 == 0 ? 1 : 0)) * kBlockRows + __shfl_sync(~0u, my_row, from)) * D + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (!mine) continue;
            if (whole) out_[e] = from_float<T>(to == 0.f ? 0.f : o2[e] * to);
            else part_[e] = to == 0.f ? 0.f : o2[e] * to;
          }
        }
      }
    }
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 8) tmem_free(tmem, kMathColumns);
}

// ---------------------------------------------------------------- parts of rows that several thread blocks read the keys of

constexpr int kJoinThreads = 128, kJoinRows = 8;                // rows of a thread block, two a warp

// Grid (G, parts of a block's rows).  The parts of a cut block of rows lie with thread blocks c0 .. c1: the first's second place, then the others' first.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) join_parts_kernel(Params p) {
  chain_enter();
  const int4 cut = p.cut[blockIdx.x];
  if (cut.x < 0) return;
  const Block w = block_of(p, cut.x);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = cut.w - cut.z + 1;
  constexpr int E = D / 32;
  for (int r = blockIdx.y * kJoinRows + warp; r < min((int)(blockIdx.y + 1) * kJoinRows, w.rows); r += kJoinThreads / 32) {
    auto place = [&](int i) { return (2ll * (cut.z + i) + (i == 0 ? 1 : 0)) * kBlockRows + r; };
    float m = -INFINITY;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, p.part_ml[place(i)].x);
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    float l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int i = 0; i < n; ++i) {
      const float2 ml = p.part_ml[place(i)];
      if (ml.x == -INFINITY && ml.y == 0.f) continue;
      const float f = exp2f(ml.x - m);
      const float *from = p.part_o + place(i) * D + lane * E;
      l += ml.y * f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += from[e] * f;
    }
    const int at = w.row0 + r, node = at / p.group, head = cut.y * p.group + at - node * p.group;
    T *out = static_cast<T *>(p.a.out_dev) + w.b * p.a.out_seq_stride + node * p.a.out_token_stride + head * p.a.out_head_stride + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = from_float<T>(l == 0.f ? 0.f : o[e] / l);
    if (p.a.lse_dev && lane == 0)
      p.a.lse_dev[((long long)w.b * p.a.max_queries + node) * p.a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
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

// ---------------------------------------------------------------- host side

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
  static const EncodeTiled fn = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(f);
  }();
  return fn;
}

// (elements, heads, places of a page, pages, layers); a box is 64 elements of one head of box_rows tokens.  What lies behind the pool reads as zeros.
bool encode_pool(const c2t_cache &c, void *pool, int box_rows, TensorMap *map) {
  static_assert(sizeof(TensorMap) == sizeof(CUtensorMap), "");
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  const cuuint64_t sizes[5] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.kv_heads, (cuuint64_t)c.page_size, (cuuint64_t)c.n_pages, (cuuint64_t)c.layers};
  const int64_t steps[4] = {c.head_stride, c.token_stride, c.page_stride, c.layer_stride};
  cuuint64_t bytes[4];
  for (int i = 0; i < 4; ++i) bytes[i] = sizes[i + 1] > 1 ? 2 * (cuuint64_t)steps[i] : 256;     // (of a size of 1 the step is never taken)
  const cuuint32_t box[5] = {64, 1, (cuuint32_t)box_rows, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return encode(reinterpret_cast<CUtensorMap *>(map), c.dtype == C2T_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, pool,
                sizes, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kMaxGrid = 256;               // workspaces are sized without asking the device: at most this many SMs are used

struct Workspace { size_t o, ml, cut, bytes; };

Workspace workspace_of(const c2t_cache &c) {
  Workspace w;
  w.o = 0;
  w.ml = w.o + sizeof(float) * 2 * kMaxGrid * kBlockRows * c.head_dim;
  w.cut = w.ml + sizeof(float2) * 2 * kMaxGrid * kBlockRows;
  w.bytes = w.cut + sizeof(int4) * kMaxGrid;
  return w;
}

template <typename T, int D>
cudaError_t launch_attention(const Params &p, const Maps &maps, int sms, cudaStream_t s) {
  constexpr size_t smem = sizeof(Shared<D>);
  static_assert(smem <= 232448, "shared memory of a thread block");
  cudaError_t e = cudaFuncSetAttribute(attend_tiles_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = launch_chained(attend_tiles_kernel<T, D>, dim3(sms), dim3(kThreads), smem, s, maps, p);
  if (e == cudaSuccess && p.split) {
    const long long rows = (long long)p.a.max_queries * p.group;
    const unsigned parts = (unsigned)((rows < kBlockRows ? rows : kBlockRows) + kJoinRows - 1) / kJoinRows;
    e = launch_chained(join_parts_kernel<T, D>, dim3(sms, parts), dim3(kJoinThreads), 0, s, p);
  }
  return e;
}

}  // namespace
}  // namespace c2t

using namespace c2t;

extern "C" {

size_t c2t_verify_attention_workspace_bytes(const c2t_cache *cache, int32_t q_heads, int32_t max_queries) {
  if (check_cache(cache) != C2T_OK || q_heads < 1 || q_heads % cache->kv_heads || max_queries < 1) return 0;
  return workspace_of(*cache).bytes;
}

int c2t_verify_attention(const c2t_cache *cache, const c2t_attention *attention, void *workspace_dev, size_t workspace_bytes, void *stream) {
  const int rc = check_attention(cache, attention);
  if (rc != C2T_OK) return rc;
  if (!workspace_dev) return C2T_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace_dev) & 255) return C2T_EALIGN;
  const Workspace at = workspace_of(*cache);
  if (workspace_bytes < at.bytes) return C2T_ERANGE;
  Params p;
  p.c = *cache;
  p.a = *attention;
  p.group = p.a.q_heads / p.c.kv_heads;
  const long long rows = (long long)p.a.max_queries * p.group, blocks = (rows + kBlockRows - 1) / kBlockRows;
  if (blocks * p.c.batch * p.c.kv_heads > 0x7FFFFFFF) return C2T_ERANGE;
  p.blocks_per_seq = (int)blocks;
  p.box_rows = p.c.page_size < kTile ? p.c.page_size : kTile;
  p.split = blocks * p.c.batch <= kMaxPairs;
  char *base = static_cast<char *>(workspace_dev);
  p.part_o = reinterpret_cast<float *>(base + at.o);
  p.part_ml = reinterpret_cast<float2 *>(base + at.ml);
  p.cut = reinterpret_cast<int4 *>(base + at.cut);
  Maps maps;
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || sms < 1 ||
      !encode_pool(p.c, p.c.k_dev, p.box_rows, &maps.k) || !encode_pool(p.c, p.c.v_dev, p.box_rows, &maps.v)) {
    cudaGetLastError();
    return C2T_ECUDA;
  }
  if (sms > kMaxGrid) sms = kMaxGrid;
  const bool bf16 = p.c.dtype == C2T_BF16;
  auto launch = p.c.head_dim == 64 ? (bf16 ? launch_attention<__nv_bfloat16, 64> : launch_attention<__half, 64>)
                                   : (bf16 ? launch_attention<__nv_bfloat16, 128> : launch_attention<__half, 128>);
  if (launch(p, maps, sms, (cudaStream_t)stream) != cudaSuccess) {
    cudaGetLastError();
    return C2T_ECUDA;
  }
  return C2T_OK;
}

}  // extern "C"
