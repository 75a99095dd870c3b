// Attention of a tree's nodes, a prompt's chunk or single tokens over the paged cache.  See include/c2t.h.
//
// Times in this file: one call among others, its inputs new from call to call; trees of 60 nodes; unless said otherwise 32 heads of 128, 8 key heads, bf16, pages
// of 16.  "A window" is trees of 16 sequences behind 20000 with a window of 1024 and 4 sinks, 64 heads of 64 over 8 key heads, f16, pages of 32; "a chunk" is
// 2 x 2048 tokens behind 6000.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include <cuda.h>

#include "cache_internal.h"
#include "tensor_core.cuh"

namespace c2t {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kMaxTokens = 0x40000000;      // of a slot; with the queries' number 32 bits hold every position
constexpr int kAnyKey = 0x60000000;         // behind every key of a slot

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
  s.prefix = min(max(a.prefix_len_dev[b], 0), kMaxTokens);      // (no page holds a position behind that)
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

// One warp, one row (b, i, h): the keys in [lo, hi) in order, with the running maximum m (in units of the exponent, base 2), the sum l of
// the weights and their sum over the values, D / 32 elements a lane.  The loads of kAtOnce keys go out together.
template <typename T, int D>
__device__ void attend_row(const c2t_cache &c, const c2t_attention &a, const Sight &see, int b, int i, int h, int lo, int hi, float &m, float &l,
                           float *o) {
  constexpr int E = D / 32, kAtOnce = D == 128 ? 8 : 2;         // (with more the kernel that calls this spills registers)
  using Elements = typename std::conditional<E == 4, uint2, uint32_t>::type;      // of a lane
  const int lane = threadIdx.x & 31;
  const T *q = static_cast<const T *>(a.q_dev) + b * a.q_seq_stride + i * a.q_token_stride + h * a.q_head_stride + lane * E;
  float qe[E];
#pragma unroll
  for (int e = 0; e < E; ++e) qe[e] = to_float(q[e]);
  const long long head = a.layer * c.layer_stride + (h / (a.q_heads / c.kv_heads)) * c.head_stride + lane * E;
  const int own = see.position(i), page_shift = __ffs(c.page_size) - 1;
  const float unit = a.scale * kLog2e;
#pragma unroll 1
  for (int p = lo; p < hi; p += kAtOnce) {
    bool seen[kAtOnce];
    long long at[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      seen[u] = p + u < hi && see.sees(i, own, p + u);
      const int page = seen[u] ? c.table_dev[(long long)b * c.max_pages + ((p + u) >> page_shift)] : 0;
      const bool there = page >= 0 && page < c.n_pages;
      if (!there) cache_fault(c, b, C2T_ST_BAD_PAGE);
      seen[u] &= there;
      at[u] = head + (there ? page : 0) * c.page_stride + ((p + u) & (c.page_size - 1)) * c.token_stride;       // (some place of the pool)
    }
    Elements x[kAtOnce];                    // of the keys, then of the values
    auto load = [&](const void *pool) {
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) x[u] = *reinterpret_cast<const Elements *>(static_cast<const T *>(pool) + at[u]);
    };
    float s[kAtOnce], top = m;
    load(c.k_dev);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      s[u] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s[u] += qe[e] * to_float(reinterpret_cast<const T *>(&x[u])[e]);
    }
    load(c.v_dev);
    for (int d = 16; d; d >>= 1)
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) s[u] += __shfl_xor_sync(~0u, s[u], d);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      s[u] = seen[u] ? s[u] * unit : -INFINITY;
      top = fmaxf(top, s[u]);
    }
    const float keep = m == top ? 1.f : exp2f(m - top);
    l *= keep;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= keep;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const float w = s[u] == -INFINITY ? 0.f : exp2f(s[u] - top);
      l += w;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += seen[u] ? w * to_float(reinterpret_cast<const T *>(&x[u])[e]) : 0.f;
    }
    m = top;
  }
}

// ---------------------------------------------------------------- the blocks of work
// The rows of a sequence and a key head are (new token, query head of the group), token-major; 256 of them, or what is left of a
// sequence, form a block of rows.  Its keys are cut into tiles of 128: those that hold the sinks, then those from the first key that a
// row's window can reach.  All of it follows from the lengths on the device.  A thread block per multiprocessor takes its share of all tiles: equal
// pieces of the blocks of rows where there are few of them, else an even deal, which cuts blocks wherever a share ends.  Rows of a cut block leave as parts
// for a second launch to add up.

constexpr int kTile = 128;                  // keys of a tile
constexpr int kRows = 128;                  // rows of one accumulator
constexpr int kBlockRows = 2 * kRows;

struct Params {
  c2t_cache c;
  c2t_attention a;
  int group, blocks_per_seq;                // query heads of a key head; blocks of max_queries * group rows
  uint32_t group_inverse;                   // 2^32 / group, rounded up (group > 1)
  int box_rows;                             // tokens of one copy: a page's, at most a tile's
  int folded;                               // 1: small pages' keys and values come with both halves of a head in one box (one accumulator's blocks)
  int copy_queries;                         // 1: queries come by copies of kQueryRows rows, whole tokens; 0: thread by thread
  int grid;                                 // thread blocks of the main launch: G
  int join_step;                            // without a common factor with the other launch's
  int split;                                // 1: blocks of rows may be cut; 0: whole ones
#ifdef C2T_DEBUG_BOUNDS
  int tries;                                // of a wait
#endif
  int least_tiles, more_tiles;              // of a piece, where all get equal ones, and how many more than an even deal they may have
  // Unfinished rows' sums over the values, two sets per thread block, and their maximum (scaled, base 2) and sum of weights.  Where a sequence has 32 rows at most
  // they lie side by side, the rows of a copy after those of the other, in a few megabytes: spread over places for 256 rows each, which is tens of megabytes, the
  // few rows of a single token behind 3000 others took 5 us longer to join.
  int part_rows, few_rows;                  // places of a set; rows of a sequence, or 0 if they may be more than 32
  float *part_o;                            // [2 G][D / 4][part_rows][4]
  float2 *part_ml;                          // [2 G][part_rows]
  int4 *cut;                                // [G]: {sequence, key head, first row, rows | first thread block << 9 | last << 17} of a cut block of rows
};

// row -> (new token, query head of the group); rows * group < 2^32, which makes the inverse exact
__device__ __forceinline__ int token_of(const Params &p, int row) { return p.group == 1 ? row : (int)__umulhi((uint32_t)row, p.group_inverse); }

struct Maps { TensorMap k, v, q, k_folded, v_folded; };
constexpr int kQueryRows = 32;              // rows of queries that one copy brings

struct Block {                              // with the tiles [k0, k1) of it that a thread block takes
  int b, head, row0, rows;                  // key head; first row; rows that are there (0: no block)
  int prefix, n, keys;                      // of the sequence, as in Sight
  int tiles, k0, k1;
  // The tiles' order: `bulk` of them side by side, from key bulk_key on, then the one at last_key, then the sinks'.  With a window of three tiles and more
  // the bulk begins with the second and the first comes behind it, else it is all of them: of the first tile and the sinks' a row may see a few keys only, and
  // its maximum would have to be raised behind them.  (With the sinks first and the others in ascending order a window takes 95 us, with the sinks last 90, so 76.)
  int bulk, bulk_key, last_key;
  __device__ __forceinline__ int key0(int t) const {
    const int behind = t - bulk;
    return behind < 0 ? bulk_key + t * kTile : behind > 0 || last_key < 0 ? (behind - (last_key < 0 ? 0 : 1)) * kTile : last_key;
  }
};

__device__ __forceinline__ Block block_of(const Params &p, int pair) {
  Block w;
  w.b = p.blocks_per_seq == 1 ? pair : pair / p.blocks_per_seq;
  w.row0 = (pair - w.b * p.blocks_per_seq) * kBlockRows;
  const Sight s = sight_of(p.c, p.a, w.b);
  w.prefix = s.prefix; w.n = s.n; w.keys = s.keys;
  w.rows = min(max(s.n * p.group - w.row0, 0), kBlockRows);
  w.tiles = w.head = w.k0 = w.k1 = w.bulk = w.bulk_key = 0;
  w.last_key = -1;
  if (w.rows == 0) return w;
  const int first_token = token_of(p, w.row0), last = token_of(p, w.row0 + w.rows - 1);
  const int end = s.bits ? s.keys : min(s.keys, s.prefix + last + 1);
  const int end_tile = (end + kTile - 1) / kTile;
  int sinks = 0, first = 0;                 // tiles that hold sinks; the first one that a row's window can reach
  if (s.window > 0) {
    const int lowest = s.prefix + (s.positions ? 0 : first_token);              // the lowest position of a row
    first = min(max(lowest - s.window + 1, 0) / kTile, max(end_tile - 1, 0));
    sinks = min((min(s.sinks, end) + kTile - 1) / kTile, first);
  }
  w.bulk = max(end_tile - first, 1);                                            // (rows that see nothing are written too)
  w.bulk_key = first * kTile;
  w.tiles = sinks + w.bulk;
  if (s.window > 0 && w.bulk > 2) {
    w.last_key = w.bulk_key;
    w.bulk_key += kTile;
    --w.bulk;
  }
  return w;
}

__device__ __forceinline__ Sight sight_of(const Params &p, const Block &w) {
  Sight s;
  s.prefix = w.prefix; s.n = w.n; s.keys = w.keys;
  s.window = p.a.window;
  s.sinks = p.a.sinks;
  s.words = p.a.mask_words;
  s.bits = p.a.mask_bits_dev ? p.a.mask_bits_dev + (long long)w.b * p.a.max_queries * p.a.mask_words : nullptr;
  s.positions = p.a.position_ids_dev ? p.a.position_ids_dev + (long long)w.b * p.a.max_queries : nullptr;
  return s;
}

// An even deal of `total` tiles to `used` thread blocks: the first `more` of them get one more than the others.
struct Deal {
  int total, used, each, more;
  __device__ __forceinline__ Deal(int total_, int grid) : total(total_) {
    used = min(max(total, 1), grid);        // (none without a tile)
    each = total / used;
    more = total - each * used;
  }
  __device__ __forceinline__ int begin(int c) const { return c >= used ? total : c * each + min(c, more); }
  __device__ __forceinline__ int owner(int x) const {           // of tile x
    const int wide = more * (each + 1);
    return x < wide ? x / (each + 1) : more + (x - wide) / each;
  }
};

// ---------------------------------------------------------------- the kernel
// Two accumulators of 128 rows, each with a group of four warps that takes its logits through the softmax.  A block of more than 128
// rows has its halves in them, which read the same tiles; a smaller one goes over its tiles with both, the even ones and the odd ones, and
// adds up at the end.  Either way one group's exponentials run while the tensor cores work for the other.
//   warps 0-3, 4-7   a thread per row: S from tensor memory, its maximum, the weights back as 16-bit numbers
//   warp 8    issues the products: logits S = Q K^T (both from shared memory), and O += P V with P, the weights, in tensor memory in S's place
//   warp 9    copies the tiles of keys and values, a box per page and 64 elements of a head, into a ring of buffers
//   warp 10   walks through the thread block's share and describes the next blocks of rows to the others
// The running maximum m is only raised when a row's new one is more than 2^9 (bf16: 2^40) in weight above it: then O and the sum are rescaled.  A weight is
// 2^kLift at m, so at most 2^15, which f16 holds, or 2^40, of which 32 bits hold any sum.  Of f16, whose numbers end at 2^-24, the lift keeps the weights of
// long flat tails: a weight is off by half a step or 2^-31 of the largest, whichever is more, so that 2^20 keys add up to half a step (without it 2^14 keys).
// Every further bit of it asks more rows for a second pass: a window takes 74.5 us with 0, 75.7 with 6, 78 with 8.
// Up to 32 (64) rows lie in the accumulator four times (twice), and each copy takes a quarter (half) of a tile's keys, with weights of 0
// for the others: all warps have work then, and a tile's softmax, which is what such a block waits for, a quarter of the steps.

constexpr int kSoftmaxThreads = 256, kThreads = 352;
constexpr int kMathColumns = 512;           // of tensor memory: S 2 x 128, O 2 x D; P in the place of S, with heads of 64 in columns of its own
template <typename T> constexpr float kLift = std::is_same<T, __half>::value ? 6.f : 0.f;
template <typename T> constexpr float kRaise = std::is_same<T, __half>::value ? 15.f - kLift<T> : 40.f;
// Of 16 powers of two, 2 kProducts are products and sums instead of the special-function unit's.  With 0, 1 and 2: trees of 8 sequences behind 2048
// 39.5, 38.7, 39.0 us; of one behind 16000, 64 heads, 53.4, 53.8, 54.8; 64 sequences' tokens behind 4096 in pages of 128 154 each; a chunk 508, 524, 536.
constexpr int kProducts = 1;
constexpr int kTries = 1 << 20;             // of a wait, 3900 cycles each: after two seconds the block gives up (but see goes_on)

template <int D> __device__ __forceinline__ constexpr int weights_at(int s) { return D == 64 ? 384 + s * 64 : s * kTile; }

template <int D> struct Ring { static constexpr int bytes = kTile * D * 2, n = D == 128 ? 5 : 10; };

constexpr int kBlocks = 4;                  // descriptions ahead
constexpr int kReaders = 10;                // warps that read them

template <int D>
struct alignas(1024) Shared {
  unsigned char q[2][kRows * D * 2];        // 64 elements of all rows after the other 64; at a block's end its sums over the values
  union {
    unsigned char ring[Ring<D>::n][Ring<D>::bytes];
    long long before[C2T_MAX_BATCH + 1];    // while the work is dealt out: of the pairs before, tiles and (upper half) how many have any
  };
  float2 ml[2][kRows];
  uint64_t full[Ring<D>::n], empty[Ring<D>::n];
  uint64_t logits[2], weights[2], done, queries, queries_free, meet, described[kBlocks], read[kBlocks];
  Block block[kBlocks];
  uint32_t tmem;
  int gave_up;
  int redoing;                              // warps that do rows once more
  uint32_t redo_ended;                      // when the last one was through; 0: none so far
#ifdef C2T_DEBUG_BOUNDS
  int tries;
#endif
  uint32_t odd[8];
  long long warp_sum[kThreads / 32];
  int left, pair, head, k0, c0, c1, long_ones;
};

constexpr int kMaxPairs = C2T_MAX_BATCH;    // for an even deal

template <int D>
__device__ __forceinline__ int tries_of(const Shared<D> &sh) {
#ifdef C2T_DEBUG_BOUNDS
  return sh.tries;
#else
  return kTries;
#endif
}

__device__ __forceinline__ uint32_t milliseconds() {            // of 2^20 ns; never 0
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return (uint32_t)(t >> 20) | 1;
}

// A wait has had its tries: it goes on while a warp does rows once more, which takes as long as their keys are many, and for two seconds behind that.  (Asked
// only then: with the question in a wait's loop a chunk took 531 us instead of 517.)
template <int D>
__device__ __noinline__ bool goes_on(Shared<D> &sh) {
  if (tries_of(sh) != kTries) return false;
  if (*(volatile int *)&sh.redoing > 0) return true;
  const uint32_t ended = *(volatile uint32_t *)&sh.redo_ended;                  // (written before the last one stops counting)
  return ended != 0 && milliseconds() - ended < 2000;
}

template <int D>
__device__ __forceinline__ bool wait(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
  for (int i = 0; i < tries_of(sh) || goes_on(sh); ++i) {
    if (barrier_try(bar, parity)) return true;
    if ((i & 63) == 63 && *(volatile int *)&sh.gave_up) return false;
  }
  sh.gave_up = 1;
  return false;
}

// The same for a whole warp, whose lanes ask together and go on together.  (Lanes that ask each for itself come back up to 750 cycles apart.)  The loop
// ends on a vote, which all lanes are known to share: the tensor-memory instructions behind it must be reached by the whole warp at once.
template <int D>
__device__ __forceinline__ bool warp_wait(Shared<D> &sh, uint64_t *bar, uint32_t parity) {
  for (int i = 0; i < tries_of(sh) || __any_sync(~0u, goes_on(sh)); ++i) {
    if (__all_sync(~0u, barrier_try(bar, parity))) return true;
    if ((i & 63) == 63 && __any_sync(~0u, *(volatile int *)&sh.gave_up)) return false;
  }
  sh.gave_up = 1;
  return false;
}

// What is still on its way, to shared or tensor memory that is about to be let go.
__device__ __forceinline__ void let_arrive(uint64_t *bar, uint32_t parity) {
  for (int tries = 0; tries < kTries && !barrier_try(bar, parity); ++tries) {}
}

// A buffer of the ring and the parity of its barriers.  The copies' order: K_0 .. K_{ahead-1}, then V_t, K_{t+ahead} in turn.
template <int n>
struct Cursor {
  int at;
  uint32_t parity;
  __device__ __forceinline__ void step(int by) {                // by < n
    at += by;
    if (at >= n) { at -= n; parity ^= 1; }
  }
};
__device__ __forceinline__ int step_of_keys(int t, int ahead) { return t + 1 < ahead ? 1 : 2; }              // from K_t to K_{t+1}
__device__ __forceinline__ int step_of_values(int t, int n, int ahead) { return t + ahead < n ? 2 : 1; }     // from V_t to V_{t+1}

// Of the box that holds a sequence's last key only the rows up to that key are copied, to the box's end; the rows before them read as zeros, or as earlier
// keys.  (What lies behind the last key in its page may be anything, and 0 times anything need not be 0.)  With `there` keys of the sequence from
// a tile's first on: the column at which that box begins, kTile if the tile has none; and by how many columns its keys are further right.
__device__ __forceinline__ int last_box(int there, int box_rows) { return there >= kTile || there <= 0 ? kTile : (there - 1) & -box_rows; }
__device__ __forceinline__ int shift_of_last_box(int there, int box_rows) {
  return there >= kTile || there <= 0 ? 0 : last_box(there, box_rows) + box_rows - there;
}

// rows of one of the copies of a block's rows: four of up to 32, two of up to 64
__device__ __forceinline__ int rows_of_copy(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : kRows; }

// Do the columns of such a block's tiles take their keys from folded pages of 16, 8 of every page after the other 8?
__device__ __forceinline__ bool is_woven(const Params &p, int rows) { return p.folded && rows <= kRows && p.box_rows == 16; }

// bits 0..31: columns c < n
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Which of the 32 keys from `key` row i sees.  (key may be below 0 where a last box reaches to the left of the first key; windows, sinks and positions may be
// any numbers: bounds are brought among the keys before they are compared, so that nothing passes 32 bits.)
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
    const uint32_t sink = low_bits(min(s.sinks, kAnyKey) - key);
    uint32_t near = ~low_bits(min(max(own - s.window + 1, 0), kAnyKey) - key);
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

// x, y = x * unit + shift, y * unit + shift and a, b += x, y, two in one instruction
__device__ __forceinline__ void scale_add2(float &x, float &y, float unit, float shift) {
  asm("{\n\t.reg .b64 v, u, s;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 u, {%2, %2};\n\tmov.b64 s, {%3, %3};\n\tfma.rn.f32x2 v, v, u, s;\n\tmov.b64 {%0, %1}, v;\n\t}"
      : "+f"(x), "+f"(y) : "f"(unit), "f"(shift));
}
__device__ __forceinline__ void add2(float &a, float &b, float x, float y) {
  asm("{\n\t.reg .b64 v, w;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %3};\n\tadd.rn.f32x2 v, v, w;\n\tmov.b64 {%0, %1}, v;\n\t}"
      : "+f"(a), "+f"(b) : "f"(x), "f"(y));
}

// 2^x and 2^y by products and sums: x = n + f with n the nearest whole number (added to 1.5 * 2^23 it stands in the low bits), 2^f by a polynomial of
// degree 5 on [-1/2, 1/2] (equal ripple, 1.6e-7 relative with its rounding, 1 at 0), n added to the exponent.  Below -127, -inf included, it is 0.
__device__ __forceinline__ void exp2_products(float &x, float &y) {
  x = fmaxf(x, -127.f);
  y = fmaxf(y, -127.f);
  float nx = x, ny = y, px, py;
  asm("{\n\t.reg .b64 v, n, f, q, c;\n\t"
      "mov.b64 v, {%4, %5};\n\t"
      "mov.b64 c, {%6, %6};\n\tadd.rn.f32x2 n, v, c;\n\tmov.b64 {%0, %1}, n;\n\t"
      "mov.b64 c, {%7, %7};\n\tadd.rn.f32x2 n, n, c;\n\t"
      "mov.b64 c, {%8, %8};\n\tfma.rn.f32x2 f, n, c, v;\n\t"
      "mov.b64 q, {%9, %9};\n\tmov.b64 c, {%10, %10};\n\tfma.rn.f32x2 q, q, f, c;\n\t"
      "mov.b64 c, {%11, %11};\n\tfma.rn.f32x2 q, q, f, c;\n\t"
      "mov.b64 c, {%12, %12};\n\tfma.rn.f32x2 q, q, f, c;\n\t"
      "mov.b64 c, {%13, %13};\n\tfma.rn.f32x2 q, q, f, c;\n\t"
      "mov.b64 c, {%14, %14};\n\tfma.rn.f32x2 q, q, f, c;\n\t"
      "mov.b64 {%2, %3}, q;\n\t}"
      : "=f"(nx), "=f"(ny), "=f"(px), "=f"(py)
      : "f"(x), "f"(y), "f"(12582912.f), "f"(-12582912.f), "f"(-1.f), "f"(0.0013274633f), "f"(0.009671962f), "f"(0.055506784f), "f"(0.24022235f),
        "f"(0.69314706f), "f"(1.f));
  x = __int_as_float(__float_as_int(px) + (__float_as_int(nx) << 23));
  y = __int_as_float(__float_as_int(py) + (__float_as_int(ny) << 23));
}

// the largest; NaN if any is
__device__ __forceinline__ float largest(float a, float b, float c) {
  float x;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(x) : "f"(a), "f"(b), "f"(c));
  return x;
}
__device__ __forceinline__ float larger(float a, float b) {
  float x;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(a), "f"(b));
  return x;
}

// the largest of a, |b| and |c|, for a >= 0; NaN if any is
__device__ __forceinline__ float largest_size(float a, float b, float c) {
  float x;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(x) : "f"(a), "f"(b), "f"(c));
  return x;
}

// logits whose bit is not set become -inf
__device__ __forceinline__ void mask32(bool masked, uint32_t on, uint32_t *y) {
  if (!masked) return;
#pragma unroll
  for (int j = 0; j < 32; ++j) y[j] = on >> j & 1 ? y[j] : 0xFF800000u;
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

// A row's softmax over `words` * 32 of a tile's logits, from column `first` on.  Once a row has a maximum the weights are computed with it at once, and their
// own maximum is taken on the way: it hardly ever asks for another one, and a tile's softmax, which the next products of its accumulator wait
// for, is one pass.  Where the weights go where the logits lie they are held back till then.
template <typename T, int D>
__device__ __forceinline__ void softmax_tile(uint32_t my_s, uint32_t my_w, uint32_t my_o, int first, int words, bool masked, uint32_t on0, uint32_t on1, uint32_t on2,
                                             uint32_t on3, float unit, bool has_sums, float &m, float &l) {
  constexpr bool kHeld = D == 128;          // the weights go where the logits lie
  uint32_t y[32], packed[kHeld ? kTile / 2 : 16];
  float sum[4];
  int again = __any_sync(~0u, m == -INFINITY);
  for (;;) {
    asm volatile("" : "+r"(again));         // (one copy of the code for both)
    if (again) {
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
      for (int i = 0; i < words; ++i) {
        __syncwarp();
        tmem_load32(my_s + first + 32 * i, y);
        tmem_wait_loads();
        mask32(masked, i == 0 ? on0 : i == 1 ? on1 : i == 2 ? on2 : on3, y);
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          top[0] = largest(top[0], __uint_as_float(y[j]), __uint_as_float(y[j + 1]));
          top[1] = largest(top[1], __uint_as_float(y[j + 2]), __uint_as_float(y[j + 3]));
        }
      }
      const float highest = larger(top[0], top[1]);
      // (m = -inf: nothing seen so far, the sums are 0 or not there yet)
      const bool raise = highest > m && (m == -INFINITY || (highest - m) * unit > kRaise<T>);
      const float factor = raise ? exp2_fast((m - highest) * unit) : 1.f;
      if (raise) { l *= factor; m = highest; }
      if (__any_sync(~0u, raise) && has_sums) {
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
          tmem_load32(my_o + i, y);
          tmem_wait_loads();
#pragma unroll
          for (int j = 0; j < 32; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * factor);
          tmem_store32(my_o + i, y);
        }
      }
    }
    const float shift = m == -INFINITY ? 0.f : kLift<T> - m * unit;
    float top[2] = {-INFINITY, -INFINITY};
    sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
    __syncwarp();
    auto word = [&](int i, uint32_t *packed) {                  // 32 logits
      tmem_load32(my_s + first + 32 * i, y);
      tmem_wait_loads();
      mask32(masked, i == 0 ? on0 : i == 1 ? on1 : i == 2 ? on2 : on3, y);
#pragma unroll
      for (int j = 0; j < 32; j += 4) {
        float a = __uint_as_float(y[j]), b = __uint_as_float(y[j + 1]), c = __uint_as_float(y[j + 2]), d = __uint_as_float(y[j + 3]);
        top[0] = largest(top[0], a, b);
        top[1] = largest(top[1], c, d);
        scale_add2(a, b, unit, shift);
        scale_add2(c, d, unit, shift);
        a = exp2_fast(a); b = exp2_fast(b);
        if (((j / 4) & 3) < kProducts) exp2_products(c, d);
        else { c = exp2_fast(c); d = exp2_fast(d); }
        add2(sum[0], sum[1], a, b);
        add2(sum[2], sum[3], c, d);
        packed[j / 2] = pack<T>(a, b);
        packed[j / 2 + 1] = pack<T>(c, d);
      }
    };
    if (kHeld) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < words) {
          word(i, packed + 16 * i);
        } else {                            // of the other copies
#pragma unroll
          for (int j = 0; j < 16; ++j) packed[16 * i + j] = 0;
        }
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        if (i < words) {
          word(i, packed);
        } else {
#pragma unroll
          for (int j = 0; j < 16; ++j) packed[j] = 0;
        }
        __syncwarp();
        tmem_store16(my_w + ((first + 32 * i) & (kTile - 1)) / 2, packed);
      }
    }
    const float highest = larger(top[0], top[1]);
    if (!(highest < INFINITY)) l = NAN;     // (a logit that is none makes the row NaN, whichever way its power is taken)
    if (again) break;
    again = __any_sync(~0u, (highest - m) * unit > kRaise<T>);
    if (!again) break;
  }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  __syncwarp();
  if (kHeld)
#pragma unroll
    for (int i = 0; i < 4; ++i) tmem_store16(my_w + ((first + 32 * i) & (kTile - 1)) / 2, packed + 16 * i);
}

// The block's rows [0, rows) of queries, `copies` times, swizzled; 256 threads.  All loads go out before `ready` is asked for, which says that the memory is free.
template <typename T, int D, typename Ready>
__device__ __forceinline__ bool load_queries(const Params &p, const Block &w, unsigned char *q, int copy_rows, Ready ready) {
  constexpr int kPieces = D / 8, kPass = kSoftmaxThreads / kPieces, kPasses = kRows / kPass;       // 16 (32) rows a pass
  const int piece = threadIdx.x % kPieces, row = threadIdx.x / kPieces;
  const T *from = static_cast<const T *>(p.a.q_dev) + w.b * p.a.q_seq_stride + piece * 8;
  uint4 x[kPasses];
#pragma unroll 1
  for (int half = 0; half < (w.rows > kRows ? 2 : 1); ++half) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int r = half * kRows + ((row + i * kPass) & (copy_rows - 1));
      x[i] = make_uint4(0, 0, 0, 0);
      if (r < w.rows) {
        const int at = w.row0 + r, node = token_of(p, at), h = w.head * p.group + at - node * p.group;
        x[i] = *reinterpret_cast<const uint4 *>(from + node * p.a.q_token_stride + h * p.a.q_head_stride);
      }
    }
    if (half == 0 && !ready()) return false;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const int place = row + i * kPass;
      *reinterpret_cast<uint4 *>(q + half * (kRows * D * 2) + (piece >> 3) * (kRows * 128) + place * 128 + (((piece & 7) ^ (place & 7)) << 4)) = x[i];
    }
  }
  return true;
}

// A row with a NaN or an infinity: from a value that it does not see (0 times it is NaN), or its own.  The row r of the block once more, key by key, by one
// warp: the keys that lie in the columns [first, first + size) of each tile, `columns` elements from column0 on; finished, or relative to the
// maximum of the part that it belongs to.  Out of line: hardly ever called.
template <typename T, int D>
__device__ __noinline__ void once_more(const Params &p, const Block &w, int r, int first, int size, int column0, int columns, bool finish, float part_m,
                                       float *to_part) {
  const int lane = threadIdx.x & 31, i = token_of(p, w.row0 + r), h = w.head * p.group + w.row0 + r - i * p.group;
  const Sight see = sight_of(p, w);
  constexpr int E = D / 32;
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 1
  for (int t = w.k0; t < w.k1; ++t) {
    const int key = w.key0(t), last = last_box(w.keys - key, p.box_rows), over = shift_of_last_box(w.keys - key, p.box_rows);
    const bool woven = is_woven(p, w.rows) && size < kTile;
#pragma unroll 1
    for (int c = first; c < first + size; c += woven ? 8 : size) {              // columns whose keys are side by side
      const int slot = woven ? (c & 63) / 8 * 16 + (c >> 6) * 8 : c, n = woven ? 8 : size;
#pragma unroll 1
      for (int shifted = 0; shifted < 2; ++shifted) {
        const int lo = shifted ? max(slot - over, last) : slot, hi = shifted ? slot + n - over : min(slot + n, last);
        if (!shifted || last < kTile) attend_row<T, D>(p.c, p.a, see, w.b, i, h, key + lo, min(key + hi, w.keys), m, l, o);
      }
    }
  }
  const float f = l == 0.f ? 0.f : finish ? 1.f / l : exp2f(m - part_m);
  T *out = static_cast<T *>(p.a.out_dev) + w.b * p.a.out_seq_stride + i * p.a.out_token_stride + h * p.a.out_head_stride;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = lane * E + e;
    const float x = f == 0.f ? 0.f : o[e] * f;
    if (d < column0 || d >= column0 + columns) continue;
    if (finish) out[d] = from_float<T>(x);
    else to_part[(d >> 2) * (p.part_rows * 4) + (d & 3)] = x;
  }
  __syncwarp();
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) attend_tiles_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  constexpr int kRing = Ring<D>::n;
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  extern __shared__ __align__(1024) unsigned char raw[];       // (the tiles' swizzle goes by the address)
  Shared<D> &sh = *reinterpret_cast<Shared<D> *>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_pairs = p.c.batch * p.blocks_per_seq, G = gridDim.x;

  if (warp == 8) {
    tmem_alloc(&sh.tmem, kMathColumns);
    chain_release();                        // (after it: a successor's blocks could take the tensor memory and wait for this one)
  }
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) { barrier_init(sh.full + i, 1); barrier_init(sh.empty + i, 1); }
    for (int s = 0; s < 2; ++s) { barrier_init(sh.logits + s, 1); barrier_init(sh.weights + s, kRows); }
    for (int i = 0; i < kBlocks; ++i) { barrier_init(sh.described + i, 1); barrier_init(sh.read + i, kReaders); }
    barrier_init(&sh.done, 1);
    barrier_init(&sh.queries, p.copy_queries ? 1 : kSoftmaxThreads);
    barrier_init(&sh.queries_free, kSoftmaxThreads);
    barrier_init(&sh.meet, kSoftmaxThreads);
    barrier_init_fence();
    sh.gave_up = sh.redoing = 0;
    sh.redo_ended = 0;
#ifdef C2T_DEBUG_BOUNDS
    sh.tries = p.tries;
#endif
    sh.left = sh.pair = sh.head = sh.k0 = 0;
    sh.c0 = -1;
    sh.long_ones = 0;
    tensor_map_prefetch(&maps.k);
    tensor_map_prefetch(&maps.v);
    if (p.copy_queries) tensor_map_prefetch(&maps.q);
  }
  chain_wait();

  // ---- the thread block's share of the tiles
  __syncthreads();
  if (p.split) {
    long long carry = 0;
#pragma unroll 1
    for (int base = 0; base < n_pairs; base += kThreads) {
      const int pair = base + tid, tiles = pair < n_pairs ? block_of(p, pair).tiles : 0;
      const long long mine = (tiles > 0 ? 1ll << 32 : 0) + tiles;
      if (tiles > p.least_tiles) sh.long_ones = 1;
      long long x = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
      }
      if (lane == 31) sh.warp_sum[warp] = x;
      __syncthreads();
      long long earlier = 0, all = 0;
#pragma unroll
      for (int v = 0; v < kThreads / 32; ++v) {
        const long long s = sh.warp_sum[v];
        earlier += v < warp ? s : 0;
        all += s;
      }
      if (pair < n_pairs) sh.before[pair] = carry + earlier + x - mine;
      carry += all;
      __syncthreads();
    }
    if (tid == 0) sh.before[n_pairs] = carry;
    __syncthreads();
    auto tiles_of = [&](int pair) { return (int)sh.before[pair + 1] - (int)sh.before[pair]; };
    const int H = p.c.kv_heads, total = (int)carry * H, blocks = (int)(carry >> 32) * H;
    // Where every block of rows finds a thread block: equal pieces of each, of so few tiles that every piece finds one.  Each warp tries a number of tiles.
    int piece = 0;
    if (blocks <= G && !sh.long_ones) {
      piece = p.least_tiles;                // (no block of rows has more)
    } else if (blocks <= G) {
      const int least = max((total + G - 1) / G, p.least_tiles);
      int pieces = 0;
      if (warp <= p.more_tiles)
#pragma unroll 1
        for (int pair = lane; pair < n_pairs; pair += 32) pieces += (tiles_of(pair) + least + warp - 1) / (least + warp);
      pieces = __reduce_add_sync(~0u, pieces) * H;
      if (lane == 0) sh.warp_sum[warp] = pieces;
      __syncthreads();
#pragma unroll 1
      for (int w = p.more_tiles; w >= 0; --w)
        if (sh.warp_sum[w] <= G) piece = least + w;
    }
    // c0, c1: of a block of rows that the thread block before this one began, the first and the last thread block
    auto found = [&](int pair, int head, int k0, int left, int c0, int c1) {    // (by one thread, or none)
      sh.pair = pair; sh.head = head; sh.k0 = k0; sh.left = left; sh.c0 = c0; sh.c1 = c1;
    };
    const int me = blockIdx.x;
    if (piece > 0) {
      if (warp == 0) {
        int before = 0;                     // pieces
#pragma unroll 1
        for (int base = 0; base < n_pairs && before <= me; base += 32) {
          const int pair = base + lane, tiles = pair < n_pairs ? tiles_of(pair) : 0, each = (tiles + piece - 1) / piece;          // of a head
          int x = each * H;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(~0u, x, d);
            if (lane >= d) x += y;
          }
          const int first = before + x - each * H;
          if (me >= first && me < before + x) {
            const int head = (me - first) / each, at = me - first - head * each;
            const int k0 = (unsigned)at * tiles / each;         // (256 thread blocks, 2^23 tiles)
            found(pair, head, k0, (int)((at + 1u) * tiles / each) - k0, at == 1 ? me - 1 : -1, me + each - 2);
          }
          before += __shfl_sync(~0u, x, 31);
        }
      }
    } else {
      const Deal deal(total, G);
      const int begin = deal.begin(me), left = deal.begin(me + 1) - begin;
#pragma unroll 1
      for (int pair = tid; pair < n_pairs && left > 0; pair += kThreads) {
        const int each = tiles_of(pair), first = (int)sh.before[pair] * H;
        if (begin < first || begin >= first + each * H) continue;
        const int head = (begin - first) / each, k0 = begin - first - head * each;
        const bool second = k0 > 0 && deal.owner(begin - k0) == me - 1;
        found(pair, head, k0, left, second ? me - 1 : -1, second ? deal.owner(begin - k0 + each - 1) : 0);
      }
    }
  }
  shared_writes_fence();                    // (the ring's copies come where the sums were)
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = sh.tmem;

  // the i-th block of rows of the share; rows = 0 behind the last
  auto described = [&](int i) {
    if (!warp_wait(sh, sh.described + i % kBlocks, i / kBlocks & 1)) return false;
#ifdef C2T_DEBUG_BOUNDS
    const Block &w = sh.block[i % kBlocks];
    if (w.rows != 0 && (w.b < 0 || w.b >= p.c.batch || w.head < 0 || w.head >= p.c.kv_heads || w.row0 < 0 || w.rows < 0 || w.rows > kBlockRows || w.k0 < 0 ||
                        w.k1 <= w.k0 || w.k1 > w.tiles || w.n > p.a.max_queries || w.row0 + w.rows > w.n * p.group)) {
      sh.gave_up = 1;
      return false;
    }
#endif
    return true;
  };
  auto block_read = [&](int i) {
    __syncwarp();
    if (lane == 0) barrier_arrive(sh.read + i % kBlocks);
  };

  if (warp == 10) {
    // ------------------------------------------------------------ the walk
    if (lane == 0) {
      int left = sh.left, pair = p.split ? sh.pair : 0, head = p.split ? sh.head : blockIdx.x, k0 = p.split ? sh.k0 : 0, known = -1;
      Block w;
      int copied = 0;                       // blocks whose queries were asked for
      for (int i = 0;; ++i) {
        bool more = false;
#pragma unroll 1
        while ((!p.split || left > 0) && !more) {
          while (head >= p.c.kv_heads) { head -= p.c.kv_heads; ++pair; }
          if (pair >= n_pairs) break;
          if (pair != known) w = block_of(p, pair);
          known = pair;
          more = w.tiles > 0;
          w.head = head;
          if (p.split && !more) head = p.c.kv_heads;            // to the next pair
          else head += p.split ? 1 : G;
        }
        if (i == 0 && p.split) p.cut[blockIdx.x] = more && sh.c0 >= 0 ? make_int4(w.b, w.head, w.row0, w.rows | sh.c0 << 9 | sh.c1 << 17) : make_int4(0, 0, 0, 0);
        w.k0 = k0;
        w.k1 = p.split ? min(w.tiles, k0 + left) : w.tiles;
        left -= w.k1 - k0;
        k0 = 0;
        if (!wait(sh, sh.read + i % kBlocks, (i / kBlocks & 1) ^ 1)) break;
        if (!more) w.rows = 0;
        sh.block[i % kBlocks] = w;
        barrier_arrive(sh.described + i % kBlocks);
        if (!more) break;
        if (p.copy_queries) {               // once the last block's sums are out of their memory
          if (i > 0 && !wait(sh, &sh.queries_free, (i - 1) & 1)) break;
          const bool two = w.rows > kRows;
          const int boxes = (two ? 2 : 1) * kRows / kQueryRows, copy_rows = rows_of_copy(w.rows);
          barrier_expect(&sh.queries, boxes * kQueryRows * D * 2);
          ++copied;
#pragma unroll 1
          for (int x = 0; x < boxes; ++x) {
            const int row = two ? x * kQueryRows : x * kQueryRows & (copy_rows - 1);
#pragma unroll 1
            for (int h = 0; h < D / 64; ++h)
              copy_box(shared_address(sh.q[0]) + (x >> 2) * (kRows * D * 2) + h * (kRows * 128) + (x & 3) * (kQueryRows * 128), &maps.q, &sh.queries, h * 64,
                       w.head * p.group, token_of(p, w.row0 + row), w.b);
          }
        }
      }
      if (copied > 0) let_arrive(&sh.queries, (copied - 1) & 1);                // (nothing may arrive in a block's memory that has ended, whoever gave up)
    }
    __syncwarp();
  } else if (warp == 9) {
    // ------------------------------------------------------------ copies
    const int parts = kTile / p.box_rows, box_bytes = p.box_rows * 128;
    const int half = lane / parts, part = lane % parts, page_shift = __ffs(p.c.page_size) - 1;
    Cursor<kRing> to = {0, 0};
    int filled = 0;
    bool ok = true;
    for (int item = 0;; ++item) {
      if (!(ok = described(item))) break;
      const Block w = sh.block[item % kBlocks];
      block_read(item);
      if (w.rows == 0) break;
      const int n = w.k1 - w.k0, ahead = w.rows > kRows ? 1 : 2, lead = min(n, ahead);
      const bool folded = p.folded && w.rows <= kRows;
      const int boxes = folded ? parts : parts * (D / 64);
      if (w.head == 0 && w.k0 == 0 && w.row0 == 0 && lane == 0 && w.keys < w.prefix + w.n) cache_fault(p.c, w.b, C2T_ST_BAD_PAGE);
      const int32_t *table = p.c.table_dev + (long long)w.b * p.c.max_pages;
      // the next copy of the order and the page that this lane copies for it (behind the pool: zeros)
      auto page_of = [&](int i, bool &values, int &key) {
        values = i >= lead && (i >= 2 * n - lead || ((i - ahead) & 1) == 0);
        const int t = values ? (i >= 2 * n - lead ? i - n : (i - ahead) >> 1) : (i < ahead ? i : (i + ahead - 1) >> 1);
        key = w.key0(w.k0 + t) + part * p.box_rows;
        if (i >= 2 * n || lane >= boxes || key >= w.keys) return p.c.n_pages;
        return (int)table[key >> page_shift];
      };
      bool values, next_values;
      int key, next_key, page = page_of(0, values, key);
      for (int i = 0; i < 2 * n; ++i) {
        const int next = page_of(i + 1, next_values, next_key);
        ok = warp_wait(sh, sh.empty + to.at, to.parity ^ 1);
        if (!ok) break;
        if (lane == 0) barrier_expect(sh.full + to.at, Ring<D>::bytes);
        if (page < 0 || page > p.c.n_pages || (page == p.c.n_pages && key < w.keys && lane < boxes)) {
          page = p.c.n_pages;
          cache_fault(p.c, w.b, C2T_ST_BAD_PAGE);
        }
        __syncwarp();
        const int place = (key & (p.c.page_size - 1)) - (key < w.keys ? max(key + p.box_rows - w.keys, 0) : 0);
        const uint32_t at = shared_address(sh.ring[to.at]);
        if (lane < boxes && folded)
          copy_box(at + part * (2 * box_bytes), values ? &maps.v_folded : &maps.k_folded, sh.full + to.at, 0, place, 0, w.head, page);
        else if (lane < boxes)
          copy_box(at + half * (kTile * 128) + part * box_bytes, values ? &maps.v : &maps.k, sh.full + to.at, half * 64, w.head, place, page, p.a.layer);
        to.step(1);
        ++filled;
        page = next; values = next_values; key = next_key;
      }
      if (!ok) break;
    }
    if (lane == 0)                          // (nor here)
      for (int i = max(filled - kRing, 0); i < filled; ++i) let_arrive(sh.full + i % kRing, i / kRing & 1);
    __syncwarp();
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    // The whole warp goes along, so that what the instructions take lies in uniform registers; one lane issues them.
    constexpr uint32_t kLogits = product_descriptor(kBf16, kTile, false), kHalfLogits = product_descriptor(kBf16, kTile / 2, false), kMix = product_descriptor(kBf16, D, true);
    const uint32_t ring = shared_address(sh.ring[0]);
    const uint64_t q_tile = tile_descriptor(shared_address(sh.q[0]), 1024, 16);
    const bool leader = elect_one();
    Cursor<kRing> keys = {0, 0}, vals;
    uint32_t weights_parity = 0;            // of both
    bool ok = true;
    int item = 0;
    auto arrived = [&](uint64_t *bar, uint32_t parity) { return warp_wait(sh, bar, parity); };
    // How a tile lies: 64 elements of its 128 keys after the other 64; or, folded, page by page both halves, 8 (16) keys each.  Of folded pages of 16 the
    // first 8 keys of all pages are one product's columns and the others another's, and the columns come in this order.  (The first way has its offsets
    // in the instructions: with them in registers a chunk took 6 % longer.)
    const uint64_t k_tile = tile_descriptor(ring, 1024, 16), v_tile = tile_descriptor(ring, 1024, kTile * 128);
    int box = 0;                            // bytes of a folded page; 0: the first way
    auto logits = [&](int s, int half, int buffer) {
      const uint64_t a = q_tile + half * (kRows * D * 2 / 16);
      const uint32_t at = (uint32_t)buffer * (Ring<D>::bytes / 16);
      if (leader) {
        if (box == 0) {
          const uint64_t b = k_tile + at;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {                    // 64 elements, then the other 64; 16 of them a step
            const int off = ((d >> 2) * (kTile * 128) + (d & 3) * 32) / 16;
            product_shared(tmem + s * kTile, a + off, b + off, kLogits, d > 0);
          }
        } else {
#pragma unroll 1
          for (int x = 0; x < (box == 4096 ? 2 : 1); ++x) {
            const uint64_t b = tile_descriptor(ring, box, 16) + at + x * (1024 / 16);
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
              product_shared(tmem + s * kTile + x * 64, a + ((d >> 2) * (kRows * 128) + (d & 3) * 32) / 16, b + (d < 4 ? 0 : box / 32) + (d & 3) * 2,
                             box == 4096 ? kHalfLogits : kLogits, d > 0);
          }
        }
        products_commit(sh.logits + s);
      }
      __syncwarp();
    };
    auto mix = [&](int s, int buffer, bool add) {
      const uint32_t at = (uint32_t)buffer * (Ring<D>::bytes / 16);
      if (leader) {
        if (box == 0) {
          const uint64_t b = v_tile + at;
#pragma unroll
          for (int d = 0; d < kTile / 16; ++d)
            product_tensor(tmem + 256 + s * D, tmem + weights_at<D>(s) + d * 8, b + d * (2048 / 16), kMix, add || d > 0);
        } else {                            // 16 columns are 8 keys each of two pages (of 16), or two pages (of 8)
          const uint64_t b = tile_descriptor(ring, box, box / 2) + at;
          const int jump = (box == 4096 ? 1024 : 8 * box) / 16;
#pragma unroll
          for (int d = 0; d < kTile / 16; ++d)
            product_tensor(tmem + 256 + s * D, tmem + weights_at<D>(s) + d * 8, b + (d & 3) * (box / 8) + (d < 4 ? 0 : jump), kMix, add || d > 0);
        }
      }
      __syncwarp();
    };
    auto free_buffer = [&](int buffer) {
      if (leader) products_commit(sh.empty + buffer);
      __syncwarp();
    };
    for (;; ++item) {
      if (!(ok = arrived(sh.described + item % kBlocks, item / kBlocks & 1))) break;
      const int n = uniform(sh.block[item % kBlocks].k1 - sh.block[item % kBlocks].k0), rows = uniform(sh.block[item % kBlocks].rows);
      block_read(item);
      if (rows == 0) break;
      // One step after the other: O += P V of an accumulator's tile, then its next logits.  With both halves of the rows over every tile the steps are
      // (tile, half), else the tiles; two steps come first that have logits only.
      const bool two = rows > kRows;
      const int ahead = two ? 1 : 2, steps = two ? 2 * n : n;
      box = p.folded && !two ? p.box_rows * 256 : 0;
      vals = keys;
      vals.step(min(n, ahead));
      if (!(ok = arrived(&sh.queries, item & 1))) break;
      tmem_fence_after();
#pragma unroll 1
      for (int e = -2; e < steps; ++e) {
        const int s = e & 1, t = two ? e >> 1 : e, next = t + ahead;
        const bool first_of = !two || s == 0, last_of = !two || s == 1;         // of the tile's steps
        if (e >= 0) {
          if (first_of && !(ok = arrived(sh.full + vals.at, vals.parity))) break;
          if (!(ok = arrived(sh.weights + s, weights_parity >> s & 1))) break;
          weights_parity ^= 1u << s;
          tmem_fence_after();
          mix(s, vals.at, t >= ahead);
          if (last_of) {
            free_buffer(vals.at);
            vals.step(step_of_values(t, n, ahead));
          }
        }
        if (next < n) {
          if (first_of && !(ok = arrived(sh.full + keys.at, keys.parity))) break;
          logits(s, two ? s : 0, keys.at);
          if (last_of) {
            free_buffer(keys.at);
            keys.step(step_of_keys(next, ahead));
          }
        }
      }
      if (!ok) break;
      if (leader) products_commit(&sh.done);
      __syncwarp();
      keys = vals;
    }
    if (leader) {                           // what is in flight must not outlive its tensor memory
      if (!ok) products_commit(&sh.done);
      if (!ok || item > 0) let_arrive(&sh.done, (ok ? item - 1 : item) & 1);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int s = warp >> 2, row = tid & 127;                   // the accumulator; the row in it = the lane of tensor memory
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, my_s = tmem + s * kTile + lanes, my_o = tmem + 256 + s * D + lanes,
                   my_w = tmem + weights_at<D>(s) + lanes;
    const float unit = p.a.scale * kLog2e;
    float *stage = reinterpret_cast<float *>(sh.q[0]) + warp * (D * 16);        // D * 64 bytes a warp
    uint32_t logits_parity = 0, meet_parity = 0;
    bool ok = true;
    int item = 0;
    auto all_meet = [&] {
      barrier_arrive(&sh.meet);
      const bool met = warp_wait(sh, &sh.meet, meet_parity);
      meet_parity ^= 1;
      return met;
    };
    for (;; ++item) {
      if (!(ok = described(item))) break;
      const Block &w = sh.block[item % kBlocks];
      if (w.rows == 0) break;
      const bool two = w.rows > kRows;
      const int copy_rows = rows_of_copy(w.rows);
      const int n = w.k1 - w.k0, ahead = two ? 1 : 2;
      if (!p.copy_queries) {                // (once no sums of the last block are in their memory any more)
        if (!(ok = load_queries<T, D>(p, w, sh.q[0], copy_rows, [&] { return item == 0 || all_meet(); }))) break;
        shared_writes_fence();
        tmem_fence_before();
        barrier_arrive(&sh.queries);
      }

      const int my_row = two ? s * kRows + row : row & (copy_rows - 1);         // in the block
      const int first_column = row & ~(copy_rows - 1);                          // of a copy's keys: as many as it has rows
      const bool live = my_row < w.rows;
      const bool warp_live = (my_row & ~31) < w.rows;
      const int node = token_of(p, w.row0 + (live ? my_row : w.rows - 1));
      const bool woven = is_woven(p, w.rows);
      float m = -INFINITY, l = 0.f;
      {
        const Sight see = sight_of(p, w);
        const int own = see.position(node);
        for (int t = two ? 0 : s; t < n; t += ahead) {
          const int key = w.key0(w.k0 + t);
          const bool all = key + kTile <= see.prefix && key + kTile <= see.keys && (see.window == 0 || key > own - see.window || key + kTile <= see.sinks);
          const bool masked = !__all_sync(~0u, all);
          const int last = last_box(see.keys - key, p.box_rows), over = shift_of_last_box(see.keys - key, p.box_rows);
          uint32_t on[4] = {~0u, ~0u, ~0u, ~0u};
          if (masked && warp_live) {        // (while the logits are on their way)
#pragma unroll 1
            for (int i = copy_rows / 32; i > 0; --i) {
              on[3] = on[2]; on[2] = on[1]; on[1] = on[0];
              // (folded pages of 16: a word's columns are 8 keys of four pages, from two words of keys)
              const int at = first_column / 32 + i - 1;
              uint32_t word = 0, other = 0;
#pragma unroll 1
              for (int x = 0; x < (woven ? 2 : 1); ++x) {
                const int c = 32 * (woven ? 2 * (at & 1) + x : at);
                other = word;
                word = 0;
#pragma unroll 1
                for (int shift = 0; shift <= over; shift += max(over, 1))       // the keys before the last box, then the box
                  word |= sight_bits(see, node, own, key + c - shift) & (shift ? ~low_bits(last + over - c) : low_bits(over ? last - c : 32));
              }
              if (woven) word = __byte_perm(other, word, at >> 1 ? 0x7531 : 0x6420);
              on[0] = word;
            }
          }
          if (!(ok = warp_wait(sh, sh.logits + s, logits_parity))) break;
          logits_parity ^= 1;
          tmem_fence_after();
          __syncwarp();
          if (warp_live) {
            softmax_tile<T, D>(my_s, my_w, my_o, first_column, copy_rows / 32, masked, on[0], on[1], on[2], on[3], unit, t >= ahead, m, l);
            tmem_wait_stores();
          }
          tmem_fence_before();
          barrier_arrive(sh.weights + s);
        }
      }
      if (!ok || !(ok = warp_wait(sh, &sh.done, item & 1))) break;
      tmem_fence_after();

      // ---- what the thread block has of its rows: finished, or a part for the other launch to add up
      const bool whole = w.k0 == 0 && w.k1 == w.tiles;
      m = m == -INFINITY ? m : m * unit - kLift<T>;          // (of which the weights are the powers' differences)
      float factor0 = 1.f, factor1 = 0.f;
      if (!two) {                           // over the two accumulators and, for a finished row, its copies
        sh.ml[s][row] = make_float2(m, l);
        if (!(ok = all_meet())) break;
        const int lane_row = whole ? my_row : row, step = whole ? copy_rows : kRows;
        float2 e[4][2];
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int v = 0; v < 2; ++v) e[x][v] = lane_row + x * step < kRows ? sh.ml[v][lane_row + x * step] : make_float2(-INFINITY, 0.f);
        m = -INFINITY;
#pragma unroll
        for (int x = 0; x < 4; ++x) m = fmaxf(m, fmaxf(e[x][0].x, e[x][1].x));
        l = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float f = e[x][v].x == -INFINITY ? 0.f : exp2_fast(e[x][v].x - m);
            l += e[x][v].x == -INFINITY ? e[x][v].y : e[x][v].y * f;            // (0, or NaN)
            if (lane_row + x * step == row) { if (v == 0) factor0 = f; else factor1 = f; }
          }
      }
      const float share = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      factor0 *= share;
      factor1 *= share;
      if (l != l) factor0 = l;
      const int head = w.head * p.group + w.row0 + my_row - node * p.group;
      const long long part = 2ll * blockIdx.x + (w.k0 == 0 ? 1 : 0);
      const int columns = two ? D : D / 2, column0 = two ? 0 : s * (D / 2);     // of both accumulators each group takes half
      __syncwarp();
      auto sums = [&](int c, float *v) {    // this lane's 32 columns from c on; the whole warp
        uint32_t *o = reinterpret_cast<uint32_t *>(v);
        __syncwarp();
        tmem_load32((two ? my_o : tmem + 256 + lanes) + c, o);
        tmem_wait_loads();
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= factor0;
        if (!two && n > 1) {                // (with one tile the other accumulator holds nothing)
          uint32_t o1[32];
          tmem_load32(tmem + 256 + D + lanes + c, o1);
          tmem_wait_loads();
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = fmaf(__uint_as_float(o1[j]), factor1, v[j]);
        }
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 32; j += 2) top = largest_size(top, v[j], v[j + 1]);
        return top < INFINITY;
      };
      // A part: 16 bytes a lane, the rows side by side.  Finished rows go through shared memory, so that they leave in whole sectors: a warp's own 32 rows as 16-bit
      // numbers, 32 columns at a time, swizzled, or, where there are copies to add up, all of their columns in 32 bits.
      const int place = two ? my_row : p.few_rows ? (row >> 5) * p.few_rows + my_row : row;
      const int rows_here = two ? 32 : copy_rows / 4, r0 = two ? my_row & ~31 : (warp & 3) * rows_here;         // that this warp writes
      const bool own_rows = two || copy_rows == kRows;          // without copies they are its own, and leave before the next columns come
      const float *from = reinterpret_cast<const float *>(sh.q[0]) + s * 4 * (D * 16);         // the group's
      // (each lane has one row's place, and the others' from their lanes: worked out row by row a block of 256 rows took 8 us here, not 3)
      const int out_row = own_rows ? my_row : r0 + (lane & (rows_here - 1)), out_node = token_of(p, w.row0 + out_row);
      const bool to_write = whole && (own_rows || lane < rows_here) && out_row < w.rows;
      const long long out_at = to_write ? w.b * p.a.out_seq_stride + out_node * p.a.out_token_stride +
                                              (w.head * p.group + w.row0 + out_row - out_node * p.group) * p.a.out_head_stride : -1;
      auto write = [&](int c, const float *v) {                 // 32 columns from c on of the warp's own rows: 64 bytes a row, 8 rows leave at a time
        uint4 *rows16 = reinterpret_cast<uint4 *>(stage);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          rows16[lane * 4 + (j ^ (lane >> 1 & 3))] = make_uint4(pack<T>(v[8 * j], v[8 * j + 1]), pack<T>(v[8 * j + 2], v[8 * j + 3]),
                                                                pack<T>(v[8 * j + 4], v[8 * j + 5]), pack<T>(v[8 * j + 6], v[8 * j + 7]));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          const int a = i + (lane >> 2);
          const uint4 x = rows16[a * 4 + ((lane & 3) ^ (a >> 1 & 3))];
          const long long at = __shfl_sync(~0u, out_at, a);
          if (at >= 0) *reinterpret_cast<uint4 *>(static_cast<T *>(p.a.out_dev) + at + c + 8 * (lane & 3)) = x;
        }
      };
      auto write_sums = [&](int c, const float *chunk) {        // of the rows whose copies it adds up
#pragma unroll 1
        for (int i = 0; i < rows_here && r0 + i < w.rows; i += 4) {
          const int r = r0 + i + (lane >> 3);
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int a = r + x * copy_rows;
            if (a >= kRows) break;
            const float4 y = *reinterpret_cast<const float4 *>(chunk + (a >> 5) * (D * 16) + (a & 31) * 32 + (((lane & 7) ^ (a & 7)) << 2));
            v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
          }
          const long long at = __shfl_sync(~0u, out_at, i + (lane >> 3));
          if (at >= 0) *reinterpret_cast<uint2 *>(static_cast<T *>(p.a.out_dev) + at + c + 4 * (lane & 7)) = make_uint2(pack<T>(v.x, v.y), pack<T>(v.z, v.w));
        }
        __syncwarp();
      };
      if (live && (two || (s == 0 && (!whole || row == my_row)))) {
        if (!whole) p.part_ml[part * p.part_rows + place] = make_float2(m, l);
        else if (p.a.lse_dev) p.a.lse_dev[((long long)w.b * p.a.max_queries + node) * p.a.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      }
      bool fine = true;
#pragma unroll 1
      for (int c = 0; c < columns; c += 32) {
        float v[32];
        if (warp_live) fine &= sums(column0 + c, v);
        if (whole && own_rows) {
          if (warp_live) write(column0 + c, v);
        } else if (live) {
          float *to = whole ? stage + c * 32 + lane * 32 : p.part_o + ((part * (D / 4) + (column0 + c) / 4) * p.part_rows + place) * 4;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4 *>(to + (whole ? (j ^ (lane & 7)) << 2 : j * (p.part_rows * 4))) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
        __syncwarp();
      }
      fine |= !live || l != l;              // (a row whose sum of weights is none stays so: a logit that it sees is none)
      if (whole && !own_rows) {
        const uint32_t odd = __ballot_sync(~0u, !fine);
        if (lane == 0) sh.odd[warp] = odd;
        if (!(ok = all_meet())) break;
#pragma unroll 1
        for (int c = 0; c < columns; c += 32) write_sums(column0 + c, from + c * 32);
        fine = true;
#pragma unroll 1
        for (int a = r0 + lane; a < kRows && lane < rows_here; a += copy_rows) fine &= !(sh.odd[s * 4 + (a >> 5)] >> (a & 31) & 1);
        fine |= r0 + lane >= w.rows;
      }
      const uint32_t odd_rows = __ballot_sync(~0u, !fine);
      if (odd_rows != 0 && lane == 0) atomicAdd(&sh.redoing, 1);
      for (uint32_t again = odd_rows; again; again &= again - 1) {
        // (a lane stands for its own row of the block, or, where there were copies to add up, for one of the rows that the warp wrote)
        const int from_lane = __ffs(again) - 1, r = __shfl_sync(~0u, whole && !own_rows ? r0 + lane : my_row, from_lane), at = __shfl_sync(~0u, place, from_lane);
        once_more<T, D>(p, w, r, whole ? 0 : first_column, whole ? kTile : copy_rows, column0, columns, whole, __shfl_sync(~0u, m, from_lane),
                        p.part_o + (part * (D / 4) * p.part_rows + at) * 4);
      }
      if (odd_rows != 0 && lane == 0) {
        *(volatile uint32_t *)&sh.redo_ended = milliseconds();
        __threadfence_block();
        atomicAdd(&sh.redoing, -1);
      }
      if (p.copy_queries) {
        shared_writes_fence();
        tmem_fence_before();
        barrier_arrive(&sh.queries_free);
      }
      block_read(item);
    }
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == 8) tmem_free(tmem, kMathColumns);
  if (sh.gave_up) {                         // the rows of every slot of the share are in doubt
    if (!p.split) {
      for (int pair = tid; pair < n_pairs; pair += kThreads) {
        const Block w = block_of(p, pair);
        const int before = (int)((long long)pair * p.c.kv_heads % G), turn = (int)blockIdx.x - before + ((int)blockIdx.x < before ? G : 0);
        if (w.tiles > 0 && turn < p.c.kv_heads) cache_fault(p.c, w.b, C2T_ST_INTERNAL);
      }
    } else if (tid == 0) {
      int left = sh.left, first = sh.pair;
      for (int pair = first; pair < n_pairs && left > 0; ++pair) {
        const Block w = block_of(p, pair);
        if (w.tiles == 0) continue;
        cache_fault(p.c, w.b, C2T_ST_INTERNAL);
        left -= w.tiles * p.c.kv_heads - (pair == first ? sh.head * w.tiles + sh.k0 : 0);
      }
    }
  }
}

// ---------------------------------------------------------------- parts of rows that several thread blocks read the keys of

// A cut block of rows.  Its parts lie with thread blocks c0 .. c1: the first's second place, then the others' first.  Of a part, 16 bytes of all rows lie
// side by side.  Rows that lay in the accumulators in copies have a part for each.
struct Parts {
  const float *o;
  const float2 *ml;
  int b, head, row0, rows;
  int c0, shift, copy_rows, n;              // copies = 1 << shift, so many places apart; parts of a row
  int places;
  __device__ __forceinline__ Parts(const Params &p, const int4 &cut) : o(p.part_o), ml(p.part_ml), b(cut.x), head(cut.y), row0(cut.z), rows(cut.w & 511) {
    c0 = cut.w >> 9 & 255;
    shift = rows > kRows ? 0 : rows <= 32 ? 2 : rows <= 64 ? 1 : 0;
    copy_rows = p.few_rows ? p.few_rows : kRows >> shift;
    places = p.part_rows;
    n = ((cut.w >> 17) - c0 + 1) << shift;
    // (a record that is none would lead anywhere)
    if (rows > kBlockRows || b < 0 || b >= p.c.batch || head < 0 || head >= p.c.kv_heads || row0 < 0 || row0 + (long long)rows > (long long)p.a.max_queries * p.group ||
        cut.w < 0 || cut.w >> 17 >= p.grid || c0 > cut.w >> 17)
      rows = 0;
  }
  __device__ __forceinline__ int set(int i) const {             // of a row's i-th part; and its place there
    const int c = c0 + (i >> shift);
    return 2 * c + (c == c0 ? 1 : 0);
  }
  __device__ __forceinline__ int place(int i, int r) const { return r + (i & ((1 << shift) - 1)) * copy_rows; }
};
static_assert(kBlockRows < 512, "rows in a cut's description");

// 4 V columns of a row: the running maximum, the sum of weights, the sums over the values.
template <int V>
struct Joined {
  float m = -INFINITY, l = 0.f;
  float4 o[V];
  __device__ __forceinline__ Joined() {
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void add(const float2 &ml, float top, const float4 *x) {           // top: the maximum of m and ml.x, to which m was raised
    const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
    l += ml.x == -INFINITY ? ml.y : ml.y * f;                   // (one that sees nothing: 0, or NaN)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      o[j].x = fmaf(x[j].x, f, o[j].x); o[j].y = fmaf(x[j].y, f, o[j].y); o[j].z = fmaf(x[j].z, f, o[j].z); o[j].w = fmaf(x[j].w, f, o[j].w);
    }
  }
  __device__ __forceinline__ void raise(float top) {
    const float f = m == top || m == -INFINITY ? 1.f : exp2f(m - top);          // (at -inf all sums are 0)
    l *= f;
#pragma unroll
    for (int j = 0; j < V; ++j) { o[j].x *= f; o[j].y *= f; o[j].z *= f; o[j].w *= f; }
    m = top;
  }
  // row r's parts first, first + step, ..: the loads of kAtOnce go out together
  template <int D, int kAtOnce>
  __device__ __forceinline__ void parts(const Parts &parts, int r, int first, int step, int vector) {
#pragma unroll 1
    for (int i = first; i < parts.n; i += kAtOnce * step) {
      float2 ml[kAtOnce];
      float4 x[kAtOnce][V];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int part = min(i + u * step, parts.n - 1), set = parts.set(part), place = parts.place(part, r);
        ml[u] = parts.ml[set * parts.places + place];
        const float4 *from = reinterpret_cast<const float4 *>(parts.o) + (set * (D / 4) + vector) * parts.places + place;
        const bool there = i + u * step < parts.n;
        if (!there) ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int j = 0; j < V; ++j) x[u][j] = there ? from[j * parts.places] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) top = fmaxf(top, ml[u].x);
      raise(top);
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) add(ml[u], top, x[u]);
    }
  }
  template <typename T>
  __device__ __forceinline__ void write(const Params &p, const Parts &parts, int r, int vector) const {
    const int at = parts.row0 + r, node = token_of(p, at), h = parts.head * p.group + at - node * p.group;
    const float share = l == 0.f ? 0.f : 1.f / l;
    if (vector == 0 && p.a.lse_dev) p.a.lse_dev[((long long)parts.b * p.a.max_queries + node) * p.a.q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    T *out = static_cast<T *>(p.a.out_dev) + parts.b * p.a.out_seq_stride + node * p.a.out_token_stride + h * p.a.out_head_stride + vector * 4;
#pragma unroll
    for (int j = 0; j < V; ++j)
      *reinterpret_cast<uint2 *>(out + 4 * j) = make_uint2(pack<T>(o[j].x * share, o[j].y * share), pack<T>(o[j].z * share, o[j].w * share));
  }
};

// The cut blocks of rows, each with as many items of work as it has groups of `per` rows, summed up.  (A grid over all records that there could be costs more than this:
// 2400 thread blocks that find nothing to do take 2.6 us longer than 1200.)
constexpr int kJoinThreads = 256, kJoinBlocks = 4;              // of a multiprocessor
constexpr int kMaxGrid = 256;               // workspaces are sized without asking the device: at most this many SMs are used
struct CutList {
  int4 cut[kMaxGrid];
  int before[kMaxGrid], warp_sum[kJoinThreads / 32];
  __device__ __forceinline__ int fill(const Params &p, int per) {               // all threads; how many items there are
    static_assert(kMaxGrid == kJoinThreads, "a record a thread");
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int4 mine = t < p.grid ? p.cut[t] : make_int4(0, 0, 0, 0);
    const int items = (Parts(p, mine).rows + per - 1) / per;
    int x = items;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(~0u, x, d);
      if (lane >= d) x += y;
    }
    cut[t] = mine;
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    int earlier = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 32; ++w) {
      const int s = warp_sum[w];
      earlier += w < warp ? s : 0;
      all += s;
    }
    before[t] = earlier + x - items;
    __syncthreads();
    return all;
  }
  __device__ __forceinline__ int find(int item) const {         // the record whose item it is: the last with no more items before it
    int at = 0;
#pragma unroll
    for (int step = kMaxGrid / 2; step > 0; step >>= 1)
      if (before[at + step] <= item) at += step;
    return at;
  }
};

// Thread blocks with numbers side by side often come to one multiprocessor, the first that has room: few items go to numbers far apart.  (A token of 32 heads
// behind 3000 others takes 15.1 us so, 19.6 with item i in thread block i.)
__device__ __forceinline__ int first_item(const Params &p) { return (int)(blockIdx.x * (unsigned)p.join_step % gridDim.x); }

// An item: 32 rows, half the columns; a row a lane, D / 16 columns a warp.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads, kJoinBlocks) join_parts_kernel(const __grid_constant__ Params p) {
  chain_enter();
  __shared__ CutList list;
  const int items = 2 * list.fill(p, 32);
  constexpr int kVectors = D / 64;          // of 4 columns
#pragma unroll 1
  for (int item = first_item(p); item < items; item += gridDim.x) {
    const int at = list.find(item >> 1), r = ((item >> 1) - list.before[at]) * 32 + (threadIdx.x & 31);
    const Parts parts(p, list.cut[at]);
    if (r >= parts.rows) continue;
    const int vector = ((item & 1) * (kJoinThreads / 32) + (threadIdx.x >> 5)) * kVectors;
    Joined<kVectors> sum;
    sum.template parts<D, 4>(parts, r, 0, 1, vector);
    sum.template write<T>(p, parts, r, vector);
  }
}

// Few rows have many parts each (copies too), which one after the other are what the launch would wait for.  An item is a row, every so many-th part a
// group of D / 4 lanes', 4 columns a lane.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads, kJoinBlocks) join_few_kernel(const __grid_constant__ Params p) {
  chain_enter();
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
  __shared__ CutList list;
  __shared__ float4 sums[kGroups][kLanes];
  __shared__ float2 ml[kGroups];
  const int items = list.fill(p, 1);
  const int group = threadIdx.x / kLanes, column = threadIdx.x % kLanes;
#pragma unroll 1
  for (int item = first_item(p); item < items; item += gridDim.x) {
    const int at = list.find(item), r = item - list.before[at];
    const Parts parts(p, list.cut[at]);
    Joined<1> sum;
    sum.template parts<D, 4>(parts, r, group, kGroups, column);
    sums[group][column] = sum.o[0];
    if (column == 0) ml[group] = make_float2(sum.m, sum.l);
    __syncthreads();
    if (group == 0) {
      float top = sum.m;
#pragma unroll
      for (int g = 1; g < kGroups; ++g) top = fmaxf(top, ml[g].x);
      sum.raise(top);
#pragma unroll
      for (int g = 1; g < kGroups; ++g) sum.add(ml[g], top, &sums[g][column]);
      sum.template write<T>(p, parts, r, column);
    }
    __syncthreads();
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
  // (two rows in one place)
  if ((c->batch > 1 && a->out_seq_stride < c->head_dim) || (a->max_queries > 1 && a->out_token_stride < c->head_dim) ||
      (a->q_heads > 1 && a->out_head_stride < c->head_dim))
    return C2T_EINVAL;
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

// (64 elements, places of a page, halves of a head, heads, pages) of one layer; a box is a whole page's tokens of one head
bool encode_folded(const c2t_cache &c, void *pool, int layer, TensorMap *map) {
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  const cuuint64_t sizes[5] = {64, (cuuint64_t)c.page_size, 2, (cuuint64_t)c.kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t bytes[4] = {2 * (cuuint64_t)c.token_stride, 128, c.kv_heads > 1 ? 2 * (cuuint64_t)c.head_stride : 256,
                               c.n_pages > 1 ? 2 * (cuuint64_t)c.page_stride : 256};
  const cuuint32_t box[5] = {64, (cuuint32_t)c.page_size, 2, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return encode(reinterpret_cast<CUtensorMap *>(map), c.dtype == C2T_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
                static_cast<uint16_t *>(pool) + layer * c.layer_stride, sizes, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// (elements, heads, tokens, sequences); a box is 64 elements of kQueryRows rows: the heads of a key head, of as many tokens as that takes
bool encode_queries(const c2t_cache &c, const c2t_attention &a, int group, TensorMap *map) {
  const EncodeTiled encode = encoder();
  if (!encode) return false;
  const cuuint64_t sizes[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)a.q_heads, (cuuint64_t)a.max_queries, (cuuint64_t)c.batch};
  const int64_t steps[3] = {a.q_head_stride, a.q_token_stride, a.q_seq_stride};
  cuuint64_t bytes[3];
  for (int i = 0; i < 3; ++i) bytes[i] = sizes[i + 1] > 1 ? 2 * (cuuint64_t)steps[i] : 256;
  const cuuint32_t box[4] = {64, (cuuint32_t)group, (cuuint32_t)(kQueryRows / group), 1}, ones[4] = {1, 1, 1, 1};
  return encode(reinterpret_cast<CUtensorMap *>(map), c.dtype == C2T_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
                const_cast<void *>(a.q_dev), sizes, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int common_factor(int a, int b) {
  while (b != 0) { const int r = a % b; a = b; b = r; }
  return a;
}

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
    // (a token of 32 heads behind 6000 others: 17.5 us with the first, 31.3 with the second)
    if (rows <= 32) e = launch_chained(join_few_kernel<T, D>, dim3(kJoinBlocks * sms), dim3(kJoinThreads), 0, s, p);
    else e = launch_chained(join_parts_kernel<T, D>, dim3(kJoinBlocks * sms), dim3(kJoinThreads), 0, s, p);
  }
  return e;
}

}  // namespace
}  // namespace c2t

using namespace c2t;

extern "C" {

#ifdef C2T_DEBUG_BOUNDS
int c2t_debug_attention_wait_limit = kTries;                    // tests let the waits run out
#endif

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
  if (blocks * p.c.batch * p.c.kv_heads > 0x7FFFFFFF || rows * p.group > 0x7FFFFFFF) return C2T_ERANGE;
  p.group_inverse = p.group > 1 ? (uint32_t)((0x100000000ull + p.group - 1) / p.group) : 0;
  p.blocks_per_seq = (int)blocks;
  p.box_rows = p.c.page_size < kTile ? p.c.page_size : kTile;
  // (tiles of all blocks of rows are counted in 32 bits; with whole blocks 64 sequences' tokens behind 4096 take 196 us instead of 174)
  p.split = blocks * p.c.batch <= kMaxPairs && blocks * p.c.batch * p.c.kv_heads * ((int64_t)p.c.max_pages * p.c.page_size / kTile + 1) <= 0x7FFFFFFF;
  // Equal pieces against an even deal: trees of 8 sequences behind 2048 take 38.7 us and 41.7, a token of 32
  // heads behind 6000 others 17.5 and 21.1.  A piece of fewer tiles than these costs more to join than it saves: 8 trees behind 300 take 23.8 us with pieces of 2 tiles, 20.2 of 3.
  p.least_tiles = rows > kRows ? 3 : 2;
#ifdef C2T_DEBUG_BOUNDS
  p.tries = c2t_debug_attention_wait_limit;
#endif
  p.more_tiles = rows > kRows ? 3 : 4;
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
  // By copies where the groups of heads divide a copy's rows and no dimension is without a stride, as broadcast queries have: a window takes 76 us, thread by
  // thread 81; trees of 32 sequences behind 3000 135.5 and 133.6; a chunk 524 and 517.
  const bool strides = (p.c.batch == 1 || p.a.q_seq_stride > 0) && (p.a.max_queries == 1 || p.a.q_token_stride > 0) && (p.a.q_heads == 1 || p.a.q_head_stride > 0);
  p.copy_queries = strides && p.group <= kQueryRows && (p.group & (p.group - 1)) == 0 && encode_queries(p.c, p.a, p.group, &maps.q);
  // Copies of 2 KB are dealt with at 140 cycles each, which is less than the memory gives.  With both halves of a head in one, 64 sequences' tokens behind 4096
  // take 174 us instead of 192, trees of 32 sequences behind 3000 with 32 key heads 304 instead of 325.  (The logits are two products of half the columns each then, which blocks of
  // more than 128 rows would wait for: they take pages half by half.)
  p.folded = p.c.head_dim == 128 && p.c.page_size <= 16 && encode_folded(p.c, p.c.k_dev, p.a.layer, &maps.k_folded) &&
             encode_folded(p.c, p.c.v_dev, p.a.layer, &maps.v_folded);
  if (sms > kMaxGrid) sms = kMaxGrid;
  p.grid = sms;
  p.few_rows = rows <= 32 ? (int)rows : 0;
  p.part_rows = rows <= 32 ? 4 * (int)rows : rows <= kRows ? kRows : kBlockRows;
  p.join_step = kJoinBlocks * sms * 309 / 500 | 1;              // (the golden section: multiples of it keep apart)
  while (common_factor(p.join_step, kJoinBlocks * sms) != 1) p.join_step += 2;
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
