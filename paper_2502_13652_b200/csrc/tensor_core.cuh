// The instructions of sm_100a that the attention kernel is made of: transaction barriers, bulk tensor copies, tensor-core products whose
// accumulators lie in tensor memory.  One thin function each.
#pragma once
#include <stdint.h>

namespace c2t {

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// one lane of a whole warp, the same one every time
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes;
}
// a value that all lanes of the warp have, in a register that they share
__device__ __forceinline__ int uniform(int x) { return __reduce_max_sync(~0u, x); }

// ---------------------------------------------------------------- barriers in shared memory

__device__ __forceinline__ void barrier_init(uint64_t *bar, int arrivals) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_arrive(uint64_t *bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(bar)) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t *bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint64_t *bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(shared_address(bar)), "r"(parity) : "memory");
  return done;
}
// orders this thread's writes to shared memory before later accesses by copies and tensor cores
__device__ __forceinline__ void shared_writes_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---------------------------------------------------------------- bulk tensor copies

struct alignas(64) TensorMap { uint64_t opaque[16]; };       // what the driver's encoder fills in

__device__ __forceinline__ void tensor_map_prefetch(const TensorMap *map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t to, const TensorMap *map, uint64_t *bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
               ::"r"(to), "l"(reinterpret_cast<uint64_t>(map)), "r"(shared_address(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}

__device__ __forceinline__ void copy_box(uint32_t to, const TensorMap *map, uint64_t *bar, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(to), "l"(reinterpret_cast<uint64_t>(map)), "r"(shared_address(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// ---------------------------------------------------------------- tensor memory

__device__ __forceinline__ void tmem_alloc(uint32_t *address, int columns) {     // one whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(address)), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t address, int columns) {       // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define C2T_R4(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3])
#define C2T_W4(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3])
// 32 columns of this warp's 32 lanes: lane's row, columns ascending
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t *r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
               "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : C2T_R4(r, 0), C2T_R4(r, 4), C2T_R4(r, 8), C2T_R4(r, 12), C2T_R4(r, 16), C2T_R4(r, 20), C2T_R4(r, 24), C2T_R4(r, 28) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
               "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
               ::C2T_W4(r, 0), C2T_W4(r, 4), C2T_W4(r, 8), C2T_W4(r, 12), C2T_W4(r, 16), C2T_W4(r, 20), C2T_W4(r, 24), C2T_W4(r, 28), "r"(at) : "memory");
}
// 16 columns
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::C2T_W4(r, 0), C2T_W4(r, 4), C2T_W4(r, 8), C2T_W4(r, 12), "r"(at) : "memory");
}
#undef C2T_R4
#undef C2T_W4

// ---------------------------------------------------------------- products

// A tile in shared memory whose rows are 128 bytes, swizzled over 8 rows (1024 bytes).  `along`: bytes to the next 8 rows; `across`: bytes
// to the next 128-byte column of blocks (used where the rows run along the product's inner dimension).
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t address, uint32_t along, uint32_t across) {
  return (uint64_t)((address & 0x3FFFF) >> 4) | (uint64_t)(across >> 4) << 16 | (uint64_t)(along >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 16-bit inputs (bf16 or f16), 32-bit sums: 128 rows of A by `n` of B; B with its rows along n, or (transposed) along the inner dimension
__host__ __device__ constexpr uint32_t product_descriptor(bool bf16, int n, bool transposed_b) {
  return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (transposed_b ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}
// 16 of the inner dimension; one thread.  add: to what the accumulator holds, else in its place.
__device__ __forceinline__ void product_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void product_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {      // A in tensor memory
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// an arrival at `bar` once this thread's products so far are done
__device__ __forceinline__ void products_commit(uint64_t *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(bar)) : "memory");
}

}  // namespace c2t
