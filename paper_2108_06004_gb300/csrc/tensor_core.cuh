// The fifth-generation tensor cores' instructions as these kernels use them: one CTA, 16-bit operands, fp32 sums in
// tensor memory, matrices in shared memory in 128-byte rows whose 16-byte words are exchanged (word w of row r
// lies at w ^ (r % 8)), as the tensor memory accelerator writes them.
#pragma once

#include "gs_layer.cuh"

namespace gs {
namespace tc {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers ---------------------------------------------------------------------------------
__device__ __forceinline__ void barrier_init(uint64_t* bar, int arrivals) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(bar)) : "memory");
}
// Waits for the end of the barrier's phase of this parity; false when that has not come after a number of tries, each of which is
// suspended for a microsecond at most.
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, int phase, int tries) {
  for (; tries > 0; --tries) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, 1000;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(shared_address(bar)), "r"(phase & 1)
        : "memory");
    if (done) return true;
  }
  return false;
}
// What this thread has written to shared memory is seen by the tensor cores and bulk copies.
__device__ __forceinline__ void shared_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// ---- tensor memory ------------------------------------------------------------------------------
// Called by one whole warp; the address is written to shared memory.
template <int COLUMNS>
__device__ __forceinline__ void tmem_alloc(uint32_t* at) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(at)), "n"(COLUMNS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLUMNS>
__device__ __forceinline__ void tmem_free(uint32_t at) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(COLUMNS) : "memory");
}
__device__ __forceinline__ void wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Adjacent columns of the warp's own 32 lanes, a lane for each thread.
#define GS_R8(v, n) "+r"(v[n]), "+r"(v[n + 1]), "+r"(v[n + 2]), "+r"(v[n + 3]), "+r"(v[n + 4]), "+r"(v[n + 5]), "+r"(v[n + 6]), "+r"(v[n + 7])
#define GS_O8(v, n) "=r"(v[n]), "=r"(v[n + 1]), "=r"(v[n + 2]), "=r"(v[n + 3]), "=r"(v[n + 4]), "=r"(v[n + 5]), "=r"(v[n + 6]), "=r"(v[n + 7])
#define GS_I8(v, n) "r"(v[n]), "r"(v[n + 1]), "r"(v[n + 2]), "r"(v[n + 3]), "r"(v[n + 4]), "r"(v[n + 5]), "r"(v[n + 6]), "r"(v[n + 7])
__device__ __forceinline__ void tmem_load(uint32_t (&v)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : GS_O8(v, 0), GS_O8(v, 8), GS_O8(v, 16), GS_O8(v, 24)
      : "r"(at)
      : "memory");
  // what was loaded is used only after the wait
  asm volatile("tcgen05.wait::ld.sync.aligned;" : GS_R8(v, 0), GS_R8(v, 8), GS_R8(v, 16)::"memory");
  asm volatile("" : GS_R8(v, 24));
}
__device__ __forceinline__ void tmem_load(uint32_t (&v)[16], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : GS_O8(v, 0), GS_O8(v, 8)
      : "r"(at)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" : GS_R8(v, 0), GS_R8(v, 8)::"memory");
}
__device__ __forceinline__ void tmem_store(const uint32_t (&v)[32], uint32_t at) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::GS_I8(v, 0),
      GS_I8(v, 8), GS_I8(v, 16), GS_I8(v, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store(const uint32_t (&v)[8], uint32_t at) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::GS_I8(v, 0), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store(const uint32_t (&v)[16], uint32_t at) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::GS_I8(v, 0),
      GS_I8(v, 8), "r"(at)
      : "memory");
}
// 8 x 8 matrices of 16-bit elements in the layout that load_across leaves them in: of 16 lanes,
// matrix 0 (lanes 0 ... 7) and 1 (lanes 8 ... 15) in four columns, 2 and 3 in the next four, and so on.
__device__ __forceinline__ void tmem_store_matrices(const uint32_t* v, uint32_t at, std::integral_constant<int, 4>) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%4], {%0, %1, %2, %3};" ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store_matrices(const uint32_t* v, uint32_t at, std::integral_constant<int, 8>) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::GS_I8(v, 0), "r"(at) : "memory");
}
// Four 8 x 8 matrices of 16-bit elements, transposed: lane l gives the address of row l % 8 of matrix l / 8, and gets elements
// (2 (l % 4), l / 4) and (2 (l % 4) + 1, l / 4) of each.
__device__ __forceinline__ void load_across(uint32_t (&v)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(at)
               : "memory");
}
#undef GS_R8
#undef GS_O8
#undef GS_I8

// ---- products -----------------------------------------------------------------------------------
// A matrix in shared memory, as the lower word of its descriptor.  `next`: along the contracted dimension where it is the
// adjacent one: not used; where the other one is: bytes from one group of 64 of them to the next.  Eight rows of 128
// bytes follow one another at 1024 bytes, which the upper word says.
__device__ __forceinline__ uint32_t matrix(uint32_t address, uint32_t next) { return (address & 0x3FFFF) >> 4 | (next >> 4) << 16; }
constexpr uint32_t kMatrixRows = 1024 >> 4 | 1u << 14 | 2u << 29;
// D (128 x n, fp32) of 16-bit A and B; `across`: B's adjacent dimension is not the contracted one.
template <typename E>
__device__ __forceinline__ constexpr uint32_t product(int n, bool across) {
  const uint32_t type = sizeof(E) == 2 && std::is_same<E, __nv_bfloat16>::value ? 1u : 0u;
  return 1u << 4 | type << 7 | type << 10 | (across ? 1u : 0u) << 16 | (uint32_t)(n / 8) << 17 | (128u / 16) << 24;
}
// D = A B, or D += A B, of 16 contracted elements.  The operands' offsets (in bytes, or columns) are added here, so that one
// register an operand is enough for any number of products: a thread that keeps a descriptor for each, in local memory,
// issues one in 180 clocks, and a product of 128 x 128 x 16 takes 64 at the tensor cores' nominal rate.
template <int AT_A, int AT_B>
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint32_t b, uint32_t how, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 da, db;\n setp.ne.u32 p, %4, 0;\n add.u32 x, %1, %5;\n add.u32 y, %2, %6;\n"
      " mov.b64 da, {x, %7};\n mov.b64 db, {y, %7};\n tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(how), "r"((uint32_t)add), "n"(AT_A / 16), "n"(AT_B / 16), "n"(kMatrixRows)
      : "memory");
}
// A in tensor memory: a lane for each row, two adjacent elements in a column.
template <int AT_A, int AT_B>
__device__ __forceinline__ void multiply_t(uint32_t d, uint32_t a, uint32_t b, uint32_t how, bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 db;\n setp.ne.u32 p, %4, 0;\n add.u32 x, %1, %5;\n add.u32 y, %2, %6;\n"
      " mov.b64 db, {y, %7};\n tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, p;\n}" ::"r"(d),
      "r"(a), "r"(b), "r"(how), "r"((uint32_t)add), "n"(AT_A), "n"(AT_B / 16), "n"(kMatrixRows)
      : "memory");
}
// f(0), f(1), ... f(N - 1), each with its number as a constant.
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>());
  }
}
// The barrier's phase ends when all products that this thread has issued are done.
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(bar)) : "memory");
}

__device__ __forceinline__ void tile_load(void* to, const CUtensorMap* map, int d, int h, int t, int b, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          shared_address(to)),
      "l"(map), "r"(d), "r"(h), "r"(t), "r"(b), "r"(shared_address(bar))
      : "memory");
}

__device__ __forceinline__ void tile_store(const void* from, const CUtensorMap* map, int d, int h, int t, int b) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(d), "r"(h), "r"(t),
               "r"(b), "r"(shared_address(from))
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// All tiles that this thread has stored have been read; are where they belong.
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

}  // namespace tc
}  // namespace gs
