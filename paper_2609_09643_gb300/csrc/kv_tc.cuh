// The fifth-generation tensor cores, as the KV-cache operators use them: inline
// PTX for mbarriers with bounded waits, tensor memory and tcgen05 products of
// 16-bit operands with 32-bit sums.
#pragma once

#include "kv.cuh"

namespace unison {

// ------------------------------------------------------------- mbarriers --
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(1000u)
      : "memory");
  return ok != 0;
}
// Waits until the phase of that parity is complete.  Gives up after about a
// second, or when another thread of the CTA has: false, and *dead is set.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *dead) {
  for (int i = 0; i < 1 << 18; i++) {
    if (bar_try(bar, parity)) return true;
    if (*dead) return false;
  }
  *dead = 1;
  return false;
}
// A place in a ring of n, and the parity of the turn: what fills the place is
// waited for with `turn`, its release by the turn before with `turn ^ 1` (true
// at once in the first turn).  No divisions: a warp of its own takes five
// cycles for each instruction.
struct Ring {
  int at = 0;
  uint32_t turn = 0;
  __device__ __forceinline__ void next(int n) {
    if (++at == n) at = 0, turn ^= 1;
  }
};
// What this thread wrote to shared memory, or knows to have been written there
// (a barrier that it waited for), is seen by the products it issues next.
__device__ __forceinline__ void fence_to_tensor() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ----------------------------------------------- two 32-bit sums at once --
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t r, float &a, float &b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// --------------------------------------------------------- tensor memory --
// By all lanes of one warp; the address is written to shared memory.
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// The same for given registers: nothing that reads them moves in front of it.
template <int N>
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[N]) {
  static_assert(N == 16 || N == 32, "what tmem_ld16 and tmem_ld32 read");
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]),
                      "+r"(r[i + 6]), "+r"(r[i + 7]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define KV_R4(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3])
#define KV_W4(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
#define KV_R8(r, i) KV_R4(r, i), KV_R4(r, i + 4)
#define KV_W8(r, i) KV_W4(r, i), KV_W4(r, i + 4)
// 32 columns of this warp's quarter of the lanes: lane i of the warp has lane i
// of the quarter.  The registers are valid after tmem_wait_ld.
__device__ __forceinline__ void tmem_ld32(uint32_t *r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : KV_R8(r, 0), KV_R8(r, 8), KV_R8(r, 16), KV_R8(r, 24)
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t *r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : KV_R8(r, 0), KV_R8(r, 8)
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,"
      "%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      KV_W8(r, 0), KV_W8(r, 8), KV_W8(r, 16), KV_W8(r, 24)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16};" ::"r"(addr),
      KV_W8(r, 0), KV_W8(r, 8)
      : "memory");
}
#undef KV_R8
#undef KV_W8
#undef KV_R4
#undef KV_W4

// --------------------------------------------------------------- products --
// Operands in shared memory lie in 128-byte rows of 64 elements, 16-byte chunk
// c of row r at c ^ (r & 7) (the 128-byte swizzle); 8 rows are 1,024 bytes,
// and blocks of 64 elements follow each other `block` bytes apart.
// Descriptor of such an operand: `block` is the leading offset, 1,024 the
// stride offset, version 1, swizzle mode 2.  The same one serves both majors:
// rows along the sum (values: MN-major) or along the other axis (K-major, where
// the leading offset is not used).
// (The upper word is the same for all of them.)
constexpr uint32_t kOperandHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t smem_operand(uint32_t addr, uint32_t block) {
  return (addr & 0x3FFFF) >> 4 | block >> 4 << 16;
}
// Instruction descriptor: 16-bit operands (type 0: fp16, 1: bf16), 32-bit sums,
// m rows, n columns; the second operand K-major or MN-major; the first negated.
__device__ __forceinline__ uint32_t product_shape(int type, int m, int n, bool b_mn_major, bool negate_a) {
  return 1u << 4 | type << 7 | type << 10 | (negate_a ? 1u : 0u) << 13 | (b_mn_major ? 1u : 0u) << 16 |
         (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
template <typename T>
constexpr int kOperandType = 1;
template <>
constexpr int kOperandType<__half> = 0;

// A value that all lanes of the warp have: told to the compiler, so that what
// follows from it (descriptors, addresses, loops) is kept in uniform registers,
// where the products take it from.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(one));
  return one != 0;
}
// d (+)= a b, both in shared memory; 16 elements of the sum.  The whole warp
// comes here and the lane with `one` issues: without a branch, the operands'
// descriptors stay in uniform registers.
__device__ __forceinline__ void product_ss(bool one, uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %6, 0;\n"
      " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add), "r"(kOperandHigh), "r"((uint32_t)one)
      : "memory");
}
// The same with a in tensor memory.
__device__ __forceinline__ void product_ts(bool one, uint32_t d, uint32_t a, uint32_t b, uint32_t shape, bool add) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %6, 0;\n"
      " mov.b64 b, {%2, %5};\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(shape), "r"((uint32_t)add), "r"(kOperandHigh), "r"((uint32_t)one)
      : "memory");
}
// The barrier gets one arrival when all products of that lane so far are done.
__device__ __forceinline__ void products_done(bool one, uint32_t bar) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar),
      "r"((uint32_t)one)
      : "memory");
}
__device__ __forceinline__ void bar_arrive_by(bool one, uint32_t bar) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n @q mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n" ::"r"(
                   bar),
               "r"((uint32_t)one)
               : "memory");
}

// Address of a 16-byte chunk in such an operand of rows * 128-byte blocks.
__device__ __forceinline__ uint32_t operand_chunk(uint32_t base, int rows, int row, int chunk) {
  return base + (chunk >> 3) * (rows * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4);
}

}  // namespace unison
