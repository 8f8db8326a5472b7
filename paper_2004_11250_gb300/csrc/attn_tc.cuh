// What the two tile kernels share (attn_tile.cu, attn8_tile.cu): descriptors, products, copies and commits issued by a
// whole warp, tensor memory.
#pragma once

#include "attn.cuh"

namespace ppc_attn {

// Shared-memory descriptors of 128-byte swizzled operands.  K-major (Q, K): rows of 128 bytes, groups of 8 rows 1024
// bytes apart.  MN-major (V): 128 bytes of values per key, groups of 8 keys 1024 bytes apart, the next 64 values `lbo`
// bytes on.
constexpr uint32_t kDescHi = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFF) | (lbo >> 4) << 16; }
template <class T>
__host__ __device__ constexpr uint32_t idesc(int m, int n, bool b_mn) {
  const uint32_t f = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (f << 7) | (f << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Copies, products and commits of a whole warp, issued by its leader.  The warp stays together, so that the operands are in
// uniform registers, as the instructions want them: behind a branch of one lane each is moved there first, and an issue
// took some 100 cycles.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t acc, uint32_t leader) {
  asm volatile(
      "{ .reg .pred p, q; .reg .b64 x, y; setp.ne.b32 p, %5, 0; setp.ne.b32 q, %6, 0; mov.b64 x, {%1, %4}; mov.b64 y, {%2, %4};"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(id), "r"(kDescHi), "r"(acc), "r"(leader)
      : "memory");
}
// the left operand in TMEM
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t acc, uint32_t leader) {
  asm volatile(
      "{ .reg .pred p, q; .reg .b64 y; setp.ne.b32 p, %5, 0; setp.ne.b32 q, %6, 0; mov.b64 y, {%2, %4};"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(id), "r"(kDescHi), "r"(acc), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %1, 0; @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(bar),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %5, 0;"
      " @q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4]; }" ::"r"(dst),
      "l"(m), "r"(x), "r"(y), "r"(bar), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void expect(uint32_t bar, int bytes, uint32_t leader) {
  asm volatile(
      "{ .reg .pred q; setp.ne.b32 q, %2, 0; @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1; }" ::"r"(bar), "r"(bytes),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ uint32_t elect() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tm_ld32(uint32_t a, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(a));
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tm_st32(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
      "r"(r[31]), "r"(a)
      : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t a, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
      "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15]), "r"(a)
      : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// the lowest c bits
__device__ __forceinline__ uint64_t below(int c) { return c >= 64 ? ~0ull : c > 0 ? (1ull << c) - 1 : 0; }

// what a wait comes to that does not find its phase complete at once
static __device__ __noinline__ void hold_on(uint32_t bar, uint32_t parity, volatile int* dead) {
  if (!*dead && !wait(bar, parity)) *dead = 1;
}

}  // namespace ppc_attn
