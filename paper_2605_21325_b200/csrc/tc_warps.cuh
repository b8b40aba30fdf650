// What the warp-specialised scans share (scan_kernel.cu with layer_kernel.cuh, linear_tc_kernel.cu): arrivals and waits of whole warps, products with an operand in
// tensor memory, transposing shared-memory moves.
#pragma once
#include "tc_device.cuh"

namespace tri_inv {
namespace {

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// whether the phase is complete, without waiting
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// One arrival for the whole warp: every lane has made its operand writes visible (the caller's fences) before the lanes
// meet; lane 0 then arrives for all of them.
__device__ __forceinline__ void warp_arrive(uint32_t bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t& m0, uint32_t& m1, uint32_t& m2, uint32_t& m3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(m0), "=r"(m1), "=r"(m2), "=r"(m3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stmatrix_x4_trans(uint32_t addr, uint32_t m0, uint32_t m1, uint32_t m2, uint32_t m3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(m0), "r"(m1), "r"(m2), "r"(m3) : "memory");
}
// D (tensor memory) += A (tensor memory, one 32-bit column = two bf16 of the summed index) . B (shared memory); called by a
// whole warp, one lane issues
__device__ __forceinline__ void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Packed pairs of a 16-lane fragment (row g: r[2 n], row g + 8: r[2 n + 1], n-tile n = columns 4 n + t) into tensor memory
__device__ __forceinline__ void tmem_st_packed16(const uint32_t (&r)[8], uint32_t taddr) {   // 16 columns
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_packed32(const uint32_t (&r)[16], uint32_t taddr) {  // 32 columns
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}

// A bounded wait whose outcome all lanes of the warp agree on.  A lane that has seen the phase may poll it again: the next phase
// of every barrier of this kernel waits for something that each of its waiting warps does after its wait.  Not inlined: the
// first polls are (below), and with the timer's loop in every wait as well the 128-column instance was 2 to 6 % slower (a vote
// behind the per-lane wait: 1 to 6 % more); in this form calls of 1 .. 300 (sequence, head) pairs and 16 .. 512 chunks
// take between 0.97 and 1.02 of the per-lane waits' time.
__device__ __noinline__ bool wait_by_warp(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
  const unsigned long long t0 = global_timer_ns();
  for (uint32_t i = 1; i < kSpinLimit; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & 63u) == 0 && __any_sync(0xffffffffu, global_timer_ns() - t0 > limit_ns)) return false;
  }
  return false;
}

}  // namespace
}  // namespace tri_inv
