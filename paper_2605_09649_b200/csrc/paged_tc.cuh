// Tensor memory and tcgen05 issue as the chunk kernels of the paged caches use them.
#pragma once

#include "tcgen05_attn.cuh"

namespace tkv {

__device__ __forceinline__ void t_tmem_ld16(uint32_t taddr, uint32_t* t) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(t[0]), "=r"(t[1]), "=r"(t[2]), "=r"(t[3]), "=r"(t[4]), "=r"(t[5]), "=r"(t[6]), "=r"(t[7]), "=r"(t[8]), "=r"(t[9]), "=r"(t[10]),
          "=r"(t[11]), "=r"(t[12]), "=r"(t[13]), "=r"(t[14]), "=r"(t[15])
        : "r"(taddr));
}
__device__ __forceinline__ void t_tmem_st16(uint32_t taddr, const uint32_t* t) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(t[0]), "r"(t[1]), "r"(t[2]), "r"(t[3]), "r"(t[4]), "r"(t[5]), "r"(t[6]), "r"(t[7]), "r"(t[8]), "r"(t[9]), "r"(t[10]), "r"(t[11]),
        "r"(t[12]), "r"(t[13]), "r"(t[14]), "r"(t[15])
        : "memory");
}
__device__ __forceinline__ void t_tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void t_tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Products issued by one lane of a converged warp: every operand is the same in all lanes, so it stays in uniform registers and
// an instruction costs a few issue slots.  (Behind a branch on the lane each took about 120 cycles beside the softmax warps, more
// than the 64 of its product.)  Descriptors: the low words change, the high words are t_desc_hi() for both operands.
constexpr uint32_t T_DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);           // rows in groups of 8, 1024 bytes apart; 128-byte swizzle
__device__ __forceinline__ uint32_t t_desc_lo(uint32_t saddr, uint32_t lead_bytes) { return ((saddr & 0x3FFFFu) >> 4) | ((lead_bytes >> 4) << 16); }
__device__ __forceinline__ uint32_t t_elect() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e;
}
__device__ __forceinline__ void t_umma(uint32_t leader, uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 e, %0, 0;\n\t"
        "mov.b64 a, {%2, %6};\n\t"
        "mov.b64 b, {%3, %6};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%1], a, b, %4, p;\n\t}" ::"r"(leader),
        "r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(T_DESC_HI)
        : "memory");
}
__device__ __forceinline__ void t_umma_ts(uint32_t leader, uint32_t tmem_d, uint32_t tmem_a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 e, %0, 0;\n\t"
        "mov.b64 b, {%3, %6};\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], b, %4, p;\n\t}" ::"r"(leader),
        "r"(tmem_d), "r"(tmem_a), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(T_DESC_HI)
        : "memory");
}
__device__ __forceinline__ void t_commit(uint32_t leader, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %0, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(leader), "r"(bar)
        : "memory");
}
// 32 bytes, a whole sector per lane: rows lie d floats apart, and two stores of 16 bytes would each move half a sector.
__device__ __forceinline__ void t_store32(float* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ uint32_t t_uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
// Barrier of the two warps that share 32 rows, the n-th time: an mbarrier, so that the wait has a limit.  false: gave up.
__device__ __forceinline__ bool t_pair_sync(uint32_t bar, unsigned n) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) a_bar_arrive(bar);
    return __all_sync(0xffffffffu, a_bar_wait(bar, n & 1u));
}

}  // namespace tkv
