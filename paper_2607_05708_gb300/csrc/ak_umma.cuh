// tcgen05 as the attention kernels use it: products issued by a whole warp, tensor memory moved in
// rows, bounded waits of a warp of one role.
#pragma once

#include "ak_sm100.cuh"

namespace ak {

// 32 registers to 32 consecutive columns of the thread's lane, and the wait.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// The kernel behind this one may be scheduled as soon as all CTAs have come here or ended (it waits for the
// end of this one all the same: griddep_wait).
__device__ __forceinline__ void griddep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// D[tmem] (+)= A[smem] B[smem]^T and D[tmem] (+)= A[tmem] B[smem], fp16, by the lane that
// has `go`.  The whole warp comes here, so that addresses stay in uniform registers
// (behind a branch on the lane an issue took 120 cycles and more; the product takes 64),
// and of a shared-memory descriptor (ak_sm100.cuh) only the low word changes.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void umma_ss(uint32_t go, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "mov.b64 x, {%2, %6};\n\t"
        "mov.b64 y, {%3, %6};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], x, y, %4, p;\n\t}" ::"r"(go),
        "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI)
        : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t go, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "mov.b64 y, {%3, %6};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], y, %4, p;\n\t}" ::"r"(go),
        "r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI)
        : "memory");
}
__device__ __forceinline__ void umma_commit_if(uint32_t go, uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(go),
        "r"(smem_u32(bar))
        : "memory");
}
// One thread's products behind elect.sync, of which the compiler knows that one thread comes through: an
// issue then costs what the product does (M = 128, 16 of K, cycles: N = 16 40, 32 41, 64 49, 128 65, 256 129, A in
// tensor memory 11, 18, 33, 65, 129; by predicate, as above, none under 70).
__device__ __forceinline__ bool elect_one() {
    uint32_t x;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(x));
    return x != 0;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
    umma_bf16(d, a, b, idesc, acc);
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}
// The same by the even CTA of a pair, for both (ak_sm100.cuh): A's rows in the tensor memory of the CTA that has
// them.
__device__ __forceinline__ void mma2_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}
// High words of descriptors: 128-byte swizzle (DESC_HI), and 64-byte swizzle: atoms of 8 K-rows x 32
// values along N, 512 bytes, one after the other along K (MN-major).
constexpr uint32_t DESC_HI_64 = (512u >> 4) | (1u << 14) | (4u << 29);
__device__ __forceinline__ uint64_t desc64(uint32_t lo, uint32_t hi = DESC_HI) { return (uint64_t)hi << 32 | lo; }
// Low words of the descriptors of K-major and MN-major tiles.
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return ((saddr & 0x3ffffu) >> 4) | 1u << 16; }
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t lbo) {
    return ((saddr & 0x3ffffu) >> 4) | (lbo >> 4) << 16;
}
// Instruction descriptor: D fp32, A and B fp16 (or both bf16), M = 128 or 64.
__host__ __device__ constexpr uint32_t idesc_f16(int n, bool bf16 = false, int m = 128) {
    return (1u << 4) | (bf16 ? 1u << 7 | 1u << 10 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// The A operand is MN-major (M contiguous in shared memory) instead of K-major.
constexpr uint32_t IDESC_A_MN_MAJOR = 1u << 15;

// Bounded wait of a warp of one role; when any role's wait has expired the others give up too.  One
// answer for all lanes: a lane that gave up beside others that did not would leave them in
// their next shuffle.
__device__ __forceinline__ bool wide_wait(uint64_t *bar, uint32_t parity, volatile int *dead,
                                          int *status) {
    bool there = mbar_test_wait(bar, parity);
    for (uint32_t i = 0; !there && i < WAIT_LIMIT; ++i) {
        there = mbar_try_wait(bar, parity);
        if ((i & 255u) == 255u && *dead) break;
    }
    if (__all_sync(0xffffffffu, there)) return true;
    if (!there && !*dead) set_status(status, AKASHIC_ETIMEOUT);
    *dead = 1;
    return false;
}

}  // namespace ak
