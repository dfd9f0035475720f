// The block-scaled tensor-core instructions of the 4-bit kernels (tcgen05 kind::mxf4).
#ifndef SAEM_MX_TC_CUH_
#define SAEM_MX_TC_CUH_

#include "mx_common.cuh"
#include "tc_common.cuh"

namespace saem {

// Shared-memory matrix descriptor of a 512-byte scale piece for tcgen05.cp: no swizzle, 16-byte rows, 8-row groups 128
// bytes apart.
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (8ull << 16) | (8ull << 32) | (1ull << 46);
}
// The warps that issue copies and MMAs run their loops as a whole, and one elected lane (`on`) issues.  What the
// instructions take then stays in uniform registers: inside an `if (lane == 0)`, or behind a wait whose result the
// compiler must take for different in every lane, each operand has to be moved to a uniform register first, and an MMA or
// a copy took 80 to 120 cycles to issue (an MMA of 128 x 48 x 64 takes 44, a scale copy 8).
__device__ __forceinline__ uint32_t warp_uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                               unsigned long long limit_ns = kWaitLimitNs) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status, limit_ns));
}
// At the end of the warps that issue copies and MMAs: whatever is under way lands before the CTA gives its shared and tensor
// memory back, also where another warp has given up meanwhile.  Bounded as every wait; without an abort the barriers have
// completed, or will before the epilogue has.
__device__ __forceinline__ bool mbar_settle_warp(uint32_t bar, uint32_t parity, int* status) {
    int never = 0;
    return mbar_wait_warp(bar, parity, &never, status);
}
// The last `n_stage` of `issued` copies; the first that does not come, seconds later, ends it.
__device__ __forceinline__ void ring_settle_warp(const uint64_t* full, int n_stage, int issued, int* status) {
    for (int q = max(0, issued - n_stage); q < issued; ++q)
        if (!mbar_settle_warp(smem_u32(&full[q % n_stage]), (q / n_stage) & 1, status)) break;
}
__device__ __forceinline__ void expect_tx_on(uint32_t on, uint32_t bar, uint32_t bytes) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes), "r"(on) : "memory");
}
__device__ __forceinline__ void bulk_g2s_on(uint32_t on, uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@p cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
        ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(on) : "memory");
}
__device__ __forceinline__ void tma_2d_on(uint32_t on, uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@p cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"(on) : "memory");
}
__device__ __forceinline__ void tc_commit_on(uint32_t on, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(on) : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void tc_cp_scales(uint32_t on, uint32_t taddr, uint64_t desc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "@p tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(desc), "r"(on) : "memory");
}
__device__ __forceinline__ void tc_mma_mxf4(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                            uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %7, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@p tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], q;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(on) : "memory");
}
// Both kinds of descriptor count the address in units of 16 bytes in their low bits: `bytes` further on.
__device__ __forceinline__ uint64_t desc_at(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }
// Instruction descriptor of kind::mxf4: E2M1 x E2M1, K-major, UE8M0 scales, M = 128, N = n; `id` (0 or 2) selects the
// upper or lower two scales of a 32-bit column for both operands.
__device__ __forceinline__ uint32_t idesc_mxf4(int n, int id) {
    return ((uint32_t)id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) |
           ((uint32_t)id << 29);
}

// The same on a pair of CTAs (cta_group::2): M = 256, 128 rows of A and half of B's rows in each CTA's shared memory; the
// scales of A's own rows and of all of B's in each CTA's tensor memory.  One thread of the leader issues for both.
__device__ __forceinline__ void tc_cp_scales_pair(uint32_t on, uint32_t taddr, uint64_t desc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "@p tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(desc), "r"(on) : "memory");
}
__device__ __forceinline__ void tc_mma_mxf4_pair(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                                 uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %7, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@p tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], q;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(on) : "memory");
}
__device__ __forceinline__ void tma_2d_pair_on(uint32_t on, uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t cluster_bar) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@p cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(cluster_bar), "r"(on) : "memory");
}
__device__ __forceinline__ void tc_commit_pair_on(uint32_t on, uint32_t bar) {
    const uint16_t mask = 3;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "@p tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
        ::"r"(bar), "h"(mask), "r"(on) : "memory");
}
__device__ __forceinline__ uint32_t idesc_mxf4_pair(int n, int id) { return idesc_mxf4(n, id) + (1u << 27); }   // M = 256

}  // namespace saem

#endif  // SAEM_MX_TC_CUH_
