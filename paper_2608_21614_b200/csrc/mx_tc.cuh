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
// The issuing warp runs its loop as a whole, operands in uniform registers, and one elected lane (`on`) issues: inside an
// `if (lane == 0)` every operand has to be moved to a uniform register first, and an instruction took some 80 cycles to
// issue (an MMA of 128 x 48 x 64 takes 44, a scale copy 8).
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
// Instruction descriptor of kind::mxf4: E2M1 x E2M1, K-major, UE8M0 scales, M = 128, N = n; `id` (0 or 2) selects the
// upper or lower two scales of a 32-bit column for both operands.
__device__ __forceinline__ uint32_t idesc_mxf4(int n, int id) {
    return ((uint32_t)id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) |
           ((uint32_t)id << 29);
}

}  // namespace saem

#endif  // SAEM_MX_TC_CUH_
