// The microscaled 4-bit format (MXFP4) as the kernels see it.
//
// 32 consecutive elements of a row form a block with one power of two 2^(s - 127) (s: one byte, 255 = NaN); an
// element is an E2M1 code of four bits: sign, then 0 .5 1 1.5 2 3 4 6.  Element 2i of a row is the low half of byte i.
//
//   codes  [rows][ceil(cols / 32) * 16 bytes]   row-major, the last block padded with zeros
//   scales [ceil(rows / 128)][ceil(cols / 128)][512 bytes]   one 512-byte piece per 128 rows x 4 blocks: the four
//          scales of row r (mod 128) are the 32-bit word at (r % 32) * 16 + (r / 32) * 4.  That is the order in which
//          tcgen05.cp (32x128b) lays them into tensor memory for the block-scaled MMA, so that a piece is copied as is.
#ifndef SAEM_MX_COMMON_CUH_
#define SAEM_MX_COMMON_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "saem_internal.h"

namespace saem {

constexpr int kMxBlock = 32;                // elements of a block
constexpr int kMxSpan = 128;                // elements of four blocks: one 32-bit word of scales
constexpr int kMxPiece = 512;               // bytes of the scales of 128 rows x kMxSpan elements

// A packed expert (the slot layout of SAEM_FFN_MX contexts) is a sequence of blocks of 128 weight rows x 256 elements,
// 17 KB each and read with one bulk copy: 128 bytes of codes per row, 16-byte chunks XOR-swizzled by (row mod 8) as the
// tensor cores want them, then the two 512-byte pieces of the scales.  Gate/up region: [d_ff / 128][ceil(d_model / 256)] of a
// gate block and the up block of the same place; down region: [d_model / 128][ceil(d_ff / 256)].  Where the row's length is
// an odd multiple of 128, the second half of its last block is zero.
constexpr int kMxChunk = 256;               // elements of a block's rows
constexpr int kMxBlockCodes = 128 * 128;
constexpr int kMxBlockBytes = kMxBlockCodes + 2 * kMxPiece;

__host__ __device__ inline size_t mx_scale_word(long long row, long long span, long long n_span) {
    return ((size_t)(row >> 7) * n_span + span) * kMxPiece + (size_t)(row & 31) * 16 + ((row >> 5) & 3) * 4;
}
__host__ __device__ inline int mx_chunks(int k) { return (k + kMxChunk - 1) / kMxChunk; }
__host__ __device__ inline size_t mx_gate_up_blocks(int d, int f) { return (size_t)(f / 128) * mx_chunks(d) * 2; }
__host__ __device__ inline size_t mx_down_blocks(int d, int f) { return (size_t)(d / 128) * mx_chunks(f); }

#ifdef __CUDACC__
// The four pairs of E2M1 values of a word of eight codes, low codes first.
__device__ __forceinline__ void mx_decode8(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// Sum of the two products of two bytes of codes (low with low, high with high).
__device__ __forceinline__ float mx_dot2(uint32_t u, uint32_t v) {
    uint32_t a, b;
    asm("{\n\t.reg .b8 c;\n\tcvt.u8.u32 c, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(a) : "r"(u));
    asm("{\n\t.reg .b8 c;\n\tcvt.u8.u32 c, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(b) : "r"(v));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
    return x.x * y.x + x.y * y.y;
}
// Eight fp32 values (already divided by the block's scale) to codes: nearest, ties to even, saturated at 6.
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8]) {
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
// Scale byte of a block whose largest magnitude has these fp32 bits: floor(log2) - 2, so that the largest element
// lands in [4, 8) and saturates at 6 at worst; 255 if it is not finite.
__device__ __forceinline__ int mx_scale_byte(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23);
    return e == 255 ? 255 : (e > 2 ? e - 2 : 0);
}
// Eight elements of a row from `col` on as fp32; what lies beyond `cols` is zero.  VEC: the row is 16-byte aligned.
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void* __restrict__ row, long long col, long long cols, float (&v)[8]) {
    if (VEC && col + 8 <= cols) {
        if (BF16) {
            const uint4 q = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + col));
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(row) + col);
            const float4 a = __ldcs(p), b = __ldcs(p + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
            if (col + i < cols)
                v[i] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[col + i] << 16)
                            : static_cast<const float*>(row)[col + i];
        }
    }
}
// Eight elements of a block that four neighbouring lanes share to their codes, and the block's scale byte.
__device__ __forceinline__ uint32_t mx_quantize8(const float (&v)[8], int& scale) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7FFFFFFFu);   // NaN above infinity
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    scale = mx_scale_byte(amax);
    const float inv = __uint_as_float((uint32_t)(254 - min(scale, 253)) << 23);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = v[i] * inv;
    return scale == 255 ? 0u : mx_encode8(u);
}
#endif

}  // namespace saem

#endif  // SAEM_MX_COMMON_CUH_
