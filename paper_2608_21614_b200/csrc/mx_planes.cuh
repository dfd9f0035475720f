// Activations for the block-scaled tensor cores without rounding them to 4 bits: five microscaled 4-bit planes.
//
// A block of 32 elements of a row is scaled by the power of two that brings its largest element into [2, 4).  Plane 0 is
// that rounded to E2M1; what is left, at most half a unit, is multiplied by 8 and so is in [-4, 4] again: the next plane,
// with an eighth of the scale.  Every step is exact in fp32 but for the roundings that the next plane takes up, so five
// planes hold a block to 2^-14 of its largest element at worst -- between bf16's 2^-9 of every element and fp32 -- and
// only the first needs a maximum over the block.  (With a maximum for each plane, six planes reached the same; the chain
// of shuffles took 1.5 us per 256 elements of a row.)  The planes are five columns of the MMA's N instead of one, of
// which a decode batch leaves most unused anyway, and their fp32 accumulators are added in the epilogue.  A block with an
// infinity or NaN becomes NaN.
//
// A tile is R rows x 256 elements as the MMA wants them: swizzled codes of 5 R columns (plane p of row r is column p R + r;
// rounded up to 16), then the 512-byte pieces of their scales, [column / 128][128 elements].
#ifndef SAEM_MX_PLANES_CUH_
#define SAEM_MX_PLANES_CUH_

#include "mx_tc.cuh"

namespace saem {

constexpr int kPlanes = 5;

template <int R>
struct TileShape {
    static constexpr int kN = (kPlanes * R + 15) / 16 * 16;                 // MMA columns
    static constexpr int kPieces = (kN + 127) / 128;
    static constexpr int kBytes = kN * 128 + kPieces * 2 * kMxPiece;        // one tile x 256 elements
    static constexpr int kScaleCols = 8 * kPieces;                          // tensor-memory columns of its scales
};
// Scale byte of plane 0, from the block's largest magnitude; plane p has kPlaneStep p less (no codes below 0).
constexpr int kPlaneStep = 3;
__device__ __forceinline__ int plane_scale_byte(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23);
    return e == 255 ? 255 : e > 1 ? e - 1 : 0;
}
__device__ __forceinline__ float inverse_power(int byte) {                  // of 2^(byte - 127); 0 for NaN's 255, whose codes are 0
    return byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23);
}

// Two values to a byte of codes (the first one low), and back.
__device__ __forceinline__ uint16_t encode2(float lo, float hi) {
    uint16_t b;
    asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %2, %1;\n\tmov.b16 %0, {c, 0};\n\t}" : "=h"(b) : "f"(lo), "f"(hi));
    return b;
}
__device__ __forceinline__ float2 decode2(uint16_t b) {
    uint32_t h;
    asm("{\n\t.reg .b8 c, z;\n\tmov.b16 {c, z}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(h) : "h"(b));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Eight bf16 values.
__device__ __forceinline__ void widen8(uint4 q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}
// 256 elements of a row, eight per lane, four lanes per block: the lane's codes in each plane, and the scales of the
// lane's 128 elements as a word.
__device__ __forceinline__ void split_planes(float (&v)[8], int lane, uint32_t (&codes)[kPlanes], uint32_t (&scales)[kPlanes]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const int sb = plane_scale_byte(m);
    const float up = inverse_power(sb);
    uint32_t word = (uint32_t)sb << (((lane >> 2) & 3) * 8);
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = sb == 255 ? 0.f : v[j] * up;
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t code = encode2(v[2 * j], v[2 * j + 1]);
            const float2 back = decode2((uint16_t)code);
            v[2 * j] = (v[2 * j] - back.x) * 8.f;
            v[2 * j + 1] = (v[2 * j + 1] - back.y) * 8.f;
            w |= code << (8 * j);
        }
        codes[p] = sb >= kPlaneStep * p ? w : 0u;
        scales[p] = __vsubus4(word, 0x01010101u * (kPlaneStep * p));         // per byte, not below 0
    }
}
// What split_planes made, to row r of the tile at dst.
template <int R>
__device__ __forceinline__ void store_tile_row(uint8_t* dst, int r, int lane, const uint32_t (&codes)[kPlanes], const uint32_t (&scales)[kPlanes]) {
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        const int n = p * R + r;
        *reinterpret_cast<uint32_t*>(dst + n * 128 + (((lane >> 2) ^ (n & 7)) << 4) + (lane & 3) * 4) = codes[p];
        if ((lane & 15) == 0)
            *reinterpret_cast<uint32_t*>(dst + TileShape<R>::kN * 128 + ((n >> 7) * 2 + (lane >> 4)) * kMxPiece + (n & 31) * 16 +
                                         ((n >> 5) & 3) * 4) = scales[p];
    }
}
// Eight rows' hidden units of one block (a lane holds one unit of each row) to the planes of rows r0 .. r0 + 7 of a tile.
template <int R>
__device__ __forceinline__ void store_planes(float (&v)[8], int r0, int rows, uint8_t* dst, int blk, int lane) {
    using T = TileShape<R>;
    const int mine = r0 + (lane & 7);                                          // the row whose codes this lane stores
    int sb[8], my_scale = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) sb[q] = plane_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v[q]) & 0x7FFFFFFFu));
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        v[q] = sb[q] == 255 ? 0.f : v[q] * inverse_power(sb[q]);
        if ((lane & 7) == q) my_scale = sb[q];
    }
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t w = 0;
#pragma unroll
        for (int q = 0; q < 8; q += 2) {                                       // two rows share a conversion
            const uint32_t code = encode2(v[q], v[q + 1]);
            const float2 back = decode2((uint16_t)code);
            v[q] = (v[q] - back.x) * 8.f;
            v[q + 1] = (v[q + 1] - back.y) * 8.f;
            w |= code << (4 * q);
        }
        // eight rows' codes of one unit to eight units' codes of one row: a transposition over eight lanes
#pragma unroll
        for (int s = 4; s > 0; s >>= 1) {
            const uint32_t low = s == 4 ? 0x0000FFFFu : s == 2 ? 0x00FF00FFu : 0x0F0F0F0Fu;
            const uint32_t o = __shfl_xor_sync(0xffffffffu, w, s);
            w = lane & s ? (w & ~low) | ((o >> (4 * s)) & low) : (w & low) | ((o << (4 * s)) & ~low);
        }
        const int col = p * R + mine, scale = my_scale - kPlaneStep * p;
        if (mine < rows) {
            *reinterpret_cast<uint32_t*>(dst + col * 128 + ((blk ^ (col & 7)) << 4) + (lane >> 3) * 4) = scale >= 0 ? w : 0u;
            if (lane < 8)
                dst[T::kN * 128 + ((col >> 7) * 2 + (blk >> 2)) * kMxPiece + (col & 31) * 16 + ((col >> 5) & 3) * 4 + (blk & 3)] =
                    (uint8_t)max(scale, 0);
        }
    }
}

// Eight columns of this warp's 32 lanes, no wait.
__device__ __forceinline__ void tc_ld8_issue(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
}
// Sum over the planes of eight rows' columns from `taddr` on (planes R columns apart).
template <int R>
__device__ __forceinline__ void plane_sums(uint32_t taddr, float (&v)[8]) {
    uint32_t r[kPlanes][8];
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) tc_ld8_issue(taddr + p * R, r[p]);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        asm volatile("" : "+r"(r[0][i]), "+r"(r[1][i]), "+r"(r[2][i]), "+r"(r[3][i]), "+r"(r[4][i]) :: "memory");
        v[i] = 0.f;
#pragma unroll
        for (int p = kPlanes - 1; p >= 0; --p) v[i] += __uint_as_float(r[p][i]);   // the small planes first
    }
}


}  // namespace saem

#endif  // SAEM_MX_PLANES_CUH_
