// Activations for the block-scaled tensor cores without rounding them to 4 bits: five microscaled 4-bit planes.
//
// A block of 32 elements of a row is scaled by the power of two that brings its largest element into [1.7, 3.41) and each
// element v is rounded once, to a multiple of 2^-12 -- 2^-13.8 of the block's largest at worst, between bf16's 2^-9 of
// every element and fp32.  The integer 4096 v is written in radix 8 with digits d_0 .. d_4 of -4 .. 3,
//     v = d_0 + d_1 / 8 + d_2 / 64 + d_3 / 512 + d_4 / 4096,
// (at most 3.42) all of which E2M1 holds: plane p is the codes of d_p with 1 / 8^p of the scale.  The planes are five columns of the
// MMA's N instead of one, of which a decode batch leaves most unused anyway, and their fp32 accumulators are added in the
// epilogue.  One FMA with a large constant rounds an element and biases it so that its digits + 4 are plain bit fields;
// a byte permutation looks four of them up at a time.  A block with an infinity or NaN becomes NaN.
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
    const int e = (int)(amax_bits >> 23) + ((amax_bits & 0x7FFFFFu) >= 0x5A0000u ? 1 : 0);   // 1.703 * 2^e on
    return amax_bits >= 0x7F800000u ? 255 : max(e - 1, 0);
}
__device__ __forceinline__ float inverse_power(int byte) {                  // of 2^(byte - 127)
    return byte == 254 ? __uint_as_float(1u << 22) : __uint_as_float((uint32_t)(254 - byte) << 23);
}
// An element (already divided by its scale) rounded to 2^-12: digit p plus 4 is bits 12 - 3 p and up.  The constant is
// 1.5 * 2^23 and 4 in every digit.
__device__ __forceinline__ uint32_t plane_digits(float v) { return __float_as_uint(fmaf(v, 4096.f, 12582912.f + 18724.f)); }
// Eight elements' digits to a word of eight codes for each plane.
__device__ __forceinline__ void plane_words(const uint32_t (&y)[8], uint32_t (&w)[kPlanes]) {
    uint32_t pair[4];                                                        // elements j and j + 4
#pragma unroll
    for (int j = 0; j < 4; ++j) pair[j] = __byte_perm(y[j], y[j + 4], 0x5410);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        const int at = 12 - 3 * p;
        uint32_t sel = 0;                                                    // digits + 4 as selectors, elements 0-3 low, 4-7 high
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int up = 4 * j - at;
            sel |= (up >= 0 ? pair[j] << up : pair[j] >> -up) & (0x00070007u << (4 * j));
        }
        // E2M1 codes of -4 .. 3
        uint32_t lo = __byte_perm(0x0A0C0D0Eu, 0x05040200u, sel), hi = __byte_perm(0x0A0C0D0Eu, 0x05040200u, sel >> 16);
        lo |= lo >> 4;                                                       // bytes 0 and 2: two codes each
        hi |= hi >> 4;
        w[p] = __byte_perm(lo, hi, 0x6420);
    }
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
__device__ __forceinline__ void split_planes(const float (&v)[8], int lane, uint32_t (&codes)[kPlanes], uint32_t (&scales)[kPlanes]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const int sb = plane_scale_byte(m);
    const float up = inverse_power(min(sb, 254));
    uint32_t word = (uint32_t)sb << (((lane >> 2) & 3) * 8);
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    uint32_t y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = plane_digits(sb == 255 ? 0.f : v[j] * up);
    plane_words(y, codes);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        if (sb < kPlaneStep * p) codes[p] = 0u;
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
// The fast exponential's documented bound grows with its argument, 2 + 1.17 |z| units in the last place: 2^-21 of the result
// for z near 0, 2^-18 at z = -20 and 2^-16 at z = -80, below what the planes keep of a block's largest element.  Below
// z = -87.3, where the quotient is less than 2^-126 of z, it is 0.
__device__ __forceinline__ float swiglu(float z, float up) { return __fdividef(z, 1.f + __expf(-z)) * up; }
// Eight rows' hidden units of one block (a lane holds one unit of each row) to the planes of rows r0 .. r0 + 7 of a tile.
template <int R>
__device__ __forceinline__ void store_planes(const float (&v)[8], int r0, int rows, uint8_t* dst, int blk, int lane) {
    using T = TileShape<R>;
    const int mine = r0 + (lane & 7);                                          // the row whose codes this lane stores
    int my_scale = 0;
    uint32_t y[8], codes[kPlanes];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        y[q] = 0;
        if (r0 + q >= rows) continue;
        const int sb = plane_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v[q]) & 0x7FFFFFFFu));
        y[q] = plane_digits(sb == 255 ? 0.f : v[q] * inverse_power(min(sb, 254)));
        if ((lane & 7) == q) my_scale = sb;
    }
    plane_words(y, codes);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t w = codes[p];
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
