// Activations for the block-scaled tensor cores without rounding them to 4 bits: six microscaled 4-bit planes.
//
// Plane 0 is a row's block of 32 elements rounded to E2M1 with a scale that reaches its largest element, plane p the same
// of what planes 0 .. p - 1 left (exact in fp32).  Each plane leaves at most a fifth of the block's largest, so that six
// hold a block to 2^-14 of its largest element (2^-17 typically), between bf16's 2^-9 of every element and fp32.  The
// planes are six more columns of the MMA's N -- rows x 6 columns, of which a decode batch leaves most unused anyway --
// and their fp32 accumulators are added in the epilogue.  A block with an infinity or NaN becomes NaN.
//
// A tile is R rows x 256 elements as the MMA wants them: swizzled codes of kPlanes * R columns (plane p of row r is column
// p R + r), then the 512-byte pieces of their scales, [column / 128][128 elements].
#ifndef SAEM_MX_PLANES_CUH_
#define SAEM_MX_PLANES_CUH_

#include "mx_tc.cuh"

namespace saem {

constexpr int kPlanes = 6;

template <int R>
struct TileShape {
    static constexpr int kN = kPlanes * R;                                  // MMA columns: plane p of row r is column p R + r
    static constexpr int kPieces = (kN + 127) / 128;
    static constexpr int kBytes = kN * 128 + kPieces * 2 * kMxPiece;        // one tile x 256 elements
    static constexpr int kScaleCols = 8 * kPieces;                          // tensor-memory columns of its scales
};
// Scale byte of a plane: the power of two that brings the block's largest magnitude into (3, 6].
__device__ __forceinline__ int plane_scale_byte(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23);
    if (e == 255) return 255;
    const int s = (e > 2 ? e - 2 : 0) + ((amax_bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
    return s < 254 ? s : 254;
}
__device__ __forceinline__ float power_of_two(int byte) { return __uint_as_float(byte ? (uint32_t)byte << 23 : 1u << 22); }
__device__ __forceinline__ float inverse_power(int byte) {                  // of 2^(byte - 127)
    return byte == 254 ? __uint_as_float(1u << 22) : __uint_as_float((uint32_t)(254 - byte) << 23);
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
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const int sb = plane_scale_byte(m);
        const float up = inverse_power(min(sb, 254)), down = power_of_two(sb);
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = v[j] * up;
        codes[p] = sb == 255 ? 0u : mx_encode8(u);
        uint32_t h[4];
        mx_decode8(codes[p], h);
#pragma unroll
        for (int j = 0; j < 4; ++j) {                                    // what is left: exact in fp32
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
            v[2 * j] = sb == 255 ? 0.f : v[2 * j] - f.x * down;
            v[2 * j + 1] = sb == 255 ? 0.f : v[2 * j + 1] - f.y * down;
        }
        uint32_t word = (uint32_t)sb << (((lane >> 2) & 3) * 8);
        word |= __shfl_xor_sync(0xffffffffu, word, 4);
        word |= __shfl_xor_sync(0xffffffffu, word, 8);
        scales[p] = word;
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
// Eight rows' hidden units of one block (a lane holds one unit of each row) to the planes of tile columns r0 .. r0 + 7.
template <int R>
__device__ __forceinline__ void store_planes(float (&v)[8], int r0, int rows, uint8_t* dst, int blk, int lane) {
    using T = TileShape<R>;
    const int mine = r0 + (lane & 7);                                          // the row whose codes this lane stores
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t w = 0, bytes = 0;
#pragma unroll
        for (int q = 0; q < 8; q += 2) {                                       // two rows share a conversion
            int sb[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                sb[z] = plane_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(v[q + z]) & 0x7FFFFFFFu));
                if ((lane & 7) == q + z) bytes = (uint32_t)sb[z];
            }
            uint32_t code = encode2(v[q] * inverse_power(min(sb[0], 254)), v[q + 1] * inverse_power(min(sb[1], 254)));
            const float2 back = decode2((uint16_t)code);
            v[q] = sb[0] == 255 ? 0.f : v[q] - back.x * power_of_two(sb[0]);   // what is left: exact in fp32
            v[q + 1] = sb[1] == 255 ? 0.f : v[q + 1] - back.y * power_of_two(sb[1]);
            w |= code << (4 * q);                                              // codes under a NaN scale do not matter
        }
        // eight rows' codes of one unit to eight units' codes of one row: a transposition over eight lanes
#pragma unroll
        for (int s = 4; s > 0; s >>= 1) {
            const uint32_t low = s == 4 ? 0x0000FFFFu : s == 2 ? 0x00FF00FFu : 0x0F0F0F0Fu;
            const uint32_t o = __shfl_xor_sync(0xffffffffu, w, s);
            w = lane & s ? (w & ~low) | ((o >> (4 * s)) & low) : (w & low) | ((o << (4 * s)) & ~low);
        }
        const int col = p * R + mine;
        if (mine < rows) {
            *reinterpret_cast<uint32_t*>(dst + col * 128 + ((blk ^ (col & 7)) << 4) + (lane >> 3) * 4) = w;
            if (lane < 8)
                dst[T::kN * 128 + ((col >> 7) * 2 + (blk >> 2)) * kMxPiece + (col & 31) * 16 + ((col >> 5) & 3) * 4 + (blk & 3)] = (uint8_t)bytes;
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
        asm volatile("" : "+r"(r[0][i]), "+r"(r[1][i]), "+r"(r[2][i]), "+r"(r[3][i]), "+r"(r[4][i]), "+r"(r[5][i]) :: "memory");
        v[i] = 0.f;
#pragma unroll
        for (int p = kPlanes - 1; p >= 0; --p) v[i] += __uint_as_float(r[p][i]);   // the small planes first
    }
}


}  // namespace saem

#endif  // SAEM_MX_PLANES_CUH_
