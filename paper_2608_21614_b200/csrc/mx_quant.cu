// The microscaled 4-bit format: quantisation, the way back, and the packing of quantised expert matrices into slots.
//
// Quantisation of a block: s = max(floor(log2 max|x|) - 2, -127), code = E2M1(x * 2^-s) to the nearest (ties to the
// even mantissa), saturated at 6.  Both the scaling and the way back are exact, so the only rounding is the one to E2M1.
// All kernels here read and write every byte once and are bound by DRAM (2.5 or 4.5 bytes per element) -- if the
// instructions per element stay few: a lane takes 16 elements of bf16 (half a block; its maximum is found in packed
// halves and scaled in packed halves) or 8 of fp32, 32 bytes in one access, and a warp four such pieces of one row, whose
// loads go out together.  14336 x 4096 in bf16, there and back: 48 us for 297 MB, 6.2 TB/s (59 us with 16-byte accesses,
// 90 us with 8 elements per lane and one block at a time).
#include <cmath>
#include <cstring>

#include "mx_common.cuh"

namespace saem {

constexpr int kQuantThreads = 256;
constexpr int kQuantUnroll = 4;             // pieces (1 KB of the row) that a warp takes, whose loads go out together

// Rows that do not begin at 32-byte addresses: a piece (1 KB) is read and written by consecutive lanes, word by word (bf16 at
// odd addresses: element by element), and changes hands in shared memory, so that an access touches four or five lines and
// not thirty-two (777 x 2501 fp32, there and back: 6.3 us against 13.9 us).
template <bool BF16>
__device__ __forceinline__ void load_piece(const uint8_t* row, long long first, long long cols, bool words, int lane, uint32_t (&v)[8]) {
    if (!BF16) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + first;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = first + 32 * i + lane < cols ? p[32 * i + lane] : 0u;
        return;
    }
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + first;
    if (words) {                                                              // pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = 64 * i + 2 * lane;
            v[i] = first + at + 1 < cols ? *reinterpret_cast<const uint32_t*>(p + at) : first + at < cols ? p[at] : 0u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = 64 * i + lane;
            const uint32_t lo = first + at < cols ? p[at] : 0u, hi = first + at + 32 < cols ? p[at + 32] : 0u;
            v[i] = lo | hi << 16;
        }
    }
}
// From what load_piece gave to the 32 bytes that are the lane's own.
template <bool BF16>
__device__ __forceinline__ void take_piece(uint4* stage, bool words, int lane, uint32_t (&v)[8]) {
    if (words) {
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<uint32_t*>(stage)[32 * i + lane] = v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            reinterpret_cast<uint16_t*>(stage)[64 * i + lane] = (uint16_t)v[i];
            reinterpret_cast<uint16_t*>(stage)[64 * i + lane + 32] = (uint16_t)(v[i] >> 16);
        }
    }
    __syncwarp();
    const uint4 a = stage[2 * lane], b = stage[2 * lane + 1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    __syncwarp();
}
// The way back: from the lane's own 32 bytes to the row.
template <bool BF16>
__device__ __forceinline__ void store_piece(uint4* stage, uint8_t* row, long long first, long long cols, bool words, int lane, const uint32_t (&o)[8]) {
    stage[2 * lane] = make_uint4(o[0], o[1], o[2], o[3]);
    stage[2 * lane + 1] = make_uint4(o[4], o[5], o[6], o[7]);
    __syncwarp();
    if (!BF16) {
        uint32_t* p = reinterpret_cast<uint32_t*>(row) + first;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (first + 32 * i + lane < cols) p[32 * i + lane] = reinterpret_cast<const uint32_t*>(stage)[32 * i + lane];
    } else if (words) {
        uint16_t* p = reinterpret_cast<uint16_t*>(row) + first;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = 64 * i + 2 * lane;
            const uint32_t w = reinterpret_cast<const uint32_t*>(stage)[32 * i + lane];
            if (first + at + 1 < cols) *reinterpret_cast<uint32_t*>(p + at) = w;
            else if (first + at < cols) p[at] = (uint16_t)w;
        }
    } else {
        uint16_t* p = reinterpret_cast<uint16_t*>(row) + first;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (first + 32 * i + lane < cols) p[32 * i + lane] = reinterpret_cast<const uint16_t*>(stage)[32 * i + lane];
    }
    __syncwarp();
}

template <bool BF16, bool VEC, int UNROLL>
__global__ void __launch_bounds__(kQuantThreads)
mx_quantize_kernel(const void* __restrict__ x, uint32_t rows, long long cols, long long row_stride, uint32_t n_strip,
                   uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    constexpr int kPerLane = BF16 ? 16 : 8, kPiece = 32 * kPerLane, kLanes = kMxBlock / kPerLane;   // kLanes share a block
    __shared__ uint4 stage[VEC ? 1 : kQuantThreads / 32][64];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5), row = unit / n_strip;
    if (row >= rows) return;
    const long long n_block = (cols + kMxBlock - 1) / kMxBlock, n_span = (cols + kMxSpan - 1) / kMxSpan;
    const long long col0 = (long long)(unit - row * n_strip) * (UNROLL * kPiece) + lane * kPerLane;
    const uint8_t* src = static_cast<const uint8_t*>(x) + (size_t)row * row_stride * (BF16 ? 2 : 4);
    uint8_t* dst = codes + (size_t)row * n_block * 16;
    uint8_t* sdst = scales + mx_scale_word(row, 0, n_span);
    // bf16: eight words of two elements; fp32: eight elements
    uint32_t v[UNROLL][8];
    const bool words = !BF16 || ((uintptr_t)src & 3) == 0;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const long long col = col0 + u * kPiece, first = col - lane * kPerLane;
        if (!VEC) {
            load_piece<BF16>(src, first, cols, words, lane, v[u]);
        } else if (col + kPerLane <= cols) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(v[u][0]), "=r"(v[u][1]), "=r"(v[u][2]), "=r"(v[u][3]), "=r"(v[u][4]), "=r"(v[u][5]), "=r"(v[u][6]), "=r"(v[u][7])
                         : "l"(src + col * (BF16 ? 2 : 4)));
        } else if (BF16) {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(src);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t lo = col + 2 * i < cols ? p[col + 2 * i] : 0u, hi = col + 2 * i + 1 < cols ? p[col + 2 * i + 1] : 0u;
                v[u][i] = lo | hi << 16;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = col + i < cols ? reinterpret_cast<const uint32_t*>(src)[col + i] : 0u;
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const long long col = col0 + u * kPiece;
        if (col0 - lane * kPerLane + u * kPiece >= n_span * kMxSpan) break;   // the same in every lane
        if (!VEC) take_piece<BF16>(stage[threadIdx.x >> 5], words, lane, v[u]);
        uint32_t m = 0;                                                       // largest magnitude's bits, NaN above infinity
        if (BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) m = __vmaxu2(m, v[u][i] & 0x7FFF7FFFu);
            m = max(m << 16, m & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, v[u][i] & 0x7FFFFFFFu);
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const int s = mx_scale_byte(m);
        const uint32_t inv = (uint32_t)(254 - min(s, 253)) << 7;              // 2^(127 - s) in bf16
        const bool in = col < n_block * kMxBlock;
        if (BF16) {
            const uint32_t inv2 = inv | inv << 16;
            uint32_t w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // by a power of two: exact, but for elements so far below the block's largest that they round to 0
                    const __nv_bfloat162 q = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v[u][4 * h + i]),
                                                     *reinterpret_cast<const __nv_bfloat162*>(&inv2));
                    const uint32_t b = *reinterpret_cast<const uint32_t*>(&q);
                    f[2 * i] = __uint_as_float(b << 16);
                    f[2 * i + 1] = __uint_as_float(b & 0xFFFF0000u);
                }
                w[h] = s == 255 ? 0u : mx_encode8(f);
            }
            if (in) *reinterpret_cast<uint2*>(dst + col / 2) = make_uint2(w[0], w[1]);
        } else {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[u][i]) * __uint_as_float(inv << 16);
            if (in) *reinterpret_cast<uint32_t*>(dst + col / 2) = s == 255 ? 0u : mx_encode8(f);
        }
        // the four scales of a 128-element span meet in one word; blocks beyond the row's last one get scale 2^-127
        uint32_t word = in ? (uint32_t)s << ((lane / kLanes & 3) * 8) : 0u;
        word |= __shfl_xor_sync(0xffffffffu, word, kLanes);
        word |= __shfl_xor_sync(0xffffffffu, word, 2 * kLanes);
        const long long span = col / kMxSpan;
        if (lane % (4 * kLanes) == 0 && span < n_span) *reinterpret_cast<uint32_t*>(sdst + span * kMxPiece) = word;
    }
}

template <bool BF16, bool VEC, int UNROLL>
__global__ void __launch_bounds__(kQuantThreads)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint32_t rows, long long cols,
                     long long row_stride, uint32_t n_strip, void* __restrict__ out) {
    constexpr int kPerLane = BF16 ? 16 : 8, kPiece = 32 * kPerLane;
    __shared__ uint4 stage[VEC ? 1 : kQuantThreads / 32][64];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5), row = unit / n_strip;
    if (row >= rows) return;
    const long long n_block = (cols + kMxBlock - 1) / kMxBlock, n_span = (cols + kMxSpan - 1) / kMxSpan;
    const long long col0 = (long long)(unit - row * n_strip) * (UNROLL * kPiece) + lane * kPerLane;
    const uint8_t* src = codes + (size_t)row * n_block * 16;
    const uint8_t* ssrc = scales + mx_scale_word(row, 0, n_span);
    uint2 w[UNROLL];
    uint32_t s[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const long long col = col0 + u * kPiece;
        w[u] = make_uint2(0u, 0u);
        s[u] = 0;
        if (col < cols) {
            if (BF16) w[u] = __ldcs(reinterpret_cast<const uint2*>(src + col / 2));   // the row of codes is padded to whole blocks
            else w[u].x = __ldcs(reinterpret_cast<const uint32_t*>(src + col / 2));
            s[u] = ssrc[col / kMxSpan * kMxPiece + ((col / kMxBlock) & 3)];
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const long long col = col0 + u * kPiece;
        if (VEC ? col >= cols : col - lane * kPerLane >= cols) break;         // without VEC the same in every lane
        const float scale = s[u] == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(s[u] ? s[u] << 23 : 1u << 22);
        const size_t at = (size_t)row * row_stride + col;
        uint32_t o[8];                                                        // the lane's 32 bytes: 16 bf16 or 8 fp32
#pragma unroll
        for (int h = 0; h < kPerLane / 8; ++h) {
            uint32_t p[4];
            mx_decode8(h ? w[u].y : w[u].x, p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p[i]));
                f.x *= scale;
                f.y *= scale;
                if (BF16) {
                    const __nv_bfloat162 q = __float22bfloat162_rn(f);        // exact: one mantissa bit
                    o[4 * h + i] = *reinterpret_cast<const uint32_t*>(&q);
                } else {
                    o[2 * i] = __float_as_uint(f.x);
                    o[2 * i + 1] = __float_as_uint(f.y);
                }
            }
        }
        if (!VEC) {
            uint8_t* row_out = static_cast<uint8_t*>(out) + (size_t)row * row_stride * (BF16 ? 2 : 4);
            store_piece<BF16>(stage[threadIdx.x >> 5], row_out, col - lane * kPerLane, cols, !BF16 || ((uintptr_t)row_out & 3) == 0, lane, o);
        } else if (col + kPerLane <= cols) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(static_cast<uint8_t*>(out) + at * (BF16 ? 2 : 4)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]),
                         "r"(o[6]), "r"(o[7]) : "memory");
        } else if (BF16) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (col + i < cols) static_cast<uint16_t*>(out)[at + i] = (uint16_t)(o[i / 2] >> (16 * (i & 1)));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < cols) static_cast<uint32_t*>(out)[at + i] = o[i];
        }
    }
}

struct MxMatrix {
    const uint8_t* codes;
    const uint8_t* scales;
};

// Which matrix, row tile and chunk a block of the slot layout holds.
struct BlockPlace {
    int matrix, tile, chunk;                // matrix: 0 gate, 1 up, 2 down
};
__host__ __device__ inline BlockPlace block_place(size_t block, int d, int f) {
    const size_t n_gu = mx_gate_up_blocks(d, f);
    if (block < n_gu) {
        const int nc = mx_chunks(d);
        return {(int)(block & 1), (int)(block / 2 / nc), (int)(block / 2 % nc)};
    }
    const int nc = mx_chunks(f);
    return {2, (int)((block - n_gu) / nc), (int)((block - n_gu) % nc)};
}

// One CTA per block of the slot layout (mx_common.cuh).
__global__ void __launch_bounds__(kQuantThreads)
mx_pack_kernel(MxMatrix gate, MxMatrix up, MxMatrix down, int d, int f, uint8_t* __restrict__ out) {
    pdl_wait();
    pdl_launch_dependents();
    const BlockPlace at = block_place(blockIdx.x, d, f);
    const MxMatrix m = at.matrix == 0 ? gate : at.matrix == 1 ? up : down;
    const int K = at.matrix == 2 ? f : d, n_span = K / kMxSpan;
    uint8_t* dst = out + (size_t)blockIdx.x * kMxBlockBytes;
    for (int i = threadIdx.x; i < 128 * 8; i += kQuantThreads) {
        const int r = i >> 3, ch = i & 7, col = at.chunk * kMxChunk + ch * 32;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (col < K) v = *reinterpret_cast<const uint4*>(m.codes + (size_t)(at.tile * 128 + r) * (K / 2) + col / 2);
        *reinterpret_cast<uint4*>(dst + r * 128 + ((ch ^ (r & 7)) << 4)) = v;
    }
    for (int i = threadIdx.x; i < 2 * kMxPiece / 16; i += kQuantThreads) {
        const int span = at.chunk * 2 + i / (kMxPiece / 16);
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (span < n_span)
            v = reinterpret_cast<const uint4*>(m.scales + ((size_t)at.tile * n_span + span) * kMxPiece)[i % (kMxPiece / 16)];
        reinterpret_cast<uint4*>(dst + kMxBlockCodes)[i] = v;
    }
}

// ---- the same on the host, for experts that stay in pinned memory --------------------------------------------------
static uint8_t host_quantize_block(const uint16_t* x, uint8_t* codes16) {
    uint32_t amax = 0;
    float v[kMxBlock];
    for (int i = 0; i < kMxBlock; ++i) {
        const uint32_t b = (uint32_t)x[i] << 16;
        memcpy(&v[i], &b, 4);
        const uint32_t m = b & 0x7FFFFFFFu;
        amax = m > amax ? m : amax;
    }
    const int e = (int)(amax >> 23);
    memset(codes16, 0, 16);
    if (e == 255) return 255;
    const int s = e > 2 ? e - 2 : 0;
    for (int i = 0; i < kMxBlock; ++i) {
        const float a = std::ldexp(std::fabs(v[i]), 127 - s);
        const int c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
        codes16[i / 2] |= (uint8_t)((c | (std::signbit(v[i]) ? 8 : 0)) << (4 * (i & 1)));
    }
    return (uint8_t)s;
}

// The slot layout of one expert from bf16 matrices in host memory (see mx_pack_kernel).
void mx_pack_expert_host(const uint16_t* gate, const uint16_t* up, const uint16_t* down, int d, int f, uint8_t* out) {
    const size_t n = mx_gate_up_blocks(d, f) + mx_down_blocks(d, f);
    memset(out, 0, n * kMxBlockBytes);
    for (size_t block = 0; block < n; ++block) {
        const BlockPlace at = block_place(block, d, f);
        const uint16_t* m = at.matrix == 0 ? gate : at.matrix == 1 ? up : down;
        const int K = at.matrix == 2 ? f : d;
        uint8_t* dst = out + block * kMxBlockBytes;
        for (int r = 0; r < 128; ++r)
            for (int ch = 0; ch < 8; ++ch) {
                const int col = at.chunk * kMxChunk + ch * 32;
                if (col >= K) break;
                dst[kMxBlockCodes + (ch >> 2) * kMxPiece + (r & 31) * 16 + (r >> 5) * 4 + (ch & 3)] =
                    host_quantize_block(m + (size_t)(at.tile * 128 + r) * K + col, dst + r * 128 + ((ch ^ (r & 7)) << 4));
            }
    }
}

// Strips of a row, and CTAs for all of them.
// Pieces of a row per warp: one while they are few (some 28 warps per SM; 16 x 4096 bf16 there and back: 2.9 us against 3.7 us in
// fours), four beyond (1000 x 4096: 5.5 us against 5.8 us).
constexpr long long kQuantFew = 4096;
static long long pieces(long long cols, bool bf16) { return (cols + (bf16 ? 511 : 255)) / (bf16 ? 512 : 256); }
static bool few_pieces(long long rows, long long cols, bool bf16) { return rows <= kQuantFew && rows * pieces(cols, bf16) <= kQuantFew; }
static uint32_t strips(long long rows, long long cols, bool bf16) {
    const long long n = pieces(cols, bf16);
    return (uint32_t)(few_pieces(rows, cols, bf16) ? n : (n + kQuantUnroll - 1) / kQuantUnroll);
}
static dim3 strip_grid(long long rows, uint32_t n_strip) {
    return dim3((unsigned)(((unsigned long long)rows * n_strip + kQuantThreads / 32 - 1) / (kQuantThreads / 32)));
}
static bool vector_rows(const void* p, long long rows, long long row_stride, bool bf16) {
    return ((uintptr_t)p & 31) == 0 && (rows == 1 || row_stride * (bf16 ? 2 : 4) % 32 == 0);
}

}  // namespace saem

using namespace saem;

// rows, cols and the number of strips a kernel counts in 32 bits
static bool mx_shape_ok(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || rows > 0x7FFFFFFFll || cols > 0x7FFFFFFFll) return false;
    return rows * ((cols + 1023) / 1024) <= 0x7FFFFFFFll;
}

extern "C" {

size_t saem_mx_codes_bytes(int64_t rows, int64_t cols) {
    if (!mx_shape_ok(rows, cols)) return 0;
    return (size_t)rows * (size_t)((cols + kMxBlock - 1) / kMxBlock) * 16;
}

size_t saem_mx_scales_bytes(int64_t rows, int64_t cols) {
    if (!mx_shape_ok(rows, cols)) return 0;
    return (size_t)((rows + 127) / 128) * (size_t)((cols + kMxSpan - 1) / kMxSpan) * kMxPiece;
}

int saem_mx_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride, void* codes, void* scales,
                     void* stream) {
    if (dtype != SAEM_OUT_F32 && dtype != SAEM_OUT_BF16) return SAEM_ERR_INVALID_ARG;
    if (!mx_shape_ok(rows, cols) || (rows > 1 && row_stride < cols)) return SAEM_ERR_SHAPE;
    if (rows == 0) return SAEM_OK;
    if (!x || !codes || !scales) return SAEM_ERR_INVALID_ARG;
    if (((uintptr_t)codes | (uintptr_t)scales) & 15) return SAEM_ERR_ALIGNMENT;
    if ((uintptr_t)x % (dtype == SAEM_OUT_BF16 ? 2 : 4)) return SAEM_ERR_ALIGNMENT;
    const bool bf16 = dtype == SAEM_OUT_BF16, vec = vector_rows(x, rows, row_stride, bf16);
    const uint32_t n_strip = strips(rows, cols, bf16);
    constexpr int U = kQuantUnroll;
    auto k = few_pieces(rows, cols, bf16)
                 ? (bf16 ? (vec ? mx_quantize_kernel<true, true, 1> : mx_quantize_kernel<true, false, 1>)
                         : (vec ? mx_quantize_kernel<false, true, 1> : mx_quantize_kernel<false, false, 1>))
                 : (bf16 ? (vec ? mx_quantize_kernel<true, true, U> : mx_quantize_kernel<true, false, U>)
                         : (vec ? mx_quantize_kernel<false, true, U> : mx_quantize_kernel<false, false, U>));
    return launch_pdl(k, strip_grid(rows, n_strip), dim3(kQuantThreads), 0, (cudaStream_t)stream, x, (uint32_t)rows, (long long)cols,
                      (long long)row_stride, n_strip, (uint8_t*)codes, (uint8_t*)scales) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}

int saem_mx_dequantize(const void* codes, const void* scales, int64_t rows, int64_t cols, void* out, int dtype,
                       int64_t row_stride, void* stream) {
    if (dtype != SAEM_OUT_F32 && dtype != SAEM_OUT_BF16) return SAEM_ERR_INVALID_ARG;
    if (!mx_shape_ok(rows, cols) || (rows > 1 && row_stride < cols)) return SAEM_ERR_SHAPE;
    if (rows == 0) return SAEM_OK;
    if (!out || !codes || !scales) return SAEM_ERR_INVALID_ARG;
    if (((uintptr_t)codes | (uintptr_t)scales) & 15) return SAEM_ERR_ALIGNMENT;
    const bool bf16 = dtype == SAEM_OUT_BF16;
    if ((uintptr_t)out % (bf16 ? 2 : 4)) return SAEM_ERR_ALIGNMENT;
    const bool vec = vector_rows(out, rows, row_stride, bf16);
    const uint32_t n_strip = strips(rows, cols, bf16);
    constexpr int U = kQuantUnroll;
    auto k = few_pieces(rows, cols, bf16)
                 ? (bf16 ? (vec ? mx_dequantize_kernel<true, true, 1> : mx_dequantize_kernel<true, false, 1>)
                         : (vec ? mx_dequantize_kernel<false, true, 1> : mx_dequantize_kernel<false, false, 1>))
                 : (bf16 ? (vec ? mx_dequantize_kernel<true, true, U> : mx_dequantize_kernel<true, false, U>)
                         : (vec ? mx_dequantize_kernel<false, true, U> : mx_dequantize_kernel<false, false, U>));
    return launch_pdl(k, strip_grid(rows, n_strip), dim3(kQuantThreads), 0, (cudaStream_t)stream, (const uint8_t*)codes,
                      (const uint8_t*)scales, (uint32_t)rows, (long long)cols, (long long)row_stride, n_strip, out) == cudaSuccess
               ? SAEM_OK : SAEM_ERR_CUDA;
}

int saem_mx_pack_expert(const saem_config* cfg, const void* gate_codes, const void* gate_scales, const void* up_codes,
                        const void* up_scales, const void* down_codes, const void* down_scales, void* packed_out,
                        void* stream) {
    const int v = validate_config(cfg);
    if (v != SAEM_OK) return v;
    if (cfg->ffn_path != SAEM_FFN_MX) return SAEM_ERR_UNSUPPORTED;
    const void* p[7] = {gate_codes, gate_scales, up_codes, up_scales, down_codes, down_scales, packed_out};
    for (const void* q : p)
        if (!q) return SAEM_ERR_INVALID_ARG;
    for (const void* q : p)
        if ((uintptr_t)q & 15) return SAEM_ERR_ALIGNMENT;
    const size_t blocks = mx_gate_up_blocks(cfg->d_model, cfg->d_ff) + mx_down_blocks(cfg->d_model, cfg->d_ff);
    const MxMatrix g = {(const uint8_t*)gate_codes, (const uint8_t*)gate_scales};
    const MxMatrix u = {(const uint8_t*)up_codes, (const uint8_t*)up_scales};
    const MxMatrix d = {(const uint8_t*)down_codes, (const uint8_t*)down_scales};
    return launch_pdl(mx_pack_kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0,
                      (cudaStream_t)stream, g, u, d, cfg->d_model, cfg->d_ff, (uint8_t*)packed_out) == cudaSuccess
               ? SAEM_OK : SAEM_ERR_CUDA;
}

}  // extern "C"
