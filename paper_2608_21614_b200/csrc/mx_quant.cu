// The microscaled 4-bit format: quantisation, the way back, and the packing of quantised expert matrices into slots.
//
// Quantisation of a block: s = max(floor(log2 max|x|) - 2, -127), code = E2M1(x * 2^-s) to the nearest (ties to the
// even mantissa), saturated at 6.  Both the scaling and the way back are exact in fp32, so the only rounding is the one
// to E2M1.  All three kernels read and write every byte once and are bound by DRAM (2.5 or 4.5 bytes per element);
// four lanes share a block (8 elements and 16 or 32 bytes each), so that the loads and stores of a warp are whole
// lines and the block's maximum is two shuffles.
#include <cmath>
#include <cstring>

#include "mx_common.cuh"

namespace saem {

constexpr int kQuantThreads = 256;
constexpr int kQuantChunk = 256;            // elements of a row that one warp takes at a time
constexpr int kQuantUnroll = 4;             // chunks whose loads a warp has in flight

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kQuantThreads)
mx_quantize_kernel(const void* __restrict__ x, long long rows, long long cols, long long row_stride, uint32_t n_chunk,
                   uint32_t total, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const long long warp = (long long)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5);
    const long long n_block = (cols + kMxBlock - 1) / kMxBlock, n_span = (cols + kMxSpan - 1) / kMxSpan;
    const size_t esize = BF16 ? 2 : 4;
    float v[kQuantUnroll][8];
    uint32_t row[kQuantUnroll], ch[kQuantUnroll];
#pragma unroll
    for (int u = 0; u < kQuantUnroll; ++u) {
        const long long c = warp * kQuantUnroll + u;
        if (c < total) {
            row[u] = (uint32_t)c / n_chunk;
            ch[u] = (uint32_t)c - row[u] * n_chunk;
            load8<BF16, VEC>(static_cast<const uint8_t*>(x) + (size_t)row[u] * row_stride * esize,
                             (long long)ch[u] * kQuantChunk + lane * 8, cols, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kQuantUnroll; ++u) {
        if (warp * kQuantUnroll + u >= total) break;
        const long long col = (long long)ch[u] * kQuantChunk + lane * 8;
        int s;
        const uint32_t w = mx_quantize8(v[u], s);
        if (col / kMxBlock < n_block)
            *reinterpret_cast<uint32_t*>(codes + (size_t)row[u] * n_block * 16 + col / 2) = w;
        // the four scales of a 128-element span meet in one word; blocks beyond the row's last one get scale 2^-127
        uint32_t word = col / kMxBlock < n_block ? (uint32_t)s << (((lane >> 2) & 3) * 8) : 0u;
        word |= __shfl_xor_sync(0xffffffffu, word, 4);
        word |= __shfl_xor_sync(0xffffffffu, word, 8);
        const long long span = col / kMxSpan;
        if ((lane & 15) == 0 && span < n_span)
            *reinterpret_cast<uint32_t*>(scales + mx_scale_word(row[u], span, n_span)) = word;
    }
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kQuantThreads)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long rows, long long cols,
                     long long row_stride, uint32_t n_chunk, uint32_t total, void* __restrict__ out) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const long long warp = (long long)blockIdx.x * (kQuantThreads / 32) + (threadIdx.x >> 5);
    const long long n_block = (cols + kMxBlock - 1) / kMxBlock, n_span = (cols + kMxSpan - 1) / kMxSpan;
    uint32_t row[kQuantUnroll], ch[kQuantUnroll], w[kQuantUnroll], s[kQuantUnroll];
#pragma unroll
    for (int u = 0; u < kQuantUnroll; ++u) {
        const long long c = warp * kQuantUnroll + u;
        w[u] = s[u] = 0;
        if (c < total) {
            row[u] = (uint32_t)c / n_chunk;
            ch[u] = (uint32_t)c - row[u] * n_chunk;
            const long long col = (long long)ch[u] * kQuantChunk + lane * 8;
            if (col < cols) {
                w[u] = *reinterpret_cast<const uint32_t*>(codes + (size_t)row[u] * n_block * 16 + col / 2);
                s[u] = scales[mx_scale_word(row[u], col / kMxSpan, n_span) + ((col / kMxBlock) & 3)];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kQuantUnroll; ++u) {
        if (warp * kQuantUnroll + u >= total) break;
        const long long col = (long long)ch[u] * kQuantChunk + lane * 8;
        if (col >= cols) continue;
        const float scale = s[u] == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(s[u] ? s[u] << 23 : 1u << 22);
        uint32_t h[4];
        mx_decode8(w[u], h);
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            v[2 * i] = p.x * scale;
            v[2 * i + 1] = p.y * scale;
        }
        const size_t at = (size_t)row[u] * row_stride + col;
        if (BF16) {
            uint16_t* o = static_cast<uint16_t*>(out) + at;
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 q = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);   // exact: one mantissa bit
                b[i] = *reinterpret_cast<const uint32_t*>(&q);
            }
            if (VEC) {
                *reinterpret_cast<uint4*>(o) = make_uint4(b[0], b[1], b[2], b[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (col + i < cols) o[i] = (uint16_t)(b[i / 2] >> (16 * (i & 1)));
            }
        } else {
            float* o = static_cast<float*>(out) + at;
            if (VEC) {
                reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (col + i < cols) o[i] = v[i];
            }
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

cudaError_t launch_mx_quantize(const void* x, int bf16, long long rows, long long cols, long long row_stride,
                               uint8_t* codes, uint8_t* scales, cudaStream_t st) {
    const uint32_t n_chunk = (uint32_t)((cols + kQuantChunk - 1) / kQuantChunk);
    const uint32_t total = (uint32_t)(rows * n_chunk);
    const int per_cta = kQuantThreads / 32 * kQuantUnroll;
    const dim3 grid((total + per_cta - 1) / per_cta);
    const bool vec = cols % 8 == 0 && ((uintptr_t)x & 15) == 0 && row_stride * (bf16 ? 2 : 4) % 16 == 0;
    auto k = bf16 ? (vec ? mx_quantize_kernel<true, true> : mx_quantize_kernel<true, false>)
                  : (vec ? mx_quantize_kernel<false, true> : mx_quantize_kernel<false, false>);
    return launch_pdl(k, grid, dim3(kQuantThreads), 0, st, x, rows, cols, row_stride, n_chunk, total, codes, scales);
}

}  // namespace saem

using namespace saem;

// rows, cols and the number of 256-element chunks a kernel counts in 32 bits
static bool mx_shape_ok(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || rows > 0x7FFFFFFFll || cols > 0x7FFFFFFFll) return false;
    return rows * ((cols + kQuantChunk - 1) / kQuantChunk) <= 0x7FFFFFFFll;
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
    return launch_mx_quantize(x, dtype == SAEM_OUT_BF16, rows, cols, row_stride, (uint8_t*)codes, (uint8_t*)scales,
                              (cudaStream_t)stream) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
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
    const uint32_t n_chunk = (uint32_t)((cols + kQuantChunk - 1) / kQuantChunk);
    const uint32_t total = (uint32_t)(rows * n_chunk);
    const int per_cta = kQuantThreads / 32 * kQuantUnroll;
    const bool vec = cols % 8 == 0 && ((uintptr_t)out & 15) == 0 && row_stride * (bf16 ? 2 : 4) % 16 == 0;
    auto k = bf16 ? (vec ? mx_dequantize_kernel<true, true> : mx_dequantize_kernel<true, false>)
                  : (vec ? mx_dequantize_kernel<false, true> : mx_dequantize_kernel<false, false>);
    return launch_pdl(k, dim3((total + per_cta - 1) / per_cta), dim3(kQuantThreads), 0, (cudaStream_t)stream,
                      (const uint8_t*)codes, (const uint8_t*)scales, (long long)rows, (long long)cols,
                      (long long)row_stride, n_chunk, total, out) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
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
