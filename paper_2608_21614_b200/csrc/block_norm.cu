// The norms around a block, fused with its gate and residual scale: one pass over the residual stream x and the block's
// output y.
//     z  = y / sqrt(mean(y^2) + eps) * w_post          (z = y without w_post)
//     x' = residual_scale * x + branch_scale * g * z   (g: per token, per channel, per element, or 1; optionally a sigmoid)
//     n  = x' / sqrt(mean(x'^2) + eps) * w_pre          the next block's input
// Without y: x' = x and n is the first block's input.
//
// One CTA per row: the row's x and y stay in registers between the two sums, so each is read once and x' and n are
// written once; the bound is DRAM for many rows and one round trip plus two block sums for a single row.  All
// arithmetic is fp32; n is computed from the unrounded x'.
#include <cuda_bf16.h>

#include "saem_internal.h"

namespace saem {

constexpr int kNormMaxThreads = 512;

struct NormArgs {
    saem_norm_config c;
    const void* x;
    const void* y;
    const void* gate;
    const void* w_post;
    const void* w_pre;
    void* x_out;
    void* n_out;
};

template <int VEC>
__device__ __forceinline__ void load_vec(const void* p, size_t at, int dtype, float (&v)[VEC]) {
    if constexpr (VEC == 8) {
        if (dtype == SAEM_OUT_BF16) {
            const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
            const float4 a = q[0], b = q[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
        v[0] = dtype == SAEM_OUT_BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16)
                                      : static_cast<const float*>(p)[at];
    }
}

template <int VEC>
__device__ __forceinline__ void store_vec(void* p, size_t at, int dtype, const float (&v)[VEC]) {
    if constexpr (VEC == 8) {
        if (dtype == SAEM_OUT_BF16) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 q = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&q);
            }
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
            q[0] = make_float4(v[0], v[1], v[2], v[3]);
            q[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
        if (dtype == SAEM_OUT_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v[0]);
        else static_cast<float*>(p)[at] = v[0];
    }
}

// Sum over the CTA in a fixed order; `red` holds one float per warp.
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// VEC elements at a time, PER of those per thread, blockDim.x vectors apart.
template <int VEC, int PER>
__global__ void __launch_bounds__(kNormMaxThreads)
block_norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[2][32];
    pdl_wait();
    pdl_launch_dependents();
    const saem_norm_config& c = a.c;
    const size_t row = blockIdx.x;
    const int cols = c.cols;
    float x[PER][VEC], y[PER][VEC];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int col = (p * blockDim.x + threadIdx.x) * VEC;
        if (col < cols) {
            load_vec<VEC>(a.x, row * c.x_stride + col, c.x_dtype, x[p]);
            if (a.y) load_vec<VEC>(a.y, row * c.y_stride + col, c.y_dtype, y[p]);
        }
    }
    if (a.y) {
        float r = 1.f;
        if (a.w_post) {
            float s = 0.f;
#pragma unroll
            for (int p = 0; p < PER; ++p)
                if ((p * blockDim.x + threadIdx.x) * VEC < cols)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) s += y[p][i] * y[p][i];
            r = 1.f / sqrtf(block_sum(s, red[0]) / (float)cols + c.eps);
        }
        float token_gate = 1.f;
        if (c.gate_mode == SAEM_GATE_TOKEN) {
            float g[1];
            load_vec<1>(a.gate, row * c.gate_stride, c.gate_dtype, g);
            token_gate = c.gate_sigmoid ? 1.f / (1.f + expf(-g[0])) : g[0];
        }
        const float b = c.branch_scale * token_gate;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int col = (p * blockDim.x + threadIdx.x) * VEC;
            if (col >= cols) continue;
            float w[VEC], g[VEC];
            if (a.w_post) load_vec<VEC>(a.w_post, col, c.w_dtype, w);
            if (c.gate_mode >= SAEM_GATE_CHANNEL)
                load_vec<VEC>(a.gate, (c.gate_mode == SAEM_GATE_FULL ? row * c.gate_stride : 0) + col, c.gate_dtype, g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float z = y[p][i];
                if (a.w_post) z = z * r * w[i];
                if (c.gate_mode >= SAEM_GATE_CHANNEL) z *= c.gate_sigmoid ? 1.f / (1.f + expf(-g[i])) : g[i];
                x[p][i] = c.residual_scale * x[p][i] + b * z;
            }
        }
        if (a.x_out) {
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const int col = (p * blockDim.x + threadIdx.x) * VEC;
                if (col < cols) store_vec<VEC>(a.x_out, row * c.x_out_stride + col, c.x_dtype, x[p]);
            }
        }
    }
    if (!a.n_out) return;
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p)
        if ((p * blockDim.x + threadIdx.x) * VEC < cols)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += x[p][i] * x[p][i];
    const float r = 1.f / sqrtf(block_sum(s, red[1]) / (float)cols + c.eps);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int col = (p * blockDim.x + threadIdx.x) * VEC;
        if (col >= cols) continue;
        float w[VEC];
        if (a.w_pre) load_vec<VEC>(a.w_pre, col, c.w_dtype, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[p][i] = a.w_pre ? x[p][i] * r * w[i] : x[p][i] * r;
        store_vec<VEC>(a.n_out, row * c.n_stride + col, c.n_dtype, x[p]);
    }
}

static cudaError_t launch_block_norm(const NormArgs& a, bool vec, cudaStream_t st) {
    const int n = vec ? (a.c.cols + 7) / 8 : a.c.cols;
    const dim3 grid((unsigned)a.c.rows);
    auto threads = [&](int per) { return dim3((unsigned)round_up((n + per - 1) / per, 32)); };
    if (vec) {
        if (n <= 256) return launch_pdl(block_norm_kernel<8, 1>, grid, threads(1), 0, st, a);
        if (n <= 512) return launch_pdl(block_norm_kernel<8, 2>, grid, threads(2), 0, st, a);
        return launch_pdl(block_norm_kernel<8, 4>, grid, threads(4), 0, st, a);
    }
    if (n <= 512) return launch_pdl(block_norm_kernel<1, 2>, grid, threads(2), 0, st, a);
    if (n <= 4096) return launch_pdl(block_norm_kernel<1, 8>, grid, threads(8), 0, st, a);
    return launch_pdl(block_norm_kernel<1, 32>, grid, threads(32), 0, st, a);
}

}  // namespace saem

using namespace saem;

extern "C" int saem_block_norm(const saem_norm_config* c, const void* x, const void* y, const void* gate,
                               const void* w_post, const void* w_pre, void* x_out, void* n_out, void* stream) {
    if (!c) return SAEM_ERR_INVALID_ARG;
    auto dtype_ok = [](int t) { return t == SAEM_OUT_F32 || t == SAEM_OUT_BF16; };
    if (!dtype_ok(c->x_dtype) || !dtype_ok(c->y_dtype) || !dtype_ok(c->n_dtype) || !dtype_ok(c->gate_dtype) ||
        !dtype_ok(c->w_dtype))
        return SAEM_ERR_INVALID_ARG;
    if (c->gate_mode < SAEM_GATE_NONE || c->gate_mode > SAEM_GATE_FULL || !(c->eps >= 0.f)) return SAEM_ERR_INVALID_ARG;
    if (c->rows < 0 || c->rows > 0x7FFFFFFFll || c->cols < 1 || c->cols > 16384) return SAEM_ERR_SHAPE;
    if (c->rows == 0) return SAEM_OK;                        // an empty tensor may have no address at all
    if (!y && (gate || w_post || x_out)) return SAEM_ERR_INVALID_ARG;
    if (!x_out && !n_out) return SAEM_ERR_INVALID_ARG;
    if (w_pre && !n_out) return SAEM_ERR_INVALID_ARG;
    if ((gate != nullptr) != (c->gate_mode != SAEM_GATE_NONE)) return SAEM_ERR_INVALID_ARG;
    if (!x) return SAEM_ERR_INVALID_ARG;
    // rows may not overlap; a gate of one value per token has any stride
    const bool many = c->rows > 1;
    if (many && (c->x_stride < c->cols || (y && c->y_stride < c->cols) || (x_out && c->x_out_stride < c->cols) ||
                 (n_out && c->n_stride < c->cols) || (c->gate_mode == SAEM_GATE_FULL && c->gate_stride < c->cols) ||
                 (c->gate_mode == SAEM_GATE_TOKEN && c->gate_stride < 0)))
        return SAEM_ERR_SHAPE;
    bool vec = c->cols % 8 == 0;
    bool ok = true;
    auto look = [&](const void* p, int dtype, int64_t stride, bool vector) {
        if (!p) return;
        const size_t e = dtype == SAEM_OUT_BF16 ? 2 : 4;
        ok = ok && (uintptr_t)p % e == 0;
        if (vector) vec = vec && ((uintptr_t)p & 15) == 0 && (!many || (stride * (int64_t)e) % 16 == 0);
    };
    look(x, c->x_dtype, c->x_stride, true);
    look(y, c->y_dtype, c->y_stride, true);
    look(gate, c->gate_dtype, c->gate_mode == SAEM_GATE_FULL ? c->gate_stride : 0, c->gate_mode >= SAEM_GATE_CHANNEL);
    look(w_post, c->w_dtype, 0, true);
    look(w_pre, c->w_dtype, 0, true);
    look(x_out, c->x_dtype, c->x_out_stride, true);
    look(n_out, c->n_dtype, c->n_stride, true);
    if (!ok) return SAEM_ERR_ALIGNMENT;
    NormArgs a = {*c, x, y, gate, w_post, w_pre, x_out, n_out};
    return launch_block_norm(a, vec, (cudaStream_t)stream) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}
