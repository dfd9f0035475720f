// The norms around a block, fused with its gate and residual scale: one pass over the residual stream x and the block's
// output y.
//     z  = y / sqrt(mean(y^2) + eps) * w_post          (z = y without w_post)
//     x' = residual_scale * x + branch_scale * g * z   (g: per token, per channel, per element, or 1; optionally a sigmoid)
//     n  = x' / sqrt(mean(x'^2) + eps) * w_pre          the next block's input
// Without y: x' = x and n is the first block's input.
//
// One CTA per row: the row's x and y stay in registers between the two sums, so each is read once and x' and n are
// written once; weights and gate are on their way before the sums.  The bound is DRAM for many rows -- if the instructions
// per element stay few, which is why the types are template parameters and fp32 moves 32 bytes per instruction: with the
// types decided at run time 8192 rows of 4096 took 88 us, now 63 us for 403 MB, 6.4 TB/s -- and one round trip plus two block
// sums for a single row (2048 elements: 2.1 us).  (A persistent form with a ring of rows in shared memory was slower.)  All arithmetic is fp32; n is computed from the
// unrounded x'.
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

// Eight elements; fp32 needs 32-byte alignment, bf16 16.
template <bool F32>
struct Vec8 {
    uint32_t w[F32 ? 8 : 4];
    __device__ __forceinline__ void load(const void* p, size_t at) {
        if constexpr (F32) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                         : "l"(static_cast<const float*>(p) + at));
        } else {
            const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        }
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (F32) v[i] = __uint_as_float(w[i]);
            else v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        }
    }
};
template <bool F32>
__device__ __forceinline__ void store8(void* p, size_t at, const float (&v)[8]) {
    if constexpr (F32) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<float*>(p) + at),
                     "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
                     "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])) : "memory");
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 q = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&q);
        }
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ float load1(const void* p, size_t at, int dtype) {
    return dtype == SAEM_OUT_BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void store1(void* p, size_t at, int dtype, float v) {
    if (dtype == SAEM_OUT_BF16) static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
    else static_cast<float*>(p)[at] = v;
}
__device__ __forceinline__ float gate_of(const saem_norm_config& c, float g) { return c.gate_sigmoid ? 1.f / (1.f + expf(-g)) : g; }
// branch_scale times the row's gate, if it has one
__device__ __forceinline__ float row_factor(const NormArgs& a, size_t row) {
    if (a.c.gate_mode != SAEM_GATE_TOKEN) return a.c.branch_scale;
    return a.c.branch_scale * gate_of(a.c, load1(a.gate, row * a.c.gate_stride, a.c.gate_dtype));
}

constexpr int kRowsPerCta = 8;              // of short rows: a warp each

// Sum over the row's threads (a warp, or the CTA) in a fixed order; `red` holds one float per warp.
template <bool WARP>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (WARP) return v;
    const int warps = blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < warps ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Aligned rows: PER vectors of eight per thread, blockDim.x vectors apart.  XF, YF, WF: x, y and the weights are fp32.
template <bool XF, bool YF, bool WF, int PER, bool WARP>
__global__ void __launch_bounds__(kNormMaxThreads)
block_norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[2][32];
    pdl_wait();
    pdl_launch_dependents();
    const saem_norm_config& c = a.c;
    const size_t row = WARP ? (size_t)blockIdx.x * kRowsPerCta + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= c.rows) return;
    const int cols = c.cols, step = (WARP ? 32 : blockDim.x) * 8, first = (WARP ? threadIdx.x & 31 : threadIdx.x) * 8;
    Vec8<XF> xr[PER];
    Vec8<YF> yr[PER];
    Vec8<WF> wp[PER], wn[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int col = first + p * step;
        if (col >= cols) break;
        xr[p].load(a.x, row * c.x_stride + col);
        if (a.y) yr[p].load(a.y, row * c.y_stride + col);
        if (a.w_post) wp[p].load(a.w_post, col);
        if (a.w_pre) wn[p].load(a.w_pre, col);
    }
    float x[PER][8];
#pragma unroll
    for (int p = 0; p < PER; ++p)
        if (first + p * step < cols) xr[p].widen(x[p]);
    if (a.y) {
        float y[PER][8], s = 0.f;
        const bool vector_gate = c.gate_mode >= SAEM_GATE_CHANNEL;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            if (first + p * step >= cols) break;
            yr[p].widen(y[p]);
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(y[p][i], y[p][i], s);
        }
        float b = row_factor(a, row);
        if (a.w_post) b *= 1.f / sqrtf(row_sum<WARP>(s, red[0]) / (float)cols + c.eps);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const int col = first + p * step;
            if (col >= cols) break;
            float w[8];
            if (a.w_post) {
                wp[p].widen(w);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] *= w[i];
            }
            if (vector_gate) {
                const size_t at = (c.gate_mode == SAEM_GATE_FULL ? row * c.gate_stride : 0) + col;
                if (c.gate_dtype == SAEM_OUT_BF16) {
                    Vec8<false> g;
                    g.load(a.gate, at);
                    g.widen(w);
                } else {
                    Vec8<true> g;
                    g.load(a.gate, at);
                    g.widen(w);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) y[p][i] *= gate_of(c, w[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) x[p][i] = fmaf(b, y[p][i], c.residual_scale * x[p][i]);
            if (a.x_out) store8<XF>(a.x_out, row * c.x_out_stride + col, x[p]);
        }
    }
    if (!a.n_out) return;
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        if (first + p * step >= cols) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[p][i], x[p][i], s);
    }
    const float r = 1.f / sqrtf(row_sum<WARP>(s, red[1]) / (float)cols + c.eps);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int col = first + p * step;
        if (col >= cols) break;
        float w[8];
        if (a.w_pre) wn[p].widen(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[p][i] *= a.w_pre ? r * w[i] : r;
        if (c.n_dtype == SAEM_OUT_BF16) store8<false>(a.n_out, row * c.n_stride + col, x[p]);
        else store8<true>(a.n_out, row * c.n_stride + col, x[p]);
    }
}

template <bool F32>
__device__ __forceinline__ float at1(const uint8_t* p, int i) {
    if constexpr (F32) return reinterpret_cast<const float*>(p)[i];
    else return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
}
__device__ __forceinline__ const uint8_t* row_of(const void* p, size_t at, bool f32) { return static_cast<const uint8_t*>(p) + at * (f32 ? 4 : 2); }

// Any rows: PER elements per thread, blockDim.x apart.  8192 rows of 4095 columns, x fp32, y bf16, a gate per row: 92 us
// (4096 columns, the kernel above: 63 us).  Elements are loaded one by one, the weights behind
// the first sum.
template <bool XF, bool YF, bool WF, int PER, bool WARP>
__global__ void __launch_bounds__(kNormMaxThreads)
block_norm_any_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float red[2][32];
    pdl_wait();
    pdl_launch_dependents();
    const saem_norm_config& c = a.c;
    const size_t row = WARP ? (size_t)blockIdx.x * kRowsPerCta + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= c.rows) return;
    const int cols = c.cols, step = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x & 31 : threadIdx.x;
    const uint8_t* xp = row_of(a.x, row * c.x_stride, XF);
    const uint8_t* yp = row_of(a.y, row * c.y_stride, YF);
    const uint8_t* wp = static_cast<const uint8_t*>(a.w_post);
    const uint8_t* wn = static_cast<const uint8_t*>(a.w_pre);
    float x[PER], y[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int col = p * step + tid;
        x[p] = y[p] = 0.f;
        if (col < cols) {
            x[p] = at1<XF>(xp, col);
            if (a.y) y[p] = at1<YF>(yp, col);
        }
    }
    if (a.y) {
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < PER; ++p) s = fmaf(y[p], y[p], s);
        float b = row_factor(a, row);
        if (wp) {
            b *= 1.f / sqrtf(row_sum<WARP>(s, red[0]) / (float)cols + c.eps);
#pragma unroll
            for (int p = 0; p < PER; ++p)
                if (p * step + tid < cols) y[p] *= at1<WF>(wp, p * step + tid);
        }
        if (c.gate_mode >= SAEM_GATE_CHANNEL) {
            const size_t at = c.gate_mode == SAEM_GATE_FULL ? row * c.gate_stride : 0;
#pragma unroll
            for (int p = 0; p < PER; ++p)
                if (p * step + tid < cols) y[p] *= gate_of(c, load1(a.gate, at + p * step + tid, c.gate_dtype));
        }
#pragma unroll
        for (int p = 0; p < PER; ++p) x[p] = fmaf(b, y[p], c.residual_scale * x[p]);
        if (a.x_out) {
            uint8_t* o = const_cast<uint8_t*>(row_of(a.x_out, row * c.x_out_stride, XF));
#pragma unroll
            for (int p = 0; p < PER; ++p)
                if (p * step + tid < cols) store1(o, p * step + tid, XF ? SAEM_OUT_F32 : SAEM_OUT_BF16, x[p]);
        }
    }
    if (!a.n_out) return;
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) s = fmaf(x[p], x[p], s);
    const float r = 1.f / sqrtf(row_sum<WARP>(s, red[1]) / (float)cols + c.eps);
    uint8_t* o = const_cast<uint8_t*>(row_of(a.n_out, row * c.n_stride, c.n_dtype == SAEM_OUT_F32));
    if (c.n_dtype == SAEM_OUT_F32) {
#pragma unroll
        for (int p = 0; p < PER; ++p)
            if (p * step + tid < cols) store1(o, p * step + tid, SAEM_OUT_F32, x[p] * (wn ? r * at1<WF>(wn, p * step + tid) : r));
    } else {
#pragma unroll
        for (int p = 0; p < PER; ++p)
            if (p * step + tid < cols) store1(o, p * step + tid, SAEM_OUT_BF16, x[p] * (wn ? r * at1<WF>(wn, p * step + tid) : r));
    }
}

template <bool XF, bool YF, bool WF>
static cudaError_t launch_typed(const NormArgs& a, bool vec, cudaStream_t st) {
    const int n = vec ? a.c.cols / 8 : a.c.cols;
    const dim3 grid((unsigned)a.c.rows), warps((unsigned)((a.c.rows + kRowsPerCta - 1) / kRowsPerCta));
    auto threads = [&](int per) { return dim3((unsigned)round_up((n + per - 1) / per, 32)); };
    // a row of up to 512 (any: 256) elements is a warp's (8192 rows of 256, bf16 x and fp32 y: 4.6 us against 8.9 us)
    const dim3 eight(kRowsPerCta * 32);
    if (!vec) {
        if (n <= 256) return launch_pdl(block_norm_any_kernel<XF, YF, WF, 8, true>, warps, eight, 0, st, a);
        if (n <= 4096) return launch_pdl(block_norm_any_kernel<XF, YF, WF, 8, false>, grid, threads(8), 0, st, a);
        return launch_pdl(block_norm_any_kernel<XF, YF, WF, 32, false>, grid, threads(32), 0, st, a);
    }
    if (n <= 64) return launch_pdl(block_norm_kernel<XF, YF, WF, 2, true>, warps, eight, 0, st, a);
    if (n <= 256) return launch_pdl(block_norm_kernel<XF, YF, WF, 1, false>, grid, threads(1), 0, st, a);
    if (n <= 1024) return launch_pdl(block_norm_kernel<XF, YF, WF, 2, false>, grid, threads(2), 0, st, a);
    return launch_pdl(block_norm_kernel<XF, YF, WF, 4, false>, grid, threads(4), 0, st, a);
}

static cudaError_t launch_block_norm(const NormArgs& a, bool vec, cudaStream_t st) {
    const bool xf = a.c.x_dtype == SAEM_OUT_F32, yf = a.c.y_dtype == SAEM_OUT_F32;
    if (a.c.w_dtype == SAEM_OUT_F32)
        return xf ? (yf ? launch_typed<true, true, true>(a, vec, st) : launch_typed<true, false, true>(a, vec, st))
                  : (yf ? launch_typed<false, true, true>(a, vec, st) : launch_typed<false, false, true>(a, vec, st));
    return xf ? (yf ? launch_typed<true, true, false>(a, vec, st) : launch_typed<true, false, false>(a, vec, st))
              : (yf ? launch_typed<false, true, false>(a, vec, st) : launch_typed<false, false, false>(a, vec, st));
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
        if (vector) vec = vec && ((uintptr_t)p | (many ? (uintptr_t)(stride * (int64_t)e) : 0)) % (8 * e) == 0;
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
