// What the attention calls share: checks of their arguments, and the places of a batch's tokens.
#ifndef SAEM_ATTEND_COMMON_CUH_
#define SAEM_ATTEND_COMMON_CUH_

#include <math.h>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "saem_internal.h"

namespace saem {

constexpr int kHeadDimMax = 128;

inline bool head_dim_ok(int d) { return d >= 8 && d <= kHeadDimMax && d % 8 == 0; }
inline bool head_dtype_ok(int t) { return t == SAEM_OUT_F32 || t == SAEM_OUT_BF16 || t == SAEM_OUT_F16; }
inline int head_elem(int t) { return t == SAEM_OUT_F32 ? 4 : 2; }
inline int rotary_status(const saem_rotary_config& r, const void* turns) {
    if (!head_dim_ok(r.head_dim) || r.rotary_dim < 0 || r.rotary_dim > r.head_dim || r.rotary_dim % 8) return SAEM_ERR_SHAPE;
    if (!(r.eps >= 0.f) || !isfinite(r.amplitude) || (r.rotary_dim && !turns)) return SAEM_ERR_INVALID_ARG;
    return SAEM_OK;
}
// Tokens x heads that are written: no two elements at one place.
inline bool heads_apart(int64_t tokens, int64_t heads, int dim, int64_t ts, int64_t hs) {
    if (tokens <= 1) ts = INT64_MAX;
    if (heads <= 1) return ts >= dim;
    if (hs < dim) return false;
    if (tokens <= 1 || ts >= (heads - 1) * hs + dim) return true;
    return ts >= dim && hs >= (tokens - 1) * ts + dim;
}
inline int cache_status(const saem_kv_cache& c) {
    if (c.dtype != SAEM_OUT_BF16 && c.dtype != SAEM_OUT_F16) return SAEM_ERR_INVALID_ARG;
    if (!head_dim_ok(c.head_dim) || c.kv_heads < 1 || c.pages < 1 || c.page_size < 16 || c.page_size % 16 || c.page_size > 65536) return SAEM_ERR_SHAPE;
    if (c.kv_heads > 65536 || c.pages > 0x7FFFFFFFll / c.kv_heads / c.page_size) return SAEM_ERR_SHAPE;
    if (!c.k || !c.v) return SAEM_ERR_INVALID_ARG;
    return ((uintptr_t)c.k | (uintptr_t)c.v) % 16 ? SAEM_ERR_ALIGNMENT : SAEM_OK;
}
// Sizes first, so that an empty batch may come without addresses.
inline int batch_shape(const saem_batch& b) {
    if (b.seqs < 0 || b.seqs > 65536 || b.tokens < 0 || b.max_pages < 0 || b.max_new < 0) return SAEM_ERR_SHAPE;
    if (b.seqs > 1 && b.table_stride < b.max_pages) return SAEM_ERR_SHAPE;
    return SAEM_OK;
}
inline int batch_status(const saem_batch& b) {
    if (!b.offsets || !b.lengths || (!b.table && b.max_pages)) return SAEM_ERR_INVALID_ARG;
    return ((uintptr_t)b.offsets | (uintptr_t)b.lengths | (uintptr_t)b.table) % 4 ? SAEM_ERR_ALIGNMENT : SAEM_OK;
}

// n / d for 0 <= n < 2^31 by a multiplication: with 2^s >= d, mul = ceil(2^(31 + s) / d) is off by less than 2^s / 2^31 of a quotient.
struct Divisor {
    uint32_t d, mul, shift;
};
inline Divisor divisor_of(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), 31 + s};
}

#ifdef __CUDACC__
__device__ __forceinline__ int quotient(int n, const Divisor& d) { return (int)((uint64_t)(uint32_t)n * d.mul >> d.shift); }
// Two fp32 values in a register pair: one instruction for both.
__device__ __forceinline__ uint64_t pack_b32x2(uint32_t lo, uint32_t hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}
__device__ __forceinline__ uint64_t pack_f32x2(float lo, float hi) { return pack_b32x2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ float low_f32(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high_f32(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// Two fp32 values to a word of two 16-bit ones, the first in the low half.
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (F16) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}
template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
    if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
#endif

}  // namespace saem

#endif  // SAEM_ATTEND_COMMON_CUH_
