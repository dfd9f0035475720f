// The gate of one token, shared by the routing kernels and the fused decode kernels: one warp routes
// one token (Background, "Mixture-of-Experts Inference": the router selects the top-k experts).
// Each lane keeps up to four logits in registers (experts lane, lane+32, ...); k rounds of a
// warp-wide arg-max by shuffles on a packed 64-bit key whose high word orders the logit and whose
// low word prefers the lower expert id; softmax over the k winners in registers.
#ifndef SAEM_ROUTE_ROW_CUH_
#define SAEM_ROUTE_ROW_CUH_

#include <math_constants.h>

#include "saem_internal.h"

namespace saem {

constexpr int kPerLane = SAEM_MAX_EXPERTS / 32;

// Order-preserving map float -> uint32: larger float <=> larger key.  NaN -> key of -inf,
// -0 -> key of +0 so that the two zeros tie.
__device__ __forceinline__ uint32_t order_key(float v) {
    if (v != v) v = -CUDART_INF_F;
    if (v == 0.0f) v = 0.0f;
    uint32_t b = __float_as_uint(v);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    uint32_t b = (k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k;
    return __uint_as_float(b);
}

// One warp routes one token: `row` holds the token's E logits (global or shared memory).
__device__ __forceinline__ void route_row(const float* __restrict__ row, int E, int k, int renorm, int lane,
                                          int32_t* __restrict__ idx_out, float* __restrict__ w_out) {
    unsigned long long key[kPerLane];
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        int e = lane + 32 * i;
        key[i] = 0ull;                                    // below every real key (a real key's high word is never 0)
        if (e < E) key[i] = ((unsigned long long)order_key(row[e]) << 32) | (uint32_t)(~(uint32_t)e);
    }

    // winners: slot j lives in lane j & 31, register j >> 5
    float win_v[kPerLane];
    float denom_all = 0.f;
    float vmax = 0.f;
    for (int j = 0; j < k; ++j) {
        unsigned long long best = key[0];
#pragma unroll
        for (int i = 1; i < kPerLane; ++i) best = key[i] > best ? key[i] : best;
        // warp-wide maximum of the 64-bit key in two 32-bit reductions: the largest value word, then
        // the largest ~id (the lowest expert id) among the lanes that hold that value
        const uint32_t hi = (uint32_t)(best >> 32);
        const uint32_t hi_max = __reduce_max_sync(0xffffffffu, hi);
        const uint32_t lo_max = __reduce_max_sync(0xffffffffu, hi == hi_max ? (uint32_t)best : 0u);
        best = ((unsigned long long)hi_max << 32) | lo_max;
        int e = (int)(~(uint32_t)best);
        float v = key_value((uint32_t)(best >> 32));
        if (j == 0) {
            vmax = v;
            if (!renorm) {                                // denominator over all experts, before any key is cleared
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < kPerLane; ++i)
                    if (lane + 32 * i < E) s += expf(key_value((uint32_t)(key[i] >> 32)) - vmax);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                denom_all = s;
            }
        }
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
            if (lane + 32 * i == e) key[i] = 0ull;        // taken
        if (lane == 0) idx_out[j] = e;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
            if ((j >> 5) == i && (j & 31) == lane) win_v[i] = v;
    }

    // softmax over the winners
    float z[kPerLane];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        int j = lane + 32 * i;
        z[i] = 0.f;
        if (j < k) {
            if (vmax == CUDART_INF_F) {
                z[i] = (win_v[i] == CUDART_INF_F) ? 1.f : 0.f;
            } else if (vmax == -CUDART_INF_F) {
                z[i] = 1.f;
            } else {
                z[i] = expf(win_v[i] - vmax);
            }
            s += z[i];
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    float denom = s;
    if (!renorm && vmax != CUDART_INF_F && vmax != -CUDART_INF_F) denom = denom_all;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        int j = lane + 32 * i;
        if (j < k) w_out[j] = z[i] / denom;
    }
}

// route_row (the same choices and weights) for k <= 8, where the gate is on the critical path: a lane's four keys are sorted first, so
// that a round looks at one of them; the winner of round j ends in lane j.
__device__ __forceinline__ void route_few(const float* __restrict__ row, int E, int k, int renorm, int lane, int& mine, float& weight) {
    uint32_t key[kPerLane];
    int id[kPerLane];
    float all = 0.f, win = 0.f;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
        id[i] = lane + 32 * i;
        key[i] = id[i] < E ? order_key(row[id[i]]) : 0u;                       // 0: below every real key
    }
    float vmax = 0.f;
    if (!renorm) {                                                             // in the order of the ids, as route_row adds
        vmax = key_value(__reduce_max_sync(0xffffffffu, max(max(key[0], key[1]), max(key[2], key[3]))));
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
            if (id[i] < E) all += expf(key_value(key[i]) - vmax);
    }
    auto sort2 = [&](int x, int y) {                                           // larger first, equal keys by id
        const bool swap = key[y] > key[x] || (key[y] == key[x] && id[y] < id[x]);
        const uint32_t kx = key[x];
        const int ix = id[x];
        key[x] = swap ? key[y] : kx;  id[x] = swap ? id[y] : ix;
        key[y] = swap ? kx : key[y];  id[y] = swap ? ix : id[y];
    };
    sort2(0, 1); sort2(2, 3); sort2(0, 2); sort2(1, 3); sort2(1, 2);
    mine = 0;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, key[0]);
        const int e = (int)__reduce_min_sync(0xffffffffu, key[0] == top ? (unsigned)id[0] : 0xffffffffu);
        if (j == 0) vmax = key_value(top);
        if (e == id[0]) {                                                      // taken
            key[0] = key[1]; key[1] = key[2]; key[2] = key[3]; key[3] = 0u;
            id[0] = id[1]; id[1] = id[2]; id[2] = id[3]; id[3] = 0x7FFFFFFF;
        }
        if (lane == j) {
            win = key_value(top);
            mine = e;
        }
    }
    float z = 0.f;
    if (lane < k)
        z = vmax == CUDART_INF_F ? (win == CUDART_INF_F ? 1.f : 0.f) : vmax == -CUDART_INF_F ? 1.f : expf(win - vmax);
    float sum = z;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);   // k <= 8: the other lanes hold nothing
    if (!renorm && vmax != CUDART_INF_F && vmax != -CUDART_INF_F) {
        sum = all;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    weight = z / sum;
}

}  // namespace saem

#endif  // SAEM_ROUTE_ROW_CUH_
