// The norm of each head with the rotation of its position, in place or on the way into the paged cache.
//     y = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> amplitude * (a cos - b sin, b cos + a sin),   angle = position * frequency
//
// A head is eight elements for each of 8 or 16 neighbouring lanes: two runs of four, which are the two halves of four pairs (half
// layout) or four pairs next to each other (interleaved), so that a rotation stays within a lane and only the norm's sum crosses
// them.  A group of lanes keeps the sines and cosines of one token for all the heads that it takes: they cost more
// instructions than the rest of a head.  The bound is DRAM for many tokens; for one it is the launch and a chain of loads.
//
// The angle in turns is position * turns[i] mod 2^64 in integers, exact but for the frequency's own rounding (2^-65 turns
// a position); its upper 32 bits, signed, times 2^-31 are the argument of sincospi in [-1, 1).
#include "attend_common.cuh"

namespace saem {

constexpr int kRotThreads = 256;
constexpr int kRotBatch = 4;                // heads whose loads are under way together

struct HeadsIn {
    const uint8_t* p;
    long long ts, hs;                       // strides in elements
};
struct RotArgs {
    int dim, rot, interleaved;
    float eps, amplitude;
    int w_bf16;
    const uint64_t* turns;
    const int32_t* positions;
    long long tokens;
    int slices;                             // groups of lanes that share a token's heads
    HeadsIn x[3];                           // q, k, v; rotate: the first alone
    const void* w[2];
    int heads[3];
    uint8_t* out;                           // q's
    long long out_ts, out_hs;
    int out_dtype;
    saem_kv_cache cache;
    saem_batch batch;
    int32_t* status;
};

// Four elements as they lie in memory.
template <int DT, bool VEC>
struct Run {
    uint32_t w[DT == SAEM_OUT_F32 ? 4 : 2];
    __device__ __forceinline__ void load(const uint8_t* p, long long at) {
        if constexpr (DT == SAEM_OUT_F32) {
            const float* f = reinterpret_cast<const float*>(p) + at;
            if constexpr (VEC) {
                const uint4 q = *reinterpret_cast<const uint4*>(f);
                w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
            }
        } else {
            const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + at;
            if constexpr (VEC) {
                const uint2 q = *reinterpret_cast<const uint2*>(h);
                w[0] = q.x; w[1] = q.y;
            } else {
                w[0] = h[0] | (uint32_t)h[1] << 16;
                w[1] = h[2] | (uint32_t)h[3] << 16;
            }
        }
    }
    __device__ __forceinline__ void widen(float* v) const {
        if constexpr (DT == SAEM_OUT_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            const float2 a = unpack2<DT == SAEM_OUT_F16>(w[0]), b = unpack2<DT == SAEM_OUT_F16>(w[1]);
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
        }
    }
};
template <bool VEC>
__device__ __forceinline__ void store4(uint8_t* p, long long at, int dtype, const float* v) {
    if (dtype == SAEM_OUT_F32) {
        float* f = reinterpret_cast<float*>(p) + at;
        if constexpr (VEC) *reinterpret_cast<float4*>(f) = make_float4(v[0], v[1], v[2], v[3]);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = v[i];
        }
        return;
    }
    uint32_t a, b;
    if (dtype == SAEM_OUT_F16) a = pack2<true>(v[0], v[1]), b = pack2<true>(v[2], v[3]);
    else a = pack2<false>(v[0], v[1]), b = pack2<false>(v[2], v[3]);
    uint16_t* h = reinterpret_cast<uint16_t*>(p) + at;
    if constexpr (VEC) *reinterpret_cast<uint2*>(h) = make_uint2(a, b);
    else {
        h[0] = (uint16_t)a; h[1] = (uint16_t)(a >> 16); h[2] = (uint16_t)b; h[3] = (uint16_t)(b >> 16);
    }
}

// The sequence that token t belongs to: the last one whose offset is at most t (offsets[0] = 0).  LANES probes a round.
template <int LANES>
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int seqs, int t, int lane, uint32_t group_mask, int group_shift) {
    int lo = 0, n = seqs;
    while (n > 1) {
        const int step = (n + LANES - 1) / LANES, at = lane * step;
        const bool below = at < n && offsets[lo + at] <= t;
        const uint32_t votes = (__ballot_sync(group_mask, below) >> group_shift) & (uint32_t)((1ull << LANES) - 1);
        const int last = max(0, __popc(votes) - 1) * step;
        lo += last;
        n = min(step, n - last);
    }
    return lo;
}

template <int DT, int LANES, bool VEC, bool APPEND>
__global__ void __launch_bounds__(kRotThreads)
rotary_kernel(const __grid_constant__ RotArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x % LANES;
    const int group_shift = (threadIdx.x & 31) / LANES * LANES;
    const uint32_t group_mask = (uint32_t)((1ull << LANES) - 1) << group_shift;
    const long long group = (long long)blockIdx.x * (kRotThreads / LANES) + threadIdx.x / LANES;
    const long long t = group / a.slices;
    const int slice = (int)(group % a.slices);
    if (t >= a.tokens) return;
    // where the lane's two runs of four lie in a head, and whether they turn
    const int unit = lane, half = a.rot / 2;
    const bool here = unit * 8 < a.dim, turn = unit * 8 < a.rot;
    const bool across = turn && !a.interleaved;
    const int at0 = across ? 4 * unit : 8 * unit, at1 = across ? half + 4 * unit : 8 * unit + 4;
    const int n_heads = a.heads[0] + a.heads[1] + a.heads[2];

    auto source = [&](int h) {
        int kind = 0;
        if (APPEND && h >= a.heads[0]) {
            h -= a.heads[0];
            kind = 1;
            if (h >= a.heads[1]) { h -= a.heads[1]; kind = 2; }
        }
        const HeadsIn& x = a.x[APPEND ? kind : 0];
        return x.p + (t * x.ts + h * x.hs) * (DT == SAEM_OUT_F32 ? 4 : 2);
    };
    Run<DT, VEC> raw[kRotBatch][2];
    auto fetch = [&](int h) {
#pragma unroll
        for (int i = 0; i < kRotBatch; ++i) {
            const int hi = h + i * a.slices;
            if (here && hi < n_heads) {
                const uint8_t* p = source(hi);
                raw[i][0].load(p, at0);
                raw[i][1].load(p, at1);
            }
        }
    };
    fetch(slice);                           // on its way while the token's place is looked up

    int place = 0, position;
    long long row = -1;                     // the token's row in the cache at head 0, in units of head_dim
    if (APPEND) {
        const int seqs = a.batch.seqs;
        if (t >= a.batch.offsets[seqs]) return;
        const int s = sequence_of<LANES>(a.batch.offsets, seqs, (int)t, lane, group_mask, group_shift);
        place = a.batch.lengths[s] - (a.batch.offsets[s + 1] - (int)t);
        if (place >= 0) {
            const int entry = place / a.cache.page_size;
            const int page = entry < a.batch.max_pages ? a.batch.table[s * a.batch.table_stride + entry] : -1;
            if (page >= 0 && page < a.cache.pages) row = (long long)page * a.cache.kv_heads * a.cache.page_size + place % a.cache.page_size;
            else if (a.status && lane == 0) atomicExch(a.status, SAEM_ERR_INVALID_ARG);
        }
        position = a.positions ? a.positions[t] : place;
    } else {
        position = a.positions[t];
    }
    float sn[4], cs[4];
    if (turn) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t u = a.turns[4 * unit + i] * (uint64_t)(long long)position;
            sincospif((float)(int32_t)(u >> 32) * 0x1p-31f, &sn[i], &cs[i]);
            sn[i] *= a.amplitude;
            cs[i] *= a.amplitude;
        }
    }
    float w[2][8];
#pragma unroll
    for (int k = 0; k < (APPEND ? 2 : 1); ++k)
        if (a.w[k] && here) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = i < 4 ? at0 + i : at1 + i - 4;
                w[k][i] = a.w_bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.w[k])[at] << 16) : static_cast<const float*>(a.w[k])[at];
            }
        }

    for (int h0 = slice; h0 < n_heads; h0 += kRotBatch * a.slices) {
        if (h0 != slice) fetch(h0);
#pragma unroll
        for (int i = 0; i < kRotBatch; ++i) {
            int h = h0 + i * a.slices;
            if (h >= n_heads) break;
            int kind = 0;
            if (APPEND && h >= a.heads[0]) {
                h -= a.heads[0];
                kind = 1;
                if (h >= a.heads[1]) { h -= a.heads[1]; kind = 2; }
            }
            float v[8];
            if (here) {
                raw[i][0].widen(v);
                raw[i][1].widen(v + 4);
            }
            if (kind < 2 && a.w[kind]) {
                float s = 0.f;
                if (here) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
                }
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(group_mask, s, o);
                const float r = 1.f / sqrtf(s / (float)a.dim + a.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= r * (APPEND && kind ? w[1][e] : w[0][e]);
            }
            if (kind < 2 && turn) {
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = v[2 * e], q = v[2 * e + 1];
                        v[2 * e] = fmaf(p, cs[e], -q * sn[e]);
                        v[2 * e + 1] = fmaf(q, cs[e], p * sn[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = v[e], q = v[e + 4];
                        v[e] = fmaf(p, cs[e], -q * sn[e]);
                        v[e + 4] = fmaf(q, cs[e], p * sn[e]);
                    }
                }
            }
            uint8_t* to;
            if (!APPEND || kind == 0) {
                to = a.out + (t * a.out_ts + h * a.out_hs) * (a.out_dtype == SAEM_OUT_F32 ? 4 : 2);
            } else {
                if (row < 0) continue;
                to = static_cast<uint8_t*>(kind == 1 ? a.cache.k : a.cache.v) + (row + (long long)h * a.cache.page_size) * a.dim * 2;
            }
            if (here) {
                store4<VEC>(to, at0, a.out_dtype, v);
                store4<VEC>(to, at1, a.out_dtype, v + 4);
            }
        }
    }
}

template <int DT, bool VEC, bool APPEND>
static cudaError_t launch_rotary_typed(RotArgs a, int n_sm, cudaStream_t st) {
    const int lanes = a.dim <= 64 ? 8 : 16, n_heads = a.heads[0] + a.heads[1] + a.heads[2];
    // as many groups as fill the SMs' threads, while a token has heads to share out
    const long long want = (long long)n_sm * 2048 / lanes;
    a.slices = (int)((want + a.tokens - 1) / a.tokens);
    if (a.slices > n_heads) a.slices = n_heads;
    const long long per = kRotThreads / lanes, grid = (a.tokens * a.slices + per - 1) / per;
    if (lanes == 8) return launch_pdl(rotary_kernel<DT, 8, VEC, APPEND>, dim3((unsigned)grid), dim3(kRotThreads), 0, st, a);
    return launch_pdl(rotary_kernel<DT, 16, VEC, APPEND>, dim3((unsigned)grid), dim3(kRotThreads), 0, st, a);
}
template <bool APPEND>
static int launch_rotary(const RotArgs& a, int x_dtype, bool vec, cudaStream_t st) {
    int n_sm;
    if (sm_count(&n_sm) != cudaSuccess) return SAEM_ERR_CUDA;
    cudaError_t e;
    if (x_dtype == SAEM_OUT_F32) e = vec ? launch_rotary_typed<SAEM_OUT_F32, true, APPEND>(a, n_sm, st) : launch_rotary_typed<SAEM_OUT_F32, false, APPEND>(a, n_sm, st);
    else if (x_dtype == SAEM_OUT_BF16) e = vec ? launch_rotary_typed<SAEM_OUT_BF16, true, APPEND>(a, n_sm, st) : launch_rotary_typed<SAEM_OUT_BF16, false, APPEND>(a, n_sm, st);
    else e = vec ? launch_rotary_typed<SAEM_OUT_F16, true, APPEND>(a, n_sm, st) : launch_rotary_typed<SAEM_OUT_F16, false, APPEND>(a, n_sm, st);
    return e == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}
// Whether runs of four elements of these heads are aligned to their size; *ok: elements to theirs.
static bool runs_aligned(const void* p, int dtype, int64_t tokens, int64_t heads, int64_t ts, int64_t hs, bool* ok) {
    const int e = head_elem(dtype);
    *ok = *ok && (uintptr_t)p % e == 0;
    return (uintptr_t)p % (4 * e) == 0 && (tokens <= 1 || ts % 4 == 0) && (heads <= 1 || hs % 4 == 0);
}

}  // namespace saem

using namespace saem;

extern "C" int saem_rotate(const saem_rotate_config* c, const void* x, const void* w, const uint64_t* turns, const int32_t* positions,
                           void* out, void* stream) {
    if (!c) return SAEM_ERR_INVALID_ARG;
    if (!head_dtype_ok(c->x_dtype) || !head_dtype_ok(c->out_dtype) || (c->w_dtype != SAEM_OUT_F32 && c->w_dtype != SAEM_OUT_BF16)) return SAEM_ERR_INVALID_ARG;
    if (c->tokens < 0 || c->heads < 1 || c->tokens > 0x7FFFFFFFll / c->heads) return SAEM_ERR_SHAPE;
    const int r = rotary_status(c->rotary, turns);
    if (r != SAEM_OK) return r;
    if (c->tokens == 0) return SAEM_OK;
    if (!x || !out || !positions) return SAEM_ERR_INVALID_ARG;
    if (c->x_token_stride < 0 || c->x_head_stride < 0 ||
        !heads_apart(c->tokens, c->heads, c->rotary.head_dim, c->out_token_stride, c->out_head_stride)) return SAEM_ERR_SHAPE;
    bool ok = (uintptr_t)positions % 4 == 0 && (uintptr_t)turns % 8 == 0 && (uintptr_t)w % head_elem(c->w_dtype) == 0;
    bool vec = runs_aligned(x, c->x_dtype, c->tokens, c->heads, c->x_token_stride, c->x_head_stride, &ok);
    vec &= runs_aligned(out, c->out_dtype, c->tokens, c->heads, c->out_token_stride, c->out_head_stride, &ok);
    if (!ok) return SAEM_ERR_ALIGNMENT;
    RotArgs a = {};
    a.dim = c->rotary.head_dim; a.rot = c->rotary.rotary_dim; a.interleaved = c->rotary.interleaved;
    a.eps = c->rotary.eps; a.amplitude = c->rotary.amplitude;
    a.w_bf16 = c->w_dtype == SAEM_OUT_BF16;
    a.turns = turns; a.positions = positions; a.tokens = c->tokens;
    a.x[0] = {static_cast<const uint8_t*>(x), c->x_token_stride, c->x_head_stride};
    a.w[0] = w; a.heads[0] = c->heads;
    a.out = static_cast<uint8_t*>(out); a.out_ts = c->out_token_stride; a.out_hs = c->out_head_stride; a.out_dtype = c->out_dtype;
    return launch_rotary<false>(a, c->x_dtype, vec, (cudaStream_t)stream);
}

extern "C" int saem_kv_append(const saem_append_config* c, const saem_kv_cache* cache, const saem_batch* b, const void* q, const void* k,
                              const void* v, const void* w_q, const void* w_k, const uint64_t* turns, const int32_t* positions,
                              void* q_out, int32_t* status, void* stream) {
    if (!c || !cache || !b) return SAEM_ERR_INVALID_ARG;
    if (!head_dtype_ok(c->x_dtype) || (c->w_dtype != SAEM_OUT_F32 && c->w_dtype != SAEM_OUT_BF16)) return SAEM_ERR_INVALID_ARG;
    int r = cache_status(*cache);
    if (r == SAEM_OK) r = batch_shape(*b);
    if (r == SAEM_OK) r = rotary_status(c->rotary, turns);
    if (r != SAEM_OK) return r;
    const int q_heads = q ? c->q_heads : 0, dim = cache->head_dim;
    if (c->rotary.head_dim != dim || (q && c->q_heads < 1)) return SAEM_ERR_SHAPE;
    if (b->tokens > 0x7FFFFFFF / (q_heads > cache->kv_heads ? q_heads : cache->kv_heads)) return SAEM_ERR_SHAPE;
    if (b->tokens == 0 || b->seqs == 0) return SAEM_OK;
    r = batch_status(*b);
    if (r != SAEM_OK) return r;
    if (!k || !v || !q != !q_out || (w_q && !q)) return SAEM_ERR_INVALID_ARG;
    if (c->k_token_stride < 0 || c->k_head_stride < 0 || c->v_token_stride < 0 || c->v_head_stride < 0) return SAEM_ERR_SHAPE;
    if (q && (c->q_token_stride < 0 || c->q_head_stride < 0 || !heads_apart(b->tokens, q_heads, dim, c->out_token_stride, c->out_head_stride)))
        return SAEM_ERR_SHAPE;
    const int we = head_elem(c->w_dtype);
    bool ok = (uintptr_t)positions % 4 == 0 && (uintptr_t)turns % 8 == 0 && (uintptr_t)w_q % we == 0 && (uintptr_t)w_k % we == 0 && (uintptr_t)status % 4 == 0;
    bool vec = runs_aligned(k, c->x_dtype, b->tokens, cache->kv_heads, c->k_token_stride, c->k_head_stride, &ok);
    vec &= runs_aligned(v, c->x_dtype, b->tokens, cache->kv_heads, c->v_token_stride, c->v_head_stride, &ok);
    if (q) {
        vec &= runs_aligned(q, c->x_dtype, b->tokens, q_heads, c->q_token_stride, c->q_head_stride, &ok);
        vec &= runs_aligned(q_out, cache->dtype, b->tokens, q_heads, c->out_token_stride, c->out_head_stride, &ok);
    }
    if (!ok) return SAEM_ERR_ALIGNMENT;
    RotArgs a = {};
    a.dim = dim; a.rot = c->rotary.rotary_dim; a.interleaved = c->rotary.interleaved;
    a.eps = c->rotary.eps; a.amplitude = c->rotary.amplitude;
    a.w_bf16 = c->w_dtype == SAEM_OUT_BF16;
    a.turns = turns; a.positions = positions; a.tokens = b->tokens;
    a.x[0] = {static_cast<const uint8_t*>(q), c->q_token_stride, c->q_head_stride};
    a.x[1] = {static_cast<const uint8_t*>(k), c->k_token_stride, c->k_head_stride};
    a.x[2] = {static_cast<const uint8_t*>(v), c->v_token_stride, c->v_head_stride};
    a.w[0] = w_q; a.w[1] = w_k;
    a.heads[0] = q_heads; a.heads[1] = a.heads[2] = cache->kv_heads;
    a.out = static_cast<uint8_t*>(q_out); a.out_ts = c->out_token_stride; a.out_hs = c->out_head_stride; a.out_dtype = cache->dtype;
    a.cache = *cache; a.batch = *b; a.status = status;
    return launch_rotary<true>(a, c->x_dtype, vec, (cudaStream_t)stream);
}
