// The norm of each head with the rotation of its position, in place or on the way into the paged cache.
//     y = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> amplitude * (a cos - b sin, b cos + a sin),   angle = position * frequency
//
// A head is eight elements for each of 8 or 16 neighbouring lanes: two runs of four, which are the two halves of four pairs (half
// layout) or four pairs next to each other (interleaved), so that a rotation stays within a lane and only the norm's sum crosses
// them.  A group of lanes takes some neighbouring heads of one token, all queries, all keys or all values, and keeps the token's sines and
// cosines for them; a warp's groups take the same heads of neighbouring tokens, so that its branches are uniform.  The bound is DRAM for many
// tokens; for one it is the launch and a chain of loads.
//
// The angle in turns is position * turns[i] mod 2^64 in integers, exact but for the frequency's own rounding (2^-65 turns
// a position).  Its upper 32 bits give the quarter turn and, signed, the rest r of at most an eighth of a turn, whose sine and cosine come
// from polynomials (turn2 below): sincospi, with its range checks, took half of the instructions of a group of eight heads.
#include "attend_common.cuh"

namespace saem {

constexpr int kRotThreads = 128;
constexpr int kRotMost = 8;                 // heads of a group at most
// Heads whose loads are under way, and CTAs per SM, which bound the registers: 8192 tokens of 40 heads rotated 29.5 us with 3 and 6, 38.5 us
// with 2 and 8, 31.5 us with 4 and 6; 8192 tokens of 32 + 8 + 8 heads appended 54.8, 40.7 and 43.7 us.
constexpr int rot_ahead(bool append) { return append ? 2 : 3; }
constexpr int rot_ctas(bool append) { return append ? 8 : 6; }

struct HeadsIn {
    const uint8_t* p;
    long long ts, hs;                       // strides in bytes
    int heads, slices;                      // groups of lanes that share a token's heads (of one kind)
};
struct RotArgs {
    int dim, rot, interleaved;
    float eps, amplitude, inv_dim;
    int w_bf16;
    const uint64_t* turns;
    const int32_t* positions;
    long long tokens;
    int per_group;                          // heads of a group
    Divisor by_slices, by_page;
    int w_runs;                             // the weights are aligned to runs of four
    HeadsIn x[3];                           // q, k, v; rotate: the first alone
    const void* w[2];
    uint8_t* out;                           // q's
    long long out_ts, out_hs;               // in bytes
    int out_dtype;
    saem_kv_cache cache;
    saem_batch batch;
    int32_t* status;
};

// How a lane's eight elements lie: two runs of four (RUNS, the half layout), one of eight (WHOLE, the interleaved one, or no rotation), or
// either at addresses that are aligned to their elements only (SINGLE).
enum { kRuns = 0, kWhole = 1, kSingle = 2 };
constexpr int elem_of(int dtype) { return dtype == SAEM_OUT_F32 ? 4 : 2; }
template <int DT, int FORM>
struct Eight {
    static constexpr int E = elem_of(DT);
    uint32_t w[2 * E];
    // p0, p1: the runs' first elements (WHOLE: p1 follows p0)
    __device__ __forceinline__ void load(const uint8_t* p0, const uint8_t* p1) {
        if constexpr (FORM == kSingle) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint8_t* p = i < 4 ? p0 + i * E : p1 + (i - 4) * E;
                if constexpr (E == 4) w[i] = *reinterpret_cast<const uint32_t*>(p);
                else if (i & 1) w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16;
                else w[i / 2] = *reinterpret_cast<const uint16_t*>(p);
            }
        } else if constexpr (E == 4 || FORM == kWhole) {
            const uint4 a = *reinterpret_cast<const uint4*>(p0);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
            if constexpr (E == 4) {
                const uint4 b = *reinterpret_cast<const uint4*>(p1);
                w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
            }
        } else {
            const uint2 a = *reinterpret_cast<const uint2*>(p0), b = *reinterpret_cast<const uint2*>(p1);
            w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
        }
    }
    // as four pairs, in the order of the elements
    __device__ __forceinline__ void widen(uint64_t (&v)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 4) v[i] = pack_b32x2(w[2 * i], w[2 * i + 1]);
            else {
                const float2 x = unpack2<DT == SAEM_OUT_F16>(w[i]);
                v[i] = pack_f32x2(x.x, x.y);
            }
        }
    }
};
constexpr int kAnyType = -1;                // the type is told at run time
template <int FORM, int OT>
__device__ __forceinline__ void store8(uint8_t* p0, uint8_t* p1, int any_dtype, const uint64_t (&v)[4]) {
    const bool f32 = OT == kAnyType ? any_dtype == SAEM_OUT_F32 : OT == SAEM_OUT_F32, f16 = OT == kAnyType ? any_dtype == SAEM_OUT_F16 : OT == SAEM_OUT_F16;
    if (f32) {
        if constexpr (FORM == kSingle) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<float*>(i < 4 ? p0 + i * 4 : p1 + (i - 4) * 4) = i & 1 ? high_f32(v[i / 2]) : low_f32(v[i / 2]);
        } else {
            *reinterpret_cast<float4*>(p0) = make_float4(low_f32(v[0]), high_f32(v[0]), low_f32(v[1]), high_f32(v[1]));
            *reinterpret_cast<float4*>(p1) = make_float4(low_f32(v[2]), high_f32(v[2]), low_f32(v[3]), high_f32(v[3]));
        }
    } else if constexpr (OT != SAEM_OUT_F32) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = f16 ? pack2<true>(low_f32(v[i]), high_f32(v[i])) : pack2<false>(low_f32(v[i]), high_f32(v[i]));
        if constexpr (FORM == kSingle) {
#pragma unroll
            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint16_t*>(i < 4 ? p0 + i * 2 : p1 + (i - 4) * 2) = (uint16_t)(w[i / 2] >> (i & 1) * 16);
        } else if constexpr (FORM == kWhole) {
            *reinterpret_cast<uint4*>(p0) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            *reinterpret_cast<uint2*>(p0) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(p1) = make_uint2(w[2], w[3]);
        }
    }
}

// The sequence that token t belongs to: the last one whose offset is at most t (offsets[0] = 0).  LANES probes a round.
template <int LANES>
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int seqs, int t, int lane, int sub) {
    const uint32_t mask = (uint32_t)((1ull << LANES) - 1) << sub * LANES;       // groups may take different numbers of rounds
    int lo = 0, n = seqs;
    while (n > 1) {
        const int step = (n + LANES - 1) / LANES, at = lane * step;
        const bool below = at < n && offsets[lo + at] <= t;
        const uint32_t votes = __ballot_sync(mask, below) & mask;
        const int last = max(0, __popc(votes) - 1) * step;
        lo += last;
        n = min(step, n - last);
    }
    return lo;
}

// Sines and cosines of two angles, given as fractions of a turn in units of 2^-64.  With r in half turns, |r| <= 1/4, and z = r^2:
// sin(pi r) = r s(z), s of degree 3 with the least largest relative error (2^-28), cos(pi r) = 1 + z c(z), c of degree 3 with the least
// largest absolute error (2^-34), both by Lawson's iteration in 64 bits; in fp32, r's own rounding included, the sine is within 2^-23.2 and the
// cosine within 2^-23.6 of the angle's in 64 bits (over 24 million angles).
__device__ __forceinline__ void turn2(uint64_t u0, uint64_t u1, float (&sn)[2], float (&cs)[2]) {
    const uint32_t h0 = (uint32_t)(u0 >> 32), h1 = (uint32_t)(u1 >> 32), q0 = (h0 + 0x20000000u) >> 30, q1 = (h1 + 0x20000000u) >> 30;
    const uint64_t r = pack_f32x2((float)(int32_t)(h0 - (q0 << 30)) * 0x1p-31f, (float)(int32_t)(h1 - (q1 << 30)) * 0x1p-31f), z = mul_f32x2(r, r);
    auto two = [](float v) { return pack_f32x2(v, v); };
    uint64_t s = fma_f32x2(z, two(-0.5890122056007385f), two(2.5497610569000244f));
    uint64_t c = fma_f32x2(z, two(0.2314295470714569f), two(-1.3350584506988525f));
    s = fma_f32x2(z, s, two(-5.167707920074463f));
    c = fma_f32x2(z, c, two(4.0587077140808105f));
    s = mul_f32x2(fma_f32x2(z, s, two(3.1415927410125732f)), r);
    c = fma_f32x2(z, fma_f32x2(z, c, two(-4.934802055358887f)), two(1.f));
    auto place = [](uint32_t q, float s, float c, float& sn, float& cs) {
        sn = __uint_as_float(__float_as_uint(q & 1 ? c : s) ^ (q & 2) << 30);
        cs = __uint_as_float(__float_as_uint(q & 1 ? s : c) ^ (q + 1 & 2) << 30);
    };
    place(q0, low_f32(s), low_f32(c), sn[0], cs[0]);
    place(q1, high_f32(s), high_f32(c), sn[1], cs[1]);
}

template <int DT, int OT, int LANES, int FORM, bool APPEND>
__global__ void __launch_bounds__(kRotThreads, rot_ctas(APPEND))
rotary_kernel(const __grid_constant__ RotArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kAhead = rot_ahead(APPEND), kTokens = 32 / LANES;             // tokens of a warp
    const bool interleaved = FORM == kSingle ? a.interleaved : FORM == kWhole;
    const int lane = threadIdx.x % LANES, sub = (threadIdx.x & 31) / LANES;
    const int warp = blockIdx.x * (kRotThreads / 32) + (threadIdx.x >> 5), many = quotient(warp, a.by_slices);
    int slice = warp - many * (int)a.by_slices.d, kind = 0;
    bool there = (long long)many * kTokens + sub < a.tokens;
    if ((long long)many * kTokens >= a.tokens) return;
    const long long t = there ? (long long)many * kTokens + sub : a.tokens - 1;     // groups without a token do what another does, but write nothing
    if (APPEND)
        while (slice >= a.x[kind].slices) slice -= a.x[kind++].slices;
    const HeadsIn& x = a.x[kind];
    const int first = slice * a.per_group, count = min(a.per_group, x.heads - first);
    // where the lane's two runs of four lie in a head, and whether they turn
    const int half = a.rot / 2;
    const bool here = lane * 8 < a.dim, turn = lane * 8 < a.rot && kind < 2;
    const bool across = lane * 8 < a.rot && !interleaved;
    const int at0 = across ? 4 * lane : 8 * lane, at1 = across ? half + 4 * lane : 8 * lane + 4;
    constexpr int E = elem_of(DT);
    const uint8_t* src = x.p + t * x.ts + first * x.hs;
    Eight<DT, FORM> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)     // on their way while the token's place is looked up
        if (here && i < count) raw[i].load(src + i * x.hs + at0 * E, src + i * x.hs + at1 * E);
    src += kAhead * x.hs;

    int position;
    uint8_t* to;
    long long step;
    int out_elem = 2;
    if (APPEND) {
        const int seqs = a.batch.seqs, s = sequence_of<LANES>(a.batch.offsets, seqs, (int)t, lane, sub);
        there = there && t < a.batch.offsets[seqs];
        const int place = a.batch.lengths[s] - (a.batch.offsets[s + 1] - (int)t);
        position = a.positions ? a.positions[t] : place;
        if (kind == 0) {
            to = a.out + t * a.out_ts + first * a.out_hs;
            step = a.out_hs;
        } else {
            const int entry = place >= 0 ? quotient(place, a.by_page) : 0;
            int page = place >= 0 && entry < a.batch.max_pages ? a.batch.table[s * a.batch.table_stride + entry] : -1;
            if (page < 0 || page >= a.cache.pages) {
                if (there && place >= 0 && a.status && lane == 0) atomicExch(a.status, SAEM_ERR_INVALID_ARG);
                there = false;
                page = 0;
            }
            step = (long long)a.cache.page_size * a.dim * 2;
            to = static_cast<uint8_t*>(kind == 1 ? a.cache.k : a.cache.v) +
                 (((long long)page * a.cache.kv_heads + first) * a.cache.page_size + (there ? place - entry * a.cache.page_size : 0)) * a.dim * 2;
        }
    } else {
        position = a.positions[t];
        to = a.out + t * a.out_ts + first * a.out_hs;
        step = a.out_hs;
        out_elem = a.out_dtype == SAEM_OUT_F32 ? 4 : 2;
    }
    const void* const weight = kind == 0 ? a.w[0] : kind == 1 ? a.w[1] : nullptr;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    if (weight && here) {
        const uint8_t* p = static_cast<const uint8_t*>(weight);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = i ? at1 : at0;
            if (a.w_bf16) {
                uint2 x;
                if (a.w_runs) x = *reinterpret_cast<const uint2*>(p + at * 2);
                else {
                    const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + at;
                    x = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
                }
                const float2 lo = unpack2<false>(x.x), hi = unpack2<false>(x.y);
                w[4 * i] = lo.x; w[4 * i + 1] = lo.y; w[4 * i + 2] = hi.x; w[4 * i + 3] = hi.y;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * i + e] = reinterpret_cast<const float*>(p)[at + e];
            }
        }
    }
    // y = x * k1 + (the pair's other element) * k2, weights and amplitude in the factors, for four pairs of elements
    uint64_t k1[4], k2[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k1[i] = pack_f32x2(w[2 * i], w[2 * i + 1]);
    if (turn) {
        float sn[4], cs[4];
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const uint64_t at = (uint64_t)(long long)position;
            float s2[2], c2[2];
            turn2(a.turns[4 * lane + i] * at, a.turns[4 * lane + i + 1] * at, s2, c2);
            sn[i] = s2[0]; sn[i + 1] = s2[1]; cs[i] = c2[0]; cs[i + 1] = c2[1];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] *= a.amplitude;
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                k1[i] = pack_f32x2(w[2 * i] * cs[i], w[2 * i + 1] * cs[i]);
                k2[i] = pack_f32x2(-w[2 * i + 1] * sn[i], w[2 * i] * sn[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                k1[i] = pack_f32x2(w[2 * i] * cs[2 * i], w[2 * i + 1] * cs[2 * i + 1]);
                k2[i] = pack_f32x2(-w[2 * i + 4] * sn[2 * i], -w[2 * i + 5] * sn[2 * i + 1]);
                k1[i + 2] = pack_f32x2(w[2 * i + 4] * cs[2 * i], w[2 * i + 5] * cs[2 * i + 1]);
                k2[i + 2] = pack_f32x2(w[2 * i] * sn[2 * i], w[2 * i + 1] * sn[2 * i + 1]);
            }
        }
    }
    uint8_t *to0 = to + at0 * out_elem, *to1 = to + at1 * out_elem;
    for (int h0 = 0; h0 < count; h0 += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (h0 + i >= count) break;
            uint64_t v[4] = {};
            if (here) {
                raw[i].widen(v);
                if (h0 + i + kAhead < count) raw[i].load(src + at0 * E, src + at1 * E);
            }
            src += x.hs;
            if (weight) {
                uint64_t sq = mul_f32x2(v[0], v[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) sq = fma_f32x2(v[e], v[e], sq);
                float s = low_f32(sq) + high_f32(sq);
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                const float r = rsqrtf(fmaf(s, a.inv_dim, a.eps));
                const uint64_t r2 = pack_f32x2(r, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mul_f32x2(v[e], r2);
            }
            if (turn) {
                uint64_t o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = mul_f32x2(interleaved ? pack_f32x2(high_f32(v[e]), low_f32(v[e])) : v[e ^ 2], k2[e]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fma_f32x2(v[e], k1[e], o[e]);
            } else if (weight) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mul_f32x2(v[e], k1[e]);
            }
            if (here && there) store8<FORM, OT>(to0, to1, a.out_dtype, v);
            to0 += step;
            to1 += step;
        }
    }
}

template <int DT, int OT, int FORM, bool APPEND>
static cudaError_t launch_rotary_typed(RotArgs a, int n_sm, cudaStream_t st) {
    const int lanes = a.dim <= 64 ? 8 : 16, kinds = APPEND ? 3 : 1;
    // as many heads to a group as leave groups for the SMs' threads
    const long long want = (long long)n_sm * 2048 / lanes;
    long long slices = 0;
    for (a.per_group = kRotMost; ; a.per_group /= 2) {
        slices = 0;
        for (int i = 0; i < kinds; ++i) slices += a.x[i].slices = (a.x[i].heads + a.per_group - 1) / a.per_group;
        if (a.per_group == 1 || a.tokens * slices >= want) break;
    }
    a.by_slices = divisor_of((uint32_t)slices);
    const long long tokens = 32 / lanes, warps = (a.tokens + tokens - 1) / tokens * slices, grid = (warps + kRotThreads / 32 - 1) / (kRotThreads / 32);
    if (lanes == 8) return launch_pdl(rotary_kernel<DT, OT, 8, FORM, APPEND>, dim3((unsigned)grid), dim3(kRotThreads), 0, st, a);
    return launch_pdl(rotary_kernel<DT, OT, 16, FORM, APPEND>, dim3((unsigned)grid), dim3(kRotThreads), 0, st, a);
}
template <int DT, int FORM, bool APPEND>
static cudaError_t launch_rotary_out(const RotArgs& a, int n_sm, cudaStream_t st) {
    if constexpr (FORM == kSingle) {
        return launch_rotary_typed<DT, kAnyType, kSingle, APPEND>(a, n_sm, st);
    } else {
        if (a.out_dtype == SAEM_OUT_BF16) return launch_rotary_typed<DT, SAEM_OUT_BF16, FORM, APPEND>(a, n_sm, st);
        if (APPEND || a.out_dtype == SAEM_OUT_F16) return launch_rotary_typed<DT, SAEM_OUT_F16, FORM, APPEND>(a, n_sm, st);
        return launch_rotary_typed<DT, APPEND ? SAEM_OUT_F16 : SAEM_OUT_F32, FORM, APPEND>(a, n_sm, st);
    }
}
template <int DT, bool APPEND>
static cudaError_t launch_rotary_form(const RotArgs& a, int aligned, int n_sm, cudaStream_t st) {
    const bool whole = a.interleaved || a.rot == 0;
    if (aligned >= 8 && whole) return launch_rotary_out<DT, kWhole, APPEND>(a, n_sm, st);
    return aligned >= 4 && !whole ? launch_rotary_out<DT, kRuns, APPEND>(a, n_sm, st) : launch_rotary_out<DT, kSingle, APPEND>(a, n_sm, st);
}
// aligned: the elements to which every head's address is a multiple (1, 4 or 8)
template <bool APPEND>
static int launch_rotary(const RotArgs& a, int x_dtype, int aligned, cudaStream_t st) {
    int n_sm;
    if (sm_count(&n_sm) != cudaSuccess) return SAEM_ERR_CUDA;
    const cudaError_t e = x_dtype == SAEM_OUT_F32    ? launch_rotary_form<SAEM_OUT_F32, APPEND>(a, aligned, n_sm, st)
                          : x_dtype == SAEM_OUT_BF16 ? launch_rotary_form<SAEM_OUT_BF16, APPEND>(a, aligned, n_sm, st)
                                                     : launch_rotary_form<SAEM_OUT_F16, APPEND>(a, aligned, n_sm, st);
    return e == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}
// The most elements (1, 4 or 8; at most `aligned`) that the heads' addresses are multiples of; *ok: they are aligned to their elements.
static int heads_aligned(const void* p, int dtype, int64_t tokens, int64_t heads, int64_t ts, int64_t hs, int aligned, bool* ok) {
    const int e = head_elem(dtype);
    *ok = *ok && (uintptr_t)p % e == 0;
    // 16 bytes at a time at most
    while (aligned > 1 && ((uintptr_t)p % (aligned * e > 16 ? 16 : aligned * e) || (tokens > 1 && ts % aligned) || (heads > 1 && hs % aligned))) aligned = aligned == 8 ? 4 : 1;
    return aligned;
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
    int aligned = heads_aligned(x, c->x_dtype, c->tokens, c->heads, c->x_token_stride, c->x_head_stride, 8, &ok);
    aligned = heads_aligned(out, c->out_dtype, c->tokens, c->heads, c->out_token_stride, c->out_head_stride, aligned, &ok);
    if (!ok) return SAEM_ERR_ALIGNMENT;
    RotArgs a = {};
    a.dim = c->rotary.head_dim; a.rot = c->rotary.rotary_dim; a.interleaved = c->rotary.interleaved;
    a.eps = c->rotary.eps; a.amplitude = c->rotary.amplitude;
    a.w_bf16 = c->w_dtype == SAEM_OUT_BF16;
    a.turns = turns; a.positions = positions; a.tokens = c->tokens;
    const int e = head_elem(c->x_dtype), oe = head_elem(c->out_dtype);
    a.inv_dim = 1.f / (float)a.dim;
    a.w_runs = (uintptr_t)w % (4 * head_elem(c->w_dtype)) == 0;
    a.x[0] = {static_cast<const uint8_t*>(x), c->x_token_stride * e, c->x_head_stride * e, c->heads, 0};
    a.w[0] = w;
    a.out = static_cast<uint8_t*>(out); a.out_ts = c->out_token_stride * oe; a.out_hs = c->out_head_stride * oe; a.out_dtype = c->out_dtype;
    return launch_rotary<false>(a, c->x_dtype, aligned, (cudaStream_t)stream);
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
    int aligned = heads_aligned(k, c->x_dtype, b->tokens, cache->kv_heads, c->k_token_stride, c->k_head_stride, 8, &ok);
    aligned = heads_aligned(v, c->x_dtype, b->tokens, cache->kv_heads, c->v_token_stride, c->v_head_stride, aligned, &ok);
    if (q) {
        aligned = heads_aligned(q, c->x_dtype, b->tokens, q_heads, c->q_token_stride, c->q_head_stride, aligned, &ok);
        aligned = heads_aligned(q_out, cache->dtype, b->tokens, q_heads, c->out_token_stride, c->out_head_stride, aligned, &ok);
    }
    if (!ok) return SAEM_ERR_ALIGNMENT;
    RotArgs a = {};
    a.dim = dim; a.rot = c->rotary.rotary_dim; a.interleaved = c->rotary.interleaved;
    a.eps = c->rotary.eps; a.amplitude = c->rotary.amplitude;
    a.w_bf16 = c->w_dtype == SAEM_OUT_BF16;
    a.turns = turns; a.positions = positions; a.tokens = b->tokens;
    const int e = head_elem(c->x_dtype);
    a.inv_dim = 1.f / (float)dim;
    a.w_runs = ((uintptr_t)w_q | (uintptr_t)w_k) % (4 * head_elem(c->w_dtype)) == 0;
    a.by_page = divisor_of(cache->page_size);
    a.x[0] = {static_cast<const uint8_t*>(q), c->q_token_stride * e, c->q_head_stride * e, q_heads, 0};
    a.x[1] = {static_cast<const uint8_t*>(k), c->k_token_stride * e, c->k_head_stride * e, cache->kv_heads, 0};
    a.x[2] = {static_cast<const uint8_t*>(v), c->v_token_stride * e, c->v_head_stride * e, cache->kv_heads, 0};
    a.w[0] = w_q; a.w[1] = w_k;
    a.out = static_cast<uint8_t*>(q_out); a.out_ts = c->out_token_stride * 2; a.out_hs = c->out_head_stride * 2; a.out_dtype = cache->dtype;
    a.cache = *cache; a.batch = *b; a.status = status;
    return launch_rotary<true>(a, c->x_dtype, aligned, (cudaStream_t)stream);
}
