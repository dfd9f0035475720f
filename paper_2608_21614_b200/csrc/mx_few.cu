// The MoE step over microscaled 4-bit experts for up to 8 tokens, in two launches (SAEM_FFN_MX contexts).
//
//     route:    top-k of the logits, softmax over the k winners
//     launch 1: h[t, e] = silu(Wg_e x_t) * (Wu_e x_t) for the chosen pairs
//     launch 2: out[t] = sum over the chosen e of w[t, e] Wd_e h[t, e]   (+ the always-on experts, weight 1)
//
// The bytes of the active experts are the bound, and at one token the chain of latencies: launch, logits, top-k, first
// weights, h, first hidden activations, result.  Every CTA therefore routes the batch itself (a warp per token).  The
// weights are the A operand of mma.sync.m16n8k16 and the batch's tokens the 8 columns: a warp takes 16 weight rows x 128
// elements (a unit) at a time, eight codes become four f16 pairs with one cvt each (E2M1 is exact in f16), and a block's
// scale, different in every row, multiplies the fp32 partial sums of its 32 elements.  (tcgen05 would take 128 rows x 8
// columns without any conversion, but its activations have to be split into 4-bit planes first -- mx_moe.cu, from 9
// tokens on.)  Because a column is a token whatever the expert, the second launch's k axis runs over all active experts,
// with the gate weight folded into the column's factor, and the merge over a token's experts costs nothing.
//
// The activations are f16, a run of 128 elements of a row at a time brought to [2^14, 2^15) by a power of two that is
// multiplied back in fp32: bf16 activations stay exact unless they are 2^-28 of the run's largest; the hidden activations
// are fp32 between the launches and are rounded here to f16's 11 bits and nowhere else.
#include "mx_common.cuh"
#include "route_row.cuh"
#include "tc_common.cuh"

namespace saem {

constexpr int kFewTokens = 8;
constexpr int kFewPairs = kFewTokens * kFewTokens;           // top_k <= 8
constexpr int kFewActive = kFewPairs + 16;                   // plus the always-on experts
constexpr int kFewWarps = 8;                                 // consumer warps; one more warp copies
constexpr int kFewThreads = (kFewWarps + 1) * 32;
constexpr int kFewMaxStages = 8;
constexpr int kFewStageA = 2 * (kMxBlockCodes / 2 + 2 * kMxPiece);   // 64 gate and 64 up rows x 256 elements, with their scales
constexpr int kFewStageB = kMxBlockBytes;
constexpr int kSmemPerSm = 227 * 1024;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Barrier of the consumer warps only.
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kFewWarps * 32) : "memory"); }

// acc += (16 weight rows x 128 elements) x 8 tokens.  Lane (g, t): `row0`, `row1` are the 128-byte code rows (swizzled
// by g) that it reads as rows g and g + 8; its words of block b are elements 32 b + 8 t .. + 7, the lane's part of two
// MMAs.  The 8 rows x 16 bytes of one load meet every bank once, thanks to the swizzle.
__device__ __forceinline__ void unit_mma(const uint8_t* row0, const uint8_t* row1, uint32_t scales0, uint32_t scales1, int span,
                                         const __half* x, float f0, float f1, int lane, float (&acc)[4]) {
    const int g = lane >> 2, t = lane & 3;
    float s0[4], s1[4], part[4] = {0.f, 0.f, 0.f, 0.f};
    mx_scales4(scales0, s0);
    mx_scales4(scales1, s1);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        const int at = (((span * 4 + b) ^ g) << 4) + 4 * t;
        uint32_t p[4], q[4];
        mx_decode8(*reinterpret_cast<const uint32_t*>(row0 + at), p);
        mx_decode8(*reinterpret_cast<const uint32_t*>(row1 + at), q);
        const uint4 v = *reinterpret_cast<const uint4*>(x + b * kMxBlock);
        float m[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(m, p[0], q[0], p[1], q[1], v.x, v.y);
        mma_f16(m, p[2], q[2], p[3], q[3], v.z, v.w);
        part[0] += s0[b] * m[0];
        part[1] += s0[b] * m[1];
        part[2] += s1[b] * m[2];
        part[3] += s1[b] * m[3];
    }
    acc[0] += f0 * part[0];
    acc[1] += f1 * part[1];
    acc[2] += f0 * part[2];
    acc[3] += f1 * part[3];
}

// Elements 4 lane .. + 3 of a 128-element run to f16 at dst; returns the factor to every lane.  A run with an infinity
// or NaN keeps its values (factor 1): every output of that row is then not finite either.
__device__ __forceinline__ float stage_run(const float (&v)[4], __half* dst, int lane) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = __reduce_max_sync(0xffffffffu, m);
    int e = (int)(m >> 23);
    e = e == 255 ? 141 : max(e, 15);                         // both powers are normal numbers
    const float up = __uint_as_float((uint32_t)(268 - e) << 23);
    const __half2 lo = __floats2half2_rn(v[0] * up, v[1] * up), hi = __floats2half2_rn(v[2] * up, v[3] * up);
    *reinterpret_cast<uint2*>(dst + 4 * lane) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    return __uint_as_float((uint32_t)(e - 14) << 23);
}

struct FewShared {
    alignas(8) uint64_t full[kFewMaxStages], empty[kFewMaxStages];
    int idx[kFewPairs];
    float w[kFewPairs];
    uint32_t mask[4];
    int n_active;
    int16_t expert[kFewActive];
    int8_t slot_of_token[kFewActive][kFewTokens];            // j of the token's pair with this expert, -1: none
    int abort_flag;
};

// Routes the batch (one consumer warp per token) and lists the active experts in ascending order, the always-on ones
// last; experts without a slot are left out (status word).  All threads call it; ends with a barrier.
__device__ __forceinline__ void few_route(FewShared& s, const MxFewArgs& a, const SlotTable& tab, int n_stage, bool report) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, P = a.T * a.k;
    if (threadIdx.x == 0) {
        for (int i = 0; i < n_stage; ++i) {
            mbar_init(smem_u32(&s.full[i]), 1);
            mbar_init(smem_u32(&s.empty[i]), kFewWarps);
        }
        s.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 4) s.mask[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < kFewActive * kFewTokens; i += kFewThreads) (&s.slot_of_token[0][0])[i] = -1;
    if (warp < a.T) route_row(a.logits + (size_t)warp * a.E, a.E, a.k, a.renorm, lane, s.idx + warp * a.k, s.w + warp * a.k);
    __syncthreads();
    const int e = threadIdx.x < P ? s.idx[threadIdx.x] : -1;
    const bool have = e >= 0 && tab.slot[e] >= 0;
    if (have) atomicOr(&s.mask[e >> 5], 1u << (e & 31));
    else if (e >= 0 && report) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
    __syncthreads();
    if (have) {
        int p = __popc(s.mask[e >> 5] & ((1u << (e & 31)) - 1u));
        for (int q = 0; q < (e >> 5); ++q) p += __popc(s.mask[q]);
        s.expert[p] = (int16_t)e;
        s.slot_of_token[p][threadIdx.x / a.k] = (int8_t)(threadIdx.x % a.k);
    }
    if (threadIdx.x == 0) {
        int n = __popc(s.mask[0]) + __popc(s.mask[1]) + __popc(s.mask[2]) + __popc(s.mask[3]);
        for (int q = 0; q < a.S; ++q) {
            if (tab.slot[a.E + q] < 0) {
                if (report) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
                continue;
            }
            s.expert[n] = (int16_t)(a.E + q);
            for (int t = 0; t < a.T; ++t) s.slot_of_token[n][t] = 0;
            ++n;
        }
        s.n_active = n;
    }
    __syncthreads();
}
// Row of h that holds (token t, active expert): the pair's id, the always-on experts' rows behind the pairs.
__device__ __forceinline__ int few_row(const FewShared& s, const MxFewArgs& a, int active, int t) {
    const int j = s.slot_of_token[active][t], e = s.expert[active];
    return e < a.E ? t * a.k + j : a.T * a.k + (e - a.E) * a.T + t;
}
// At an abort: copies that are still under way land before the CTA ends.
__device__ __noinline__ void few_drain(FewShared& s, int n_stage, int issued, int* status) {
    for (int i = max(0, issued - n_stage); i < issued; ++i) {
        s.abort_flag = 0;
        mbar_wait(smem_u32(&s.full[i % n_stage]), (i / n_stage) & 1, &s.abort_flag, status);
        s.abort_flag = 1;
    }
}

// Gate, and gate/up projection: items are (active expert, 64 hidden units), each warp 8 of them, its MMA's rows the 8
// gate and the 8 up rows (so that a thread holds gate and up of the same unit).  x stays in shared memory for all items.
__global__ void __launch_bounds__(kFewThreads)
mx_few_gate_up_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ FewShared s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n_span = a.d / kMxSpan, n_chunk = mx_chunks(a.d), pitch = a.d + 32;   // f16 elements; 64 bytes off a multiple of 128
    const int n = a.stages_a;
    __half* xs = reinterpret_cast<__half*>(smem + n * kFewStageA);             // [T][pitch]
    float* xf = reinterpret_cast<float*>(xs + (size_t)a.T * pitch);            // [n_span][8]
    volatile int* abort_p = &s.abort_flag;
    pdl_wait();
    pdl_launch_dependents();
    few_route(s, a, tab, n, blockIdx.x == 0);
    if (blockIdx.x == 0 && threadIdx.x < a.T * a.k) {
        a.topk_idx[threadIdx.x] = s.idx[threadIdx.x];
        a.topk_w[threadIdx.x] = s.w[threadIdx.x];
    }
    const int per = a.f / 64, total = s.n_active * per;
    if (warp == kFewWarps) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
                const int act = i / per, part = i - act * per, half = part & 1;
                const uint8_t* w = a.slot_region + (size_t)tab.slot[s.expert[act]] * a.slot_bytes +
                                   (size_t)(part >> 1) * n_chunk * 2 * kMxBlockBytes;
                for (int c = 0; c < n_chunk; ++c, ++it, w += 2 * kMxBlockBytes) {
                    const int st = it % n;
                    if (it >= n) {
                        ok = mbar_wait(smem_u32(&s.empty[st]), (it / n - 1) & 1, abort_p, a.status);
                        if (!ok) break;
                    }
                    const uint32_t bar = smem_u32(&s.full[st]), dst = smem_u32(smem) + st * kFewStageA;
                    mbar_expect_tx(bar, kFewStageA);
#pragma unroll
                    for (int m = 0; m < 2; ++m) {                              // gate, up: codes of the half, scales of the block
                        bulk_g2s(dst + m * (kMxBlockCodes / 2), w + m * kMxBlockBytes + half * (kMxBlockCodes / 2), kMxBlockCodes / 2, bar);
                        bulk_g2s(dst + kMxBlockCodes + m * 2 * kMxPiece, w + m * kMxBlockBytes + kMxBlockCodes, 2 * kMxPiece, bar);
                    }
                }
            }
            if (!ok) few_drain(s, n, it, a.status);
        }
        return;
    }
    for (int i = warp; i < a.T * n_span; i += 4 * kFewWarps) {                 // four runs' loads under way at a time
        uint2 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * kFewWarps < a.T * n_span)
                q[u] = reinterpret_cast<const uint2*>(a.x + (size_t)(i + u * kFewWarps) * kMxSpan)[lane];   // rows follow each other
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = i + u * kFewWarps;
            if (at >= a.T * n_span) break;
            const int r = at / n_span, sp = at - r * n_span;
            const float v[4] = {__uint_as_float(q[u].x << 16), __uint_as_float(q[u].x & 0xFFFF0000u),
                                __uint_as_float(q[u].y << 16), __uint_as_float(q[u].y & 0xFFFF0000u)};
            const float f = stage_run(v, xs + (size_t)r * pitch + sp * kMxSpan, lane);
            if (lane == 0) xf[sp * 8 + r] = f;
        }
    }
    consumer_sync();
    // columns beyond the batch repeat its last token; their sums are not used
    const __half* xrow = xs + (size_t)min(g, a.T - 1) * pitch + 8 * t;
    const int c0 = min(2 * t, a.T - 1), c1 = min(2 * t + 1, a.T - 1);
    const int local = warp * 8 + g;                                            // row within the half block
    int it = 0;
    bool ok = true;
    for (int i = blockIdx.x; i < total; i += gridDim.x) {
        const int act = i / per, part = i - act * per, row = (part & 1) * 64 + local;
        const int scale_at = (row & 31) * 16 + (row >> 5) * 4;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (int c = 0; c < n_chunk; ++c, ++it) {
            const int st = it % n;
            ok = ok && mbar_wait(smem_u32(&s.full[st]), (it / n) & 1, abort_p, a.status);
            const uint8_t* base = smem + (size_t)st * kFewStageA;
            if (ok)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int sp = 2 * c + q;
                    if (sp >= n_span) break;
                    const uint8_t* sc = base + kMxBlockCodes + q * kMxPiece + scale_at;
                    unit_mma(base + local * 128, base + kMxBlockCodes / 2 + local * 128, *reinterpret_cast<const uint32_t*>(sc),
                             *reinterpret_cast<const uint32_t*>(sc + 2 * kMxPiece), q, xrow + sp * kMxSpan, xf[sp * 8 + c0],
                             xf[sp * 8 + c1], lane, acc);
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s.empty[st]));
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int tok = 2 * t + q;
            if (ok && tok < a.T && s.slot_of_token[act][tok] >= 0)
                a.h[(size_t)few_row(s, a, act, tok) * a.f + part * 64 + local] = acc[q] / (1.f + expf(-acc[q])) * acc[q + 2];
        }
    }
}

// Down projection and merge.  A cluster owns 128 output columns, its CTAs equal parts of the k axis (active experts x
// chunks of 256 hidden units); each warp has 16 of the columns.  The parts meet in distributed shared memory, in order.
__global__ void __launch_bounds__(kFewThreads)
mx_few_down_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ FewShared s;
    __shared__ alignas(16) float sums[128 * kFewTokens];                       // [output column][token]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    constexpr int kPitch = kMxChunk + 32;                                      // f16 elements between staged rows
    const int n = a.stages_b, n_chunk = mx_chunks(a.f), n_span = a.f / kMxSpan;
    __half* hs = reinterpret_cast<__half*>(smem + n * kFewStageB);             // [2][T][kPitch]
    float* hf = reinterpret_cast<float*>(hs + (size_t)2 * a.T * kPitch);       // [2][2 spans][8]: factor x gate weight
    volatile int* abort_p = &s.abort_flag;
    // The logits are complete when this launch starts (the CTAs of the first one wait for them before they let it begin)
    // and no weight is written by the first launch: only h has to be waited for.
    few_route(s, a, tab, n, false);
    const int all = s.n_active * n_chunk, rank = (int)cluster_ctarank();
    const int q0 = (int)((long long)all * rank / a.split_b), q1 = (int)((long long)all * (rank + 1) / a.split_b);
    const size_t tile = blockIdx.x / a.split_b;
    bool ok = true;
    if (warp == kFewWarps) {
        if (lane == 0) {
            int it = 0;
            for (int q = q0; q < q1; ++q, ++it) {
                const int st = it % n, act = q / n_chunk;
                if (it >= n) {
                    ok = mbar_wait(smem_u32(&s.empty[st]), (it / n - 1) & 1, abort_p, a.status);
                    if (!ok) break;
                }
                mbar_expect_tx(smem_u32(&s.full[st]), kMxBlockBytes);
                bulk_g2s(smem_u32(smem) + st * kFewStageB,
                         a.slot_region + (size_t)tab.slot[s.expert[act]] * a.slot_bytes +
                             (mx_gate_up_blocks(a.d, a.f) + tile * n_chunk + (q - act * n_chunk)) * kMxBlockBytes,
                         kMxBlockBytes, smem_u32(&s.full[st]));
            }
            if (!ok) few_drain(s, n, it, a.status);
        }
        __syncwarp();
        pdl_wait();
        pdl_launch_dependents();
    } else {
        pdl_wait();
        pdl_launch_dependents();
        // A chunk's hidden activations: warp w loads token w's two runs (a lane four elements of each) one chunk ahead.
        float4 v[2];
        auto fetch = [&](int q) {
            const int act = q / n_chunk, c = q - act * n_chunk;
            if (warp >= a.T || q >= q1) return;
            const bool on = s.slot_of_token[act][warp] >= 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (on && 2 * c + i < n_span)
                    v[i] = __ldcg(reinterpret_cast<const float4*>(a.h + (size_t)few_row(s, a, act, warp) * a.f + (2 * c + i) * kMxSpan) + lane);
            }
        };
        const int crow = min(g, a.T - 1), c0 = min(2 * t, a.T - 1), c1 = min(2 * t + 1, a.T - 1);
        const int r0 = warp * 16 + g, r1 = r0 + 8;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        fetch(q0);
        for (int q = q0, it = 0; q < q1; ++q, ++it) {
            const int act = q / n_chunk, c = q - act * n_chunk, buf = it & 1;
            __half* hb = hs + (size_t)buf * a.T * kPitch;
            float* fb = hf + buf * 16;
            if (warp < a.T) {
                const int j = s.slot_of_token[act][warp];
                const float w = j < 0 ? 0.f : s.expert[act] < a.E ? s.w[warp * a.k + j] : 1.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float e[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    const float f = stage_run(e, hb + (size_t)warp * kPitch + i * kMxSpan, lane);
                    if (lane == 0) fb[i * 8 + warp] = f * w;
                }
            }
            fetch(q + 1);
            consumer_sync();                                                   // two buffers: the other one may still be read
            const int st = it % n;
            ok = ok && mbar_wait(smem_u32(&s.full[st]), (it / n) & 1, abort_p, a.status);
            const uint8_t* base = smem + (size_t)st * kFewStageB;
            if (ok)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (2 * c + i >= n_span) break;
                    const uint8_t* sc = base + kMxBlockCodes + i * kMxPiece;
                    unit_mma(base + r0 * 128, base + r1 * 128,
                             *reinterpret_cast<const uint32_t*>(sc + (r0 & 31) * 16 + (r0 >> 5) * 4),
                             *reinterpret_cast<const uint32_t*>(sc + (r1 & 31) * 16 + (r1 >> 5) * 4), i,
                             hb + (size_t)crow * kPitch + i * kMxSpan + 8 * t, fb[i * 8 + c0], fb[i * 8 + c1], lane, acc);
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s.empty[st]));
        }
        *reinterpret_cast<float2*>(&sums[r0 * kFewTokens + 2 * t]) = make_float2(acc[0], acc[1]);
        *reinterpret_cast<float2*>(&sums[r1 * kFewTokens + 2 * t]) = make_float2(acc[2], acc[3]);
    }
    __syncthreads();
    cluster_sync_all();
    // this CTA's share of the 128 columns, every token: the parts in order
    const int share = 128 / a.split_b;
    for (int i = threadIdx.x; i < share * a.T; i += kFewThreads) {
        const int tok = i / share, col = rank * share + (i - tok * share);
        float v = 0.f;
        for (int r = 0; r < a.split_b; ++r) {
            float p;
            asm volatile("ld.shared::cluster.f32 %0, [%1];"
                         : "=f"(p) : "r"(mapa_u32(smem_u32(&sums[col * kFewTokens + tok]), r)) : "memory");
            v += p;
        }
        const size_t at = (size_t)tok * a.d + tile * 128 + col;
        if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.out)[at] = v;
    }
    __syncwarp();
    cluster_sync_all();                                                        // no CTA ends while another reads its sums
}

// The staged x may take 64 KB; beyond that (8 tokens of d_model > 4096) the packed form takes over.
bool mx_few_supported(int T, int k, int d) { return T <= kFewTokens && k <= kFewTokens && (long long)T * d <= 32768; }

cudaError_t launch_mx_few(MxFewArgs a, const SlotTable& tab, int n_sm, cudaStream_t st, int* n_launch) {
    static bool done[64];
    if (first_call_on_device(done)) {
        cudaError_t e = cudaFuncSetAttribute(mx_few_gate_up_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 216 * 1024);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_few_down_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 216 * 1024);
        if (e != cudaSuccess) return e;
    }
    const int pairs = a.T * a.k, active = (pairs < a.E ? pairs : a.E) + a.S;
    const long long items = (long long)active * (a.f / 64);
    const size_t x_bytes = (size_t)a.T * (a.d + 32) * 2 + (size_t)(a.d / kMxSpan) * 8 * 4;
    // one CTA per SM with a deep ring where the items do not outnumber the SMs, else two
    const int per_sm_a = items > n_sm ? 2 : 1;
    const int budget = per_sm_a == 2 ? kSmemPerSm / 2 - 4096 : 140 * 1024;
    a.stages_a = (int)((budget - (long long)x_bytes) / kFewStageA);
    if (a.stages_a > kFewMaxStages) a.stages_a = kFewMaxStages;
    if (a.stages_a < 2) a.stages_a = 2;
    const size_t smem_a = (size_t)a.stages_a * kFewStageA + x_bytes;
    const long long most = (long long)n_sm * per_sm_a;
    cudaError_t e = launch_pdl(mx_few_gate_up_kernel, dim3((unsigned)(items < most ? items : most)), dim3(kFewThreads), smem_a, st, a, tab);
    if (e != cudaSuccess) return e;
    *n_launch += 1;
    a.split_b = 8;
    const size_t h_bytes = (size_t)2 * a.T * (kMxChunk + 32) * 2 + 2 * 16 * 4;
    a.stages_b = 4;
    const size_t smem_b = (size_t)a.stages_b * kFewStageB + h_bytes;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.split_b;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.d / 128 * a.split_b));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = smem_b;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, mx_few_down_kernel, a, tab);
    if (e == cudaSuccess) *n_launch += 1;
    return e;
}

}  // namespace saem
