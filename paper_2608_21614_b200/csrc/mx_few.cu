// The MoE step over microscaled 4-bit experts for up to 8 tokens, in two launches (SAEM_FFN_MX contexts).
//
//     route:    top-k of the logits, softmax over the k winners
//     launch 1: h[t, e] = w[t, e] silu(Wg_e x_t) * (Wu_e x_t) for the chosen pairs, 0 for the others
//     launch 2: out[t] = sum over the active e of Wd_e h[t, e]   (always-on experts with weight 1)
//
// The bytes of the active experts are the bound, and at one token the chain of latencies: launch, logits, top-k, first
// weights, h, result.  Every CTA therefore routes the batch itself (a warp per token).  The products are those of
// mx_moe.cu (4-bit weights straight from shared memory to tcgen05 kind::mxf4, activations as five 4-bit planes), but a
// column is a token whatever the expert: x's tile stays in shared memory for all items, the second launch's k axis runs
// over all active experts, and the merge over a token's experts costs nothing because h carries the gate weight.  (The
// same two launches with mma.sync, the weights converted to f16, were bound by instruction issue: 50 us for 8 tokens of a
// 2048 x 768 layer of 128 experts against 26.5 us, 93 MB at 3.5 TB/s.)  One token takes 14 us: routing 1.7 us, the first
// weights' way 1 us, the products 2.5 us, their sums and planes of h 2 us, the hand-over 1.2 us, the down projection with the
// cluster's sum 3 us, and the two launches.  A CTA of the second launch (99 KB) finds no place beside one of the first (up to
// 222 KB and all of tensor memory), so its routing and first weights begin when a CTA of the first launch ends on its SM.
#include "mx_planes.cuh"
#include "route_row.cuh"

namespace saem {

constexpr int kFewTokens = 8;
constexpr int kFewPairs = kFewTokens * kFewTokens;           // top_k <= 8
constexpr int kFewActive = kFewPairs + 16;                   // plus the always-on experts
constexpr int kFewThreads = 320;                             // warp 0: copies, warp 1: MMA issue, warps 2-9: epilogue
constexpr int kGateUpThreads = kFewThreads + 256;            // gate/up: warps 10-17 split x into planes while the others route
constexpr int kFewMaxStages = 8;
constexpr int kFewSplit = 8;                                 // CTAs of a cluster: parts of the down projection's k axis
using FewTile = TileShape<kFewTokens>;
constexpr int kFewHalf = kMxBlockCodes / 2 + 2 * kMxPiece;     // 64 rows of a block, and its scales
constexpr int kFewStageB = kMxBlockBytes + FewTile::kBytes;
constexpr int kFewStagesB = 4;
constexpr int kFewSfB = 8 + FewTile::kScaleCols;             // tensor-memory columns of a stage's scales (gate/up: 16, x's are loaded once)
constexpr int kFewMaxChunks = 16;                            // of x: d_model <= 4096

constexpr float kNotChosen = -1.f;                           // gate weights are 0 or more

struct FewShared {
    alignas(8) uint64_t full[kFewMaxStages], empty[kFewMaxStages], acc[2], free[2], x;
    int slot[SAEM_MAX_EXPERTS];
    uint32_t mask[4];
    int n_active;
    int16_t expert[kFewActive];
    float weight[kFewActive][kFewTokens];                    // gate weight of (active expert, token), or kNotChosen
    uint32_t tmem;
    int abort_flag;
};

// What needs no input: barriers, tables.  Ends with a barrier.
__device__ __forceinline__ void few_init(FewShared& s, const MxFewArgs& a, const SlotTable& tab, int n_stage) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < n_stage; ++i) {
            mbar_init(smem_u32(&s.full[i]), 1);
            mbar_init(smem_u32(&s.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s.acc[i]), 1);
            mbar_init(smem_u32(&s.free[i]), 4);
        }
        mbar_init(smem_u32(&s.x), 16);
        s.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 4) s.mask[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < a.E + a.S; i += blockDim.x) s.slot[i] = tab.slot[i];
    for (int i = threadIdx.x; i < kFewActive * kFewTokens; i += blockDim.x) (&s.weight[0][0])[i] = kNotChosen;
    __syncthreads();
}
// Routes the batch (one warp per token) and lists the active experts in ascending order, the always-on ones last; experts
// without a slot are left out (status word).  The first kFewThreads threads call it; ends with a barrier of theirs.
__device__ __forceinline__ void few_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kFewThreads) : "memory"); }
__device__ __forceinline__ void few_route(FewShared& s, const MxFewArgs& a, bool report) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int e = -1;
    float w = 0.f;
    if (warp < a.T) {
        route_few(a.logits + (size_t)warp * a.E, a.E, a.k, a.renorm, lane, e, w);
        if (lane >= a.k) {
            e = -1;
        } else {
            if (report) {
                a.topk_idx[warp * a.k + lane] = e;
                a.topk_w[warp * a.k + lane] = w;
            }
            if (s.slot[e] >= 0) {
                atomicOr(&s.mask[e >> 5], 1u << (e & 31));
            } else {
                if (report) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
                e = -1;
            }
        }
    }
    few_sync();
    const uint32_t m0 = s.mask[0], m1 = s.mask[1], m2 = s.mask[2], m3 = s.mask[3];
    if (e >= 0) {
        const int word = e >> 5;
        const int p = __popc(s.mask[word] & ((1u << (e & 31)) - 1u)) + (word > 0 ? __popc(m0) : 0) + (word > 1 ? __popc(m1) : 0) +
                      (word > 2 ? __popc(m2) : 0);
        s.expert[p] = (int16_t)e;
        s.weight[p][warp] = w;
    }
    if (threadIdx.x == kFewThreads - 1) {
        int n = __popc(m0) + __popc(m1) + __popc(m2) + __popc(m3);
        for (int q = 0; q < a.S; ++q) {
            if (s.slot[a.E + q] < 0) {
                if (report) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
                continue;
            }
            s.expert[n] = (int16_t)(a.E + q);
            for (int t = 0; t < a.T; ++t) s.weight[n][t] = 1.f;
            ++n;
        }
        s.n_active = n;
    }
    few_sync();
}
// Where a warp gave up a wait: the copies and MMAs that are still under way, which take microseconds, land before the CTA
// ends.  By the clock: waiting on their barriers, as the other 4-bit kernels do, makes every call longer by its code alone
// (one token 0.25 us of 14.6 us).  Behind a barrier of the CTA.
__device__ __forceinline__ void few_settle(const FewShared& s) {
    if (!s.abort_flag) return;
    const unsigned long long t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) {}
}
__device__ __forceinline__ void few_alloc(FewShared& s, uint32_t cols) {
    if (threadIdx.x >> 5 == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "r"(cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
}
__device__ __forceinline__ void few_free(uint32_t tmem, uint32_t cols) {
    if (threadIdx.x >> 5 == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
    }
}

// Gate, and gate/up projection: items are (active expert, 128 hidden units), or halves of that (HALF) while those would not
// occupy the SMs: a stage then holds 64 rows of the gate block and of the up block, and the MMA's other 64 rows read
// whatever lies beside them (inside the CTA's shared memory), for lanes that nobody looks at.
template <bool HALF>
__global__ void __launch_bounds__(kGateUpThreads, 1)
mx_few_gate_up_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ FewShared s;
    constexpr int kStage = 2 * (HALF ? kFewHalf : kMxBlockBytes);
    constexpr int kCodes = HALF ? kMxBlockCodes / 2 : kMxBlockCodes;
    const uint32_t raw = smem_u32(smem_raw), xs_addr = (raw + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, nc = mx_chunks(a.d), n = a.stages_a;
    uint8_t* xs = smem_raw + (xs_addr - raw);                                  // x's tiles, one per chunk (7 KB each)
    const uint32_t base = xs_addr + max(nc * FewTile::kBytes, 8192);           // the ring: 8 KB before it and behind it are ours
    volatile int* abort_p = &s.abort_flag;
    few_alloc(s, 512);
    few_init(s, a, tab, n);
    pdl_wait();
    pdl_launch_dependents();
    // x's planes: five eighths of the runs (all, if they are few) by warps 10-17 at once, the rest by warps 2-9 after routing
    const int tasks = a.T * nc, mine = tasks <= 16 ? tasks : (tasks * 5 + 7) / 8;
    auto split_x = [&](int begin, int end) {
        constexpr int kAhead = 4;                                              // runs whose loads are under way
        for (int first = begin; first < end; first += 8 * kAhead) {
            uint4 q[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = first + 8 * u, t = i / nc, col = (i - t * nc) * kMxChunk + lane * 8;
                q[u] = i < end && col < a.d ? *reinterpret_cast<const uint4*>(a.x + (size_t)t * a.d + col) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = first + 8 * u, t = i / nc, c = i - t * nc;
                if (i >= end) break;
                float v[8];
                uint32_t codes[kPlanes], scales[kPlanes];
                widen8(q[u], v);
                split_planes(v, lane, codes, scales);
                store_tile_row<kFewTokens>(xs + (size_t)c * FewTile::kBytes, t, lane, codes, scales);
            }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s.x));
    };
    if (warp >= 10) split_x(warp - 10, mine);
    else few_route(s, a, blockIdx.x == 0);
    tc_fence_after();
    const uint32_t tmem = warp_uniform(s.tmem), tmem_sf = tmem + 4 * FewTile::kN;
    const int per = a.f / 128 * (HALF ? 2 : 1), total = (int)warp_uniform(s.n_active) * per;
    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        int st = 0, turn = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            const int act = i / per, part = i - act * per, tile = HALF ? part >> 1 : part;
            const uint8_t* w = a.slot_region + (size_t)warp_uniform(s.slot[s.expert[act]]) * a.slot_bytes + (size_t)tile * nc * 2 * kMxBlockBytes;
            for (int c = 0; c < nc; ++c, w += 2 * kMxBlockBytes) {
                if (turn) {
                    ok = mbar_wait_warp(smem_u32(&s.empty[st]), (turn - 1) & 1, abort_p, a.status);
                    if (!ok) break;
                }
                const uint32_t bar = smem_u32(&s.full[st]), dst = base + st * kStage;
                expect_tx_on(on, bar, kStage);
                if (HALF) {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {                              // codes of gate and up, then the scales of both
                        bulk_g2s_on(on, dst + m * kCodes, w + m * kMxBlockBytes + (part & 1) * kCodes, kCodes, bar);
                        bulk_g2s_on(on, dst + 2 * kCodes + m * 2 * kMxPiece, w + m * kMxBlockBytes + kMxBlockCodes, 2 * kMxPiece, bar);
                    }
                } else {
                    bulk_g2s_on(on, dst, w, kStage, bar);
                }
                if (++st == n) { st = 0; ++turn; }
            }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        const uint64_t codes0 = smem_desc_sw128(base), x0 = smem_desc_sw128(xs_addr), scales0 = smem_desc_scales(base);
        const uint64_t xscales0 = smem_desc_scales(xs_addr + FewTile::kN * 128);
        int st = 0, turn = 0, k = 0;
        bool ok = mbar_wait_warp(smem_u32(&s.x), 0, abort_p, a.status);
        tc_fence_after();
        const uint32_t tmem_x = tmem_sf + n * 16;                              // x's scales stay in tensor memory for all items
        // The copies are waited for with the first item's sums, so a CTA without an item (the grid is made for as many active
        // experts as there can be) starts none: nothing would hold back the end of its memory until they have landed.
        for (int c = 0; c < nc && ok && (int)blockIdx.x < total; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) tc_cp_scales(on, tmem_x + c * 8 + 4 * h, desc_at(xscales0, c * FewTile::kBytes + h * kMxPiece));
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x, ++k) {
            const int set = k & 1;
            const uint32_t acc = tmem + set * 2 * FewTile::kN;
            if (k >= 2) ok = mbar_wait_warp(smem_u32(&s.free[set]), ((k >> 1) - 1) & 1, abort_p, a.status);
            tc_fence_after();
            for (int c = 0; c < nc && ok; ++c) {
                ok = mbar_wait_warp(smem_u32(&s.full[st]), turn & 1, abort_p, a.status);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = st * kStage, sf = tmem_sf + st * 16, sfx = tmem_x + c * 8;
                const uint64_t ds = desc_at(scales0, at), dx = desc_at(x0, c * FewTile::kBytes);
                const int steps = min(4, (a.d - c * kMxChunk) / 64);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * h >= steps) break;
#pragma unroll
                    for (int m = 0; m < 2; ++m)                                // behind the codes of both, or behind each one's own
                        tc_cp_scales(on, sf + m * 8 + 4 * h, desc_at(ds, (HALF ? 2 * kCodes + m * 2 * kMxPiece : m * kMxBlockBytes + kCodes) + h * kMxPiece));
                }
                // a second half's row 64 stands first: its block would begin 8 KB before
                const uint64_t dw = desc_at(codes0, at) - (HALF && (i & 1) ? kCodes / 16 : 0);
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps)
                            tc_mma_mxf4(on, acc + m * FewTile::kN, desc_at(dw, m * (HALF ? kCodes : kMxBlockBytes) + 32 * j), desc_at(dx, 32 * j),
                                        idesc_mxf4(FewTile::kN, (j & 1) * 2), sf + m * 8 + 4 * (j >> 1), sfx + 4 * (j >> 1), c > 0 || j > 0);
                tc_commit_on(on, smem_u32(&s.empty[st]));
                if (++st == n) { st = 0; ++turn; }
            }
            tc_commit_on(on, smem_u32(&s.acc[set]));
        }
    } else if (warp < 10) {
        split_x(mine + warp - 2, tasks);
        // ---------------------------------------------------------------- epilogue
        const int quad = warp & 3, group = (warp - 2) >> 2;                    // each group of four warps has its own accumulators
        const uint32_t acc = tmem + group * 2 * FewTile::kN + ((uint32_t)(quad * 32) << 16);
        int k = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < total; i += gridDim.x, ++k) {
            if ((k & 1) != group) continue;
            const int act = i / per, part = i - act * per, tile = HALF ? part >> 1 : part;
            ok = ok && mbar_wait(smem_u32(&s.acc[group]), (k >> 1) & 1, abort_p, a.status);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (ok && (!HALF || (quad >> 1) == (part & 1))) {
                float v[8], u[8];
                plane_sums<kFewTokens>(acc, v);
                plane_sums<kFewTokens>(acc + FewTile::kN, u);
                tc_fence_before();
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float w = s.weight[act][t];
                    v[t] = w != kNotChosen ? w * swiglu(v[t], u[t]) : 0.f;     // columns of other tokens hold anything
                }
                store_planes<kFewTokens>(v, 0, a.T, a.h_tiles + ((size_t)act * mx_chunks(a.f) + (tile >> 1)) * FewTile::kBytes,
                                         (tile & 1) * 4 + quad, lane);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&s.free[group]));
        }
    }
    __syncthreads();
    few_settle(s);
    few_free(tmem, 512);
}

// One output of the down projection from its token's own experts alone, where the product over all active experts is NaN:
// there an expert whose weights hold a NaN block reaches every token, since 0 * NaN is NaN.  Slow, and only for such outputs.
// `row`: of the 128 rows of the column tile.
__device__ __forceinline__ float few_own_sum(const FewShared& s, const MxFewArgs& a, size_t tile, int tok, int row) {
    const int nc = mx_chunks(a.f), blocks = a.f / kMxBlock;
    auto power = [](int byte) { return __uint_as_float(byte ? (uint32_t)byte << 23 : 1u << 22); };   // 2^(byte - 127)
    float sum = 0.f;
#pragma unroll 1
    for (int i = 0; i < s.n_active * blocks; ++i) {
        const int act = i / blocks, b = i - act * blocks, at = b & 7, half = (at >> 2) * kMxPiece + (at & 3);
        if (s.weight[act][tok] == kNotChosen) continue;
        const uint8_t* w = a.slot_region + (size_t)s.slot[s.expert[act]] * a.slot_bytes + (mx_gate_up_blocks(a.d, a.f) + tile * nc + (b >> 3)) * kMxBlockBytes;
        const uint8_t* h = a.h_tiles + ((size_t)act * nc + (b >> 3)) * FewTile::kBytes;
        const int ws = w[kMxBlockCodes + half + (row & 31) * 16 + (row >> 5) * 4];
        if (ws == 255 || h[FewTile::kN * 128 + half + tok * 16] == 255) return __uint_as_float(0x7FC00000u);
        w += row * 128 + ((at ^ (row & 7)) << 4);
#pragma unroll 1
        for (int p = kPlanes - 1; p >= 0; --p) {
            const int col = p * kFewTokens + tok;                              // below 64: one piece of scales
            const uint8_t* c = h + col * 128 + ((at ^ tok) << 4);
            float part = 0.f;                                                  // of 32 products of E2M1 values: exact
#pragma unroll 1
            for (int q = 0; q < 16; ++q) part += mx_dot2(w[q], c[q]);
            const int e = ws + h[FewTile::kN * 128 + half + (col & 31) * 16 + (col >> 5) * 4] - 254, e0 = e / 2;
            sum += part * power(127 + e0) * power(127 + e - e0);               // in two steps: neither power leaves fp32's range
        }
    }
    return sum;
}

// Down projection and merge.  A cluster owns 128 output columns, its CTAs equal parts of the k axis (active experts x
// chunks of 256 hidden units), whose sums meet in distributed shared memory, in order.
__global__ void __launch_bounds__(kFewThreads, 1)
mx_few_down_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ FewShared s;
    __shared__ alignas(16) float sums[128 * kFewTokens];                       // [output column][token]
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int nc = mx_chunks(a.f);
    constexpr int n = kFewStagesB;
    volatile int* abort_p = &s.abort_flag;
    few_alloc(s, 128);
    few_init(s, a, tab, n);
    // The logits are complete when this launch starts (the CTAs of the first one wait for them before they let it begin)
    // and no weight is written by the first launch: only h has to be waited for.
    few_route(s, a, false);
    tc_fence_after();
    const uint32_t tmem = warp_uniform(s.tmem), tmem_sf = tmem + 64;
    const int all = (int)warp_uniform(s.n_active) * nc, rank = (int)cluster_ctarank();
    const int q0 = all * rank / kFewSplit, q1 = all * (rank + 1) / kFewSplit;
    const size_t tile = blockIdx.x / kFewSplit;
    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        auto weights = [&](int q, int st) {
            const int act = q / nc;
            expect_tx_on(on, smem_u32(&s.full[st]), kFewStageB);
            bulk_g2s_on(on, base + st * kFewStageB,
                        a.slot_region + (size_t)warp_uniform(s.slot[s.expert[act]]) * a.slot_bytes +
                            (mx_gate_up_blocks(a.d, a.f) + tile * nc + (q - act * nc)) * kMxBlockBytes,
                        kMxBlockBytes, smem_u32(&s.full[st]));
        };
        const int early = min(q1, q0 + n);
        for (int q = q0; q < early; ++q) weights(q, q - q0);
        pdl_wait();
        pdl_launch_dependents();
        int st = 0, turn = 0;
        for (int q = q0; q < q1; ++q) {
            if (turn) {
                if (!mbar_wait_warp(smem_u32(&s.empty[st]), (turn - 1) & 1, abort_p, a.status)) break;
                weights(q, st);
            }
            bulk_g2s_on(on, base + st * kFewStageB + kMxBlockBytes, a.h_tiles + (size_t)q * FewTile::kBytes, FewTile::kBytes, smem_u32(&s.full[st]));
            if (++st == n) { st = 0; ++turn; }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        bool ok = true;
        const uint64_t codes0 = smem_desc_sw128(base), scales0 = smem_desc_scales(base);
        int st = 0, turn = 0;
        for (int q = q0; q < q1; ++q) {
            const int c = q % nc;
            ok = mbar_wait_warp(smem_u32(&s.full[st]), turn & 1, abort_p, a.status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t at = st * kFewStageB, sf = tmem_sf + st * kFewSfB;
            const uint64_t dw = desc_at(codes0, at), dx = desc_at(codes0, at + kMxBlockBytes), ds = desc_at(scales0, at);
            const int steps = min(4, (a.f - c * kMxChunk) / 64);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (2 * h >= steps) break;
                tc_cp_scales(on, sf + 4 * h, desc_at(ds, kMxBlockCodes + h * kMxPiece));
                tc_cp_scales(on, sf + 8 + 4 * h, desc_at(ds, kMxBlockBytes + FewTile::kN * 128 + h * kMxPiece));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < steps)
                    tc_mma_mxf4(on, tmem, desc_at(dw, 32 * j), desc_at(dx, 32 * j), idesc_mxf4(FewTile::kN, (j & 1) * 2), sf + 4 * (j >> 1),
                                sf + 8 + 4 * (j >> 1), q > q0 || j > 0);
            tc_commit_on(on, smem_u32(&s.empty[st]));
            if (++st == n) { st = 0; ++turn; }
        }
        tc_commit_on(on, smem_u32(&s.acc[0]));
    } else if (warp < 6) {
        const int quad = warp & 3;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bool ok = mbar_wait(smem_u32(&s.acc[0]), 0, abort_p, a.status);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (ok && q1 > q0) plane_sums<kFewTokens>(tmem + ((uint32_t)(quad * 32) << 16), v);
        tc_fence_before();
        float4* o = reinterpret_cast<float4*>(&sums[(quad * 32 + lane) * kFewTokens]);
        o[0] = make_float4(v[0], v[1], v[2], v[3]);
        o[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    __syncthreads();
    cluster_sync_all();
    pdl_wait();                                                                // out may still be read by what ran before
    // this CTA's share of the 128 columns, every token: the parts in order
    constexpr int kShare = 128 / kFewSplit;
    if (threadIdx.x < kShare * a.T) {
        const int tok = threadIdx.x / kShare, col = rank * kShare + threadIdx.x % kShare;
        float p[kFewSplit], v = 0.f;
#pragma unroll
        for (int r = 0; r < kFewSplit; ++r)
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p[r]) : "r"(mapa_u32(smem_u32(&sums[col * kFewTokens + tok]), r)));
#pragma unroll
        for (int r = 0; r < kFewSplit; ++r) v += p[r];
        if (__builtin_expect(v != v, 0)) v = few_own_sum(s, a, tile, tok, col);
        const size_t at = (size_t)tok * a.d + tile * 128 + col;
        if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.out)[at] = v;
    }
    few_settle(s);
    __syncwarp();
    cluster_sync_all();                                                        // no CTA ends while another reads its sums
    few_free(tmem, 128);
}

// x's tiles (7 KB per 256 elements) stand beside three stages of weights at least.
bool mx_few_supported(int T, int k, int d) { return T <= kFewTokens && k <= kFewTokens && mx_chunks(d) <= kFewMaxChunks; }

cudaError_t launch_mx_few(MxFewArgs a, const SlotTable& tab, int n_sm, cudaStream_t st, int* n_launch) {
    static DeviceOnce once;
    constexpr int kMost = 222 * 1024, kSmemB = kFewStagesB * kFewStageB + 1024;
    cudaError_t e = once_on_device(once, [] {
        cudaError_t s = cudaFuncSetAttribute(mx_few_gate_up_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (s == cudaSuccess) s = cudaFuncSetAttribute(mx_few_gate_up_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (s == cudaSuccess) s = cudaFuncSetAttribute(mx_few_down_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemB);
        return s;
    });
    if (e != cudaSuccess) return e;
    const int pairs = a.T * a.k, active = (pairs < a.E ? pairs : a.E) + a.S;
    long long items = (long long)active * (a.f / 128);
    const bool half = items <= n_sm;
    if (half) items *= 2;
    const int x_bytes = mx_chunks(a.d) * FewTile::kBytes, before = x_bytes > 8192 ? x_bytes : 8192, stage = 2 * (half ? kFewHalf : kMxBlockBytes);
    const int around = 1024 + before + (half ? 8192 : 0);
    a.stages_a = (kMost - around) / stage;
    const int most = kFewMaxStages;                                            // tensor memory: 192 columns of sums, 16 per stage, 8 per chunk of x
    if (a.stages_a > most) a.stages_a = most;
    e = launch_pdl(half ? mx_few_gate_up_kernel<true> : mx_few_gate_up_kernel<false>, dim3((unsigned)(items < n_sm ? items : n_sm)),
                               dim3(kGateUpThreads), (size_t)(around + a.stages_a * stage), st, a, tab);
    if (e != cudaSuccess) return e;
    *n_launch += 1;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kFewSplit;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.d / 128 * kFewSplit));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = kSmemB;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, mx_few_down_kernel, a, tab);
    if (e == cudaSuccess) *n_launch += 1;
    return e;
}

}  // namespace saem
