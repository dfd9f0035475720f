// The expert FFN over microscaled 4-bit experts for rows packed by expert (SAEM_FFN_MX contexts, more than 8 tokens):
// h = silu(Wg x) * (Wu x), y = Wd h on the block-scaled tensor cores (tcgen05 kind::mxf4), which take the 4-bit weights out
// of shared memory as they are.  (Converting them to f16 for mma.sync costs some 150 instructions per 1088 bytes, and that,
// not DRAM, was the bound: 232 us against 120 us now for 16 tokens of a 4096 x 14336 layer of 8 experts.)
//
// The other operand has to be 4-bit too: the activations are split into five 4-bit planes (mx_planes.cuh), whose
// accumulators are added in fp32 in the epilogue.  Prefill pays for it: five times the work at four times bf16's rate.
//
// Few rows per expert: the bound is the weights' bytes.  The step just named moves 749 MB, 6.2 TB/s over all its
// launches; 61 tokens of a 2560 x 1536 layer of 64 + 2 experts take 87 us for 372 MB, of which the launches around the
// products (gate and indices, tiles of x, combine) are some 13 us.  Many rows: 2048 tokens of a 2048 x 1408 layer of 64 + 2
// experts take 525 us (bf16 slots: 375 us).  The MMAs are not the bound there: the tensor pipe is busy for 33 % of the gate/up
// launch and 46 % of the down launch.  With tiles of 32 rows tensor memory holds one set of the gate/up accumulators, so that
// an epilogue and the next item's products take turns, and the ring has three stages.
//
// A tile is R (8, 16, 32) rows of one expert; an item is a tile x 128 hidden units (gate and up accumulators side by
// side) or x 128 output columns.  Tiles of the activations are laid out as the MMA wants them (swizzled codes of
// kPlanes * R columns x 256 elements, then their scales), by mx_tile_kernel for x and by the gate/up epilogue for h --
// where a warp's 32 lanes are 32 hidden units of a row, exactly a block -- so that a stage is two bulk copies.  One
// persistent CTA per SM; where tensor memory allows, two sets of accumulators, so that an epilogue runs beside the next
// item's products.
#include "mx_planes.cuh"

namespace saem {

constexpr int kMoeThreads = 320;            // warp 0: copies, warp 1: MMA issue, warps 2-5 and 6-9: epilogue
constexpr int kMoeMaxStages = 8;

template <int MODE, int R>
struct FfnShape {
    static constexpr int kWBytes = (MODE == 0 ? 2 : 1) * kMxBlockBytes;
    static constexpr int kStageBytes = kWBytes + TileShape<R>::kBytes;
    static constexpr int kAccCols = (MODE == 0 ? 2 : 1) * TileShape<R>::kN; // one set of accumulators
    static constexpr int kSets = 2 * kAccCols <= 384 ? 2 : 1;
    static constexpr int kSfCols = (MODE == 0 ? 16 : 8) + TileShape<R>::kScaleCols;
    static constexpr int kFit = (222 * 1024) / kStageBytes;
    static constexpr int kSfFit = (512 - kSets * kAccCols) / kSfCols;
    static constexpr int kMost = kFit < kSfFit ? kFit : kSfFit;
    static constexpr int kStages = kMost < kMoeMaxStages ? kMost : kMoeMaxStages;
    static constexpr int kSmem = kStages * kStageBytes + 1024;
    static_assert(kStages >= 3 && kSets * kAccCols + kStages * kSfCols <= 512, "tensor memory");
};

// The segments as every kernel here reads them: rows, first row and first tile of each expert.
struct Segments {
    int rows[SAEM_MAX_EXPERTS], start[SAEM_MAX_EXPERTS], tile0[SAEM_MAX_EXPERTS + 1];
    int warp_sum[4];
};
// 128 threads or more; ends with a barrier.  Offsets that do not ascend could name more tiles than the workspace has
// room for (`most`): then there are none, and the status word says so.
template <int R>
__device__ __forceinline__ void read_segments(Segments& s, const int32_t* offsets, int E, int max_rows, int most, int* status) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int v = 0;
    if (threadIdx.x < SAEM_MAX_EXPERTS) {
        const int e = threadIdx.x;
        int lo = max_rows, hi = max_rows;                                      // what is beyond E starts behind the last row
        if (e < E) {
            lo = offsets ? offsets[e] : 0;
            hi = offsets ? offsets[e + 1] : max_rows;
            lo = min(max(lo, 0), max_rows);
            hi = min(max(hi, lo), max_rows);
        }
        s.rows[e] = hi - lo;
        s.start[e] = lo;
        v = (hi - lo + R - 1) / R;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) s.warp_sum[warp] = v;
    }
    __syncthreads();
    if (threadIdx.x < SAEM_MAX_EXPERTS) {
        for (int w = 0; w < warp; ++w) v += s.warp_sum[w];
        const bool fits = s.warp_sum[0] + s.warp_sum[1] + s.warp_sum[2] + s.warp_sum[3] <= most;
        if (!fits) {
            v = s.rows[threadIdx.x] = 0;
            if (threadIdx.x == 0) atomicExch(status, SAEM_ERR_INVALID_ARG);
        }
        s.tile0[threadIdx.x + 1] = v;
        if (threadIdx.x == 0) s.tile0[0] = 0;
    }
    __syncthreads();
}

// x to tiles: one warp per token x 256 elements, eight elements per lane, four lanes per block.  The planes are made once
// and stored in the token's k + S rows (inv_perm; the always-on experts' segments behind them).  inv_perm nullptr: x holds
// packed rows already (k = 1, S = 0).
template <int R>
__global__ void __launch_bounds__(256)
mx_tile_kernel(const uint16_t* __restrict__ x, const int32_t* __restrict__ inv_perm, const int32_t* __restrict__ offsets, int T, int k,
               int S, int E, int K, int most, uint8_t* __restrict__ tiles, int* __restrict__ status) {
    using Ts = TileShape<R>;
    __shared__ Segments s;
    const int lane = threadIdx.x & 31, nc = mx_chunks(K);
    const long long total = (long long)T * nc, first = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    uint32_t codes[kPlanes], scales[kPlanes];
    auto split = [&](long long i) {
        const int t = (int)(i / nc), col = (int)(i - (long long)t * nc) * kMxChunk + lane * 8;
        float v[8];
        widen8(col < K ? *reinterpret_cast<const uint4*>(x + (size_t)t * K + col) : make_uint4(0u, 0u, 0u, 0u), v);
        split_planes(v, lane, codes, scales);
    };
    // Within a step x is older than the launch before this one (the routing): the first planes are made while that ends.
    const bool early = inv_perm != nullptr;
    if (early && first < total) split(first);
    pdl_wait();
    pdl_launch_dependents();
    read_segments<R>(s, offsets, E, T * (k + S), most, status);
    for (long long i = first; i < total; i += (long long)gridDim.x * 8) {
        const int t = (int)(i / nc), c = (int)(i - (long long)t * nc);
        if (!early || i != first) split(i);
        for (int j0 = 0; j0 < k + S; j0 += 32) {
            int place = -1;                                                  // tile * R + row of the tile, of this lane's copy
            const int j = j0 + lane;
            if (j < k + S) {
                const int row = j >= k ? T * k + (j - k) * T + t : inv_perm ? inv_perm[t * k + j] : t;
                if (row >= 0) {
                    int e = 0;
#pragma unroll
                    for (int step = 64; step > 0; step >>= 1)                // the last segment that starts at or before the row
                        if (s.start[e + step] <= row) e += step;
                    const int local = row - s.start[e];
                    if (local < s.rows[e]) place = (s.tile0[e] + local / R) * R + local % R;
                }
            }
            const int now = min(32, k + S - j0);
            for (int q = 0; q < now; ++q) {
                const int at = __shfl_sync(0xffffffffu, place, q);
                if (at < 0) continue;                                        // a dropped pair
                const int r = at % R;
                uint8_t* dst = tiles + ((size_t)(at / R) * nc + c) * Ts::kBytes;
                store_tile_row<R>(dst, r, lane, codes, scales);
            }
        }
    }
}

struct MoeArgs {
    const uint8_t* tiles;       // activations: tiles of x (MODE 0) or h (MODE 1)
    const int32_t* offsets;     // [E + 1], or nullptr: one segment [0, max_rows)
    int max_rows, E, d, f;
    int most;                   // tiles the workspace has room for
    const uint8_t* slot_region;
    size_t slot_bytes;
    uint8_t* h_tiles;           // MODE 0: output
    float* y;                   // MODE 1: output [max_rows, d]
    int* status;
};

template <int MODE, int R>
__global__ void __launch_bounds__(kMoeThreads, 1)
mx_ffn_kernel(const __grid_constant__ MoeArgs a, const __grid_constant__ SlotTable tab) {
    using T = TileShape<R>;
    using F = FfnShape<MODE, R>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Segments s;
    __shared__ alignas(8) uint64_t bar_full[F::kStages], bar_empty[F::kStages], bar_acc[2], bar_free[2];
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int K = MODE == 0 ? a.d : a.f, nc = mx_chunks(K), n_gb = (MODE == 0 ? a.f : a.d) / 128;
    volatile int* abort_p = &abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < F::kStages; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bar_acc[i]), 1);
            mbar_init(smem_u32(&bar_free[i]), F::kSets == 2 ? 4 : 8);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "n"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    // The launch before this one only writes activations; what it waited for itself (the offsets) is complete.  The segments
    // and the first weights are on their way while it ends.
    read_segments<R>(s, a.offsets, a.E, a.max_rows, a.most, a.status);
    tc_fence_after();
    if (MODE == 0 && blockIdx.x == 0)
        for (int e = threadIdx.x; e < a.E; e += kMoeThreads)
            if (s.rows[e] > 0 && tab.slot[e] < 0 && tab.in_subset[e]) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
    const uint32_t tmem = warp_uniform(tmem_s), tmem_sf = tmem + F::kSets * F::kAccCols;
    const int total = (int)warp_uniform(s.tile0[SAEM_MAX_EXPERTS]) * n_gb;

    // Items of an expert: its tiles fastest, so that a weight block is read from DRAM once.
    struct Item { int e, gb, tile, row0, rows; };
    auto item_at = [&](int i) {
        int e = 0;
#pragma unroll
        for (int step = 64; step > 0; step >>= 1)                              // the last e whose first item is not beyond i
            if (s.tile0[e + step] * n_gb <= i) e += step;
        e = (int)warp_uniform(e);
        const int tile0 = (int)warp_uniform(s.tile0[e]), tiles = (int)warp_uniform(s.tile0[e + 1]) - tile0, rem = i - tile0 * n_gb;
        const int gb = rem / tiles, t = rem - gb * tiles;
        return Item{e, gb, tile0 + t, s.start[e] + t * R, min(R, s.rows[e] - t * R)};
    };

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        const size_t region = MODE == 0 ? 0 : mx_gate_up_blocks(a.d, a.f);
        int it = 0, st = 0, turn = 0;
        bool ok = true;
        // Every stage's weights are requested `early` stages before its activations: all of the ring's before the wait for
        // the launch before, none ahead afterwards.
        struct Walk { int i, c; const uint8_t *w, *x; } ahead = {(int)blockIdx.x - (int)gridDim.x, nc, nullptr, nullptr}, now = ahead;
        auto step = [&](Walk& k) {                                             // to the next stage; false: there is none
            if (++k.c < nc) {
                k.w += F::kWBytes;
                k.x += T::kBytes;
                return true;
            }
            for (k.i += gridDim.x; k.i < total; k.i += gridDim.x) {
                const Item t = item_at(k.i);
                const int slot = (int)warp_uniform(tab.slot[t.e]);
                if (slot < 0) continue;
                k.c = 0;
                k.w = a.slot_region + (size_t)slot * a.slot_bytes + region * kMxBlockBytes + (size_t)t.gb * nc * F::kWBytes;
                k.x = a.tiles + (size_t)t.tile * nc * T::kBytes;
                return true;
            }
            return false;
        };
        auto weights = [&](const Walk& k, int place) {
            expect_tx_on(on, smem_u32(&bar_full[place]), F::kStageBytes);
            bulk_g2s_on(on, base + place * F::kStageBytes, k.w, F::kWBytes, smem_u32(&bar_full[place]));
        };
        int early = 0;
        while (early < F::kStages && step(ahead)) weights(ahead, early++);
        pdl_wait();
        pdl_launch_dependents();
        while (step(now)) {
            if (turn) {
                ok = mbar_wait_warp(smem_u32(&bar_empty[st]), (turn - 1) & 1, abort_p, a.status);
                if (!ok) break;
                weights(now, st);
            }
            bulk_g2s_on(on, base + st * F::kStageBytes + F::kWBytes, now.x, T::kBytes, smem_u32(&bar_full[st]));
            ++it;
            if (++st == F::kStages) { st = 0; ++turn; }
        }
        ring_settle_warp(bar_full, F::kStages, it, a.status);
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        const uint64_t codes0 = smem_desc_sw128(base), scales0 = smem_desc_scales(base);
        int st = 0, turn = 0, n = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            if ((int)warp_uniform(tab.slot[item_at(i).e]) < 0) continue;
            const int set = n % F::kSets;
            const uint32_t acc = tmem + set * F::kAccCols;
            if (n >= F::kSets) ok = mbar_wait_warp(smem_u32(&bar_free[set]), (n / F::kSets - 1) & 1, abort_p, a.status);
            tc_fence_after();
            for (int c = 0; c < nc && ok; ++c) {
                ok = mbar_wait_warp(smem_u32(&bar_full[st]), turn & 1, abort_p, a.status);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = st * F::kStageBytes;
                const uint64_t dw = desc_at(codes0, at), dx = desc_at(codes0, at + F::kWBytes), ds = desc_at(scales0, at);
                const uint32_t sf = tmem_sf + st * F::kSfCols, sfx = sf + (MODE == 0 ? 16 : 8);
                const int steps = min(4, (K - c * kMxChunk) / 64);             // K is a multiple of 128
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * h >= steps) break;
#pragma unroll
                    for (int m = 0; m < (MODE == 0 ? 2 : 1); ++m)
                        tc_cp_scales(on, sf + m * 8 + 4 * h, desc_at(ds, m * kMxBlockBytes + kMxBlockCodes + h * kMxPiece));
#pragma unroll
                    for (int q = 0; q < T::kPieces; ++q)
                        tc_cp_scales(on, sfx + 4 * (h * T::kPieces + q), desc_at(ds, F::kWBytes + T::kN * 128 + (q * 2 + h) * kMxPiece));
                }
#pragma unroll
                for (int m = 0; m < (MODE == 0 ? 2 : 1); ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps)
                            tc_mma_mxf4(on, acc + m * T::kN, desc_at(dw, m * kMxBlockBytes + 32 * j), desc_at(dx, 32 * j),
                                        idesc_mxf4(T::kN, (j & 1) * 2), sf + m * 8 + 4 * (j >> 1), sfx + 4 * (j >> 1) * T::kPieces, c > 0 || j > 0);
                tc_commit_on(on, smem_u32(&bar_empty[st]));
                if (++st == F::kStages) { st = 0; ++turn; }
            }
            tc_commit_on(on, smem_u32(&bar_acc[set]));
            ++n;
        }
        if (n) mbar_settle_warp(smem_u32(&bar_acc[(n - 1) % F::kSets]), ((n - 1) / F::kSets) & 1, a.status);
    } else if (warp >= 2) {
        // ---------------------------------------------------------------- epilogue
        // Two groups of four warps (one per quarter of the lanes): with two sets of accumulators each group has its own
        // set, i.e. every other item; with one set they share the rows of every item.
        const int quad = warp & 3, group = (warp - 2) >> 2;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        int n = 0;
        bool ok = true;
        pdl_wait();                                                            // nothing is written before older launches have ended
        for (int i = blockIdx.x; i < total; i += gridDim.x) {
            const Item t = item_at(i);
            if (tab.slot[t.e] < 0) continue;
            const int set = n % F::kSets, turn = n / F::kSets;
            ++n;
            if (F::kSets == 2 && set != group) continue;
            ok = ok && mbar_wait(smem_u32(&bar_acc[set]), turn & 1, abort_p, a.status);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            const uint32_t acc = tmem + set * F::kAccCols + lane_base;
            for (int r0 = F::kSets == 2 ? 0 : 8 * group; r0 < t.rows && ok; r0 += F::kSets == 2 ? 8 : 16) {
                float v[8];
                plane_sums<R>(acc + r0, v);
                if (MODE == 1) {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (r0 + q < t.rows) a.y[(size_t)(t.row0 + r0 + q) * a.d + t.gb * 128 + quad * 32 + lane] = v[q];
                } else {
                    float u[8];
                    plane_sums<R>(acc + T::kN + r0, u);
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = swiglu(v[q], u[q]);
                    // the warp's 32 hidden units are one block of each row: chunk gb / 2 of the row, block (gb & 1) * 4 + quad
                    uint8_t* dst = a.h_tiles + ((size_t)t.tile * mx_chunks(a.f) + (t.gb >> 1)) * T::kBytes;
                    store_planes<R>(v, r0, t.rows, dst, (t.gb & 1) * 4 + quad, lane);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_free[set]));
        }
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512));
    }
}

// ------------------------------------------------------------------------------------------------------------- host
// Rows per tile, by the rows that a segment of a step of this many tokens has on average, times two (segments differ; per
// token k routed and always-on rows over E experts): 8 up to 8 rows, 16 up to 24, else 32, which is what tensor memory
// holds.  (64 tokens of a 2048 x 768 layer of 128 experts, 8 rows in twice the average: 8-row tiles.)
static int tile_rows(int tokens, int k, int E) {
    const long long twice = 2LL * tokens * k / E;
    return tokens <= 8 || twice <= 8 ? 8 : tokens <= 16 || twice <= 24 ? 16 : 32;
}
static long long most_tiles(long long rows, int experts, int R) { return (rows < experts ? rows : experts) + rows / R; }
static size_t tile_bytes(int R) { return R == 8 ? TileShape<8>::kBytes : R == 16 ? TileShape<16>::kBytes : TileShape<32>::kBytes; }

// A step of fewer tokens than the context was made for may take smaller tiles: the largest of the three, each with the most
// tokens that take it.  (The form for up to 8 tokens needs no more than 8-row tiles.)
size_t mx_workspace_bytes(int max_tokens, int k, int E, int S, int d, int f) {
    const int per = k + S, all = E + S;
    size_t most = 0;
    for (int R = 8; R <= 32; R *= 2) {
        long long tokens = max_tokens;
        if (R < 32) {
            const long long twice = R == 8 ? 9 : 25, few = R == 8 ? 8 : 16;    // twice * all - 1 rows still round down to the limit
            const long long fit = (twice * all - 1) / (2 * per);
            tokens = fit > few ? fit : few;
            if (tokens > max_tokens) tokens = max_tokens;
        }
        const size_t b = (size_t)most_tiles(tokens * per, all, R) * tile_bytes(R) * (mx_chunks(d) + mx_chunks(f));
        if (b > most) most = b;
    }
    return most;
}

template <int R>
static cudaError_t launch_tiles(const FfnArgs& f, const MxTokens& x, const SlotTable& tab, cudaStream_t st) {
    static DeviceOnce once;
    using A = FfnShape<0, R>;
    using B = FfnShape<1, R>;
    cudaError_t e = once_on_device(once, [] {
        const cudaError_t s = cudaFuncSetAttribute(mx_ffn_kernel<0, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, A::kSmem);
        return s != cudaSuccess ? s : cudaFuncSetAttribute(mx_ffn_kernel<1, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, B::kSmem);
    });
    if (e != cudaSuccess) return e;
    uint8_t* x_tiles = reinterpret_cast<uint8_t*>(f.h);
    const int most = (int)most_tiles(f.max_rows, f.E, R);
    uint8_t* h_tiles = x_tiles + (size_t)most * mx_chunks(f.d) * TileShape<R>::kBytes;
    MoeArgs a = {};
    a.tiles = x_tiles; a.offsets = f.offsets; a.max_rows = f.max_rows; a.E = f.E; a.d = f.d; a.f = f.f; a.most = most;
    a.slot_region = f.slot_region; a.slot_bytes = f.slot_bytes; a.h_tiles = h_tiles; a.y = f.y_packed; a.status = f.status;
    const int T = x.inv_perm ? x.T : f.max_rows, k = x.inv_perm ? x.k : 1, S = x.inv_perm ? x.S : 0;
    const long long tasks = (long long)T * mx_chunks(f.d), ctas = (tasks + 7) / 8, wave = (long long)f.n_sm * 8;
    e = launch_pdl(mx_tile_kernel<R>, dim3((unsigned)(ctas < wave ? ctas : wave)), dim3(256), 0, st, f.x_packed, x.inv_perm, f.offsets, T, k, S,
                   f.E, f.d, most, x_tiles, f.status);
    if (e != cudaSuccess) return e;
    e = launch_pdl(mx_ffn_kernel<0, R>, dim3((unsigned)f.n_sm), dim3(kMoeThreads), (size_t)A::kSmem, st, a, tab);
    if (e != cudaSuccess) return e;
    a.tiles = h_tiles;
    return launch_pdl(mx_ffn_kernel<1, R>, dim3((unsigned)f.n_sm), dim3(kMoeThreads), (size_t)B::kSmem, st, a, tab);
}

cudaError_t launch_mx_ffn(const FfnArgs& f, const MxTokens& x, const SlotTable& tab, cudaStream_t st, int* n_launch) {
    const int R = tile_rows(f.tokens, f.per_token, f.E);
    const cudaError_t e = R == 8 ? launch_tiles<8>(f, x, tab, st) : R == 16 ? launch_tiles<16>(f, x, tab, st) : launch_tiles<32>(f, x, tab, st);
    if (e == cudaSuccess) *n_launch += 3;
    return e;
}

}  // namespace saem
