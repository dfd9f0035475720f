// Product of two MXFP4 matrices on the block-scaled tensor cores: out[m, n] = sum_k A[m, k] W[n, k].
//
// tcgen05.mma kind::mxf4 multiplies E2M1 operands out of shared memory, takes the scale of every 32 elements from
// tensor memory and accumulates in fp32 (an E2M1 product times a power of two is exact; the sum's rounding is the only
// one before the output's).  The weights' rows are the MMA's M (128 lanes of tensor memory), the tokens its N (16..256
// columns), so that one instruction shape serves one token and thousands, and a warp's stores of the result are
// consecutive n.  A stage is 256 elements of k: 128-byte rows of codes under the 128-byte swizzle (TMA) and the scales'
// 512-byte pieces (plain bulk copies, moved to tensor memory by tcgen05.cp as they are).
//
// Three forms, by the number of tokens and tiles (measured side by side for n 1024 .. 14336 and k 1024 .. 4096; the product
// alone unless it says otherwise).
//   few tiles         mx_matmul_kernel, one CTA per tile of 128 x 64 (or fewer tokens), up to 64 tokens always and beyond while
//                     all tiles are under way at once, two per SM (333 tokens of 2563 x 1500: 5.5 us against 10.8 us in tiles
//                     of 256 tokens; 512 of 4096 x 4096 9.8 us against 10.8 us).  The weights' bytes and the latency of one tile
//                     are the bound, so the k range is split over a cluster of 2 or 4 CTAs while there are SMs for them;
//                     their sums meet in distributed shared memory in a fixed order (16 tokens of 4096 x 4096: 5.3 us
//                     in four parts, 9 us in one; parts of fewer than four stages, or eight parts, cost more than they
//                     give).  Up to 8 tokens the CTA quantises its part of the activations itself, if the parts fit into
//                     the ring (16 tokens of 14336 x 4096 that way: 24 us against 9.7 us, quantisation launch included).
//   more              mx_matmul_tiles_kernel, tiles of 128 x 256, a CTA each.
//   many tiles        mx_matmul_pair_kernel, persistent CTA pairs (cta_group::2) with tiles of 256 x 256 and the epilogue beside
//                     the next tile's products, when these are at least half as many as the SMs: each operand crosses shared
//                     memory half as often (8192 tokens of 14336 x 4096, quantisation included: 205 us, 4.7 PFLOP/s, in a
//                     burst at 1965 MHz, 239 us in seconds of it, at 1.44 to 1.5 GHz under the power cap; persistent tiles
//                     of 128 x 256 took 255 us).
// Two runs give the same bits.
#include "mx_tc.cuh"

namespace saem {

constexpr int kMmThreads = 320;             // warp 0: copies, warp 1: MMA issue, warps 2-9: quantisation, epilogue
constexpr int kMmStageK = 256;              // elements of k per stage (128 bytes of codes)
constexpr int kMmMaxStages = 12;
constexpr int kMmSmem = 226 * 1024;         // dynamic shared memory at most
constexpr int kMmSfCols = 16;               // tensor-memory columns of a stage's scales: 8 for W, 8 for A

__device__ int mx_status_sink;              // where a run-out wait is noted when the caller gave no status word

struct MmArgs {
    const uint8_t* a_scales;
    const uint8_t* w_scales;
    void* out;
    int* status;
    long long out_stride;
    int m, n, k;
    int n_tile;                             // tokens of a tile: all, rounded up to 16, or 64 (256 in the other two kernels)
    int n_stage;                            // stages of the ring
    int stage_bytes;
    int tmem_cols;
    int split;                              // CTAs of the cluster
    int out_bf16;
    int w_early;                            // the launch before this one wrote only A: W may be read before it is complete
    const void* x;                          // quantise A from here (every stage of the CTA has its place in the ring), or nullptr
    long long x_stride;
    int x_bf16, x_vec;
    int out_pairs;                          // bf16 output whose rows begin at 4-byte addresses, n even
};

__global__ void __launch_bounds__(kMmThreads, 1)
mx_matmul_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a,
                 const __grid_constant__ MmArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bar_full[kMmMaxStages], bar_empty[kMmMaxStages], bar_acc;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
    const int n0 = blockIdx.y * 128, t0 = blockIdx.z * p.n_tile, tokens = min(p.n_tile, p.m - t0), n_mma = p.n_tile;
    const long long kp = (p.k + kMxBlock - 1) / kMxBlock * kMxBlock;        // padded with zeros to whole blocks
    const int n_span = (p.k + kMxSpan - 1) / kMxSpan;
    const int all = (int)((kp + kMmStageK - 1) / kMmStageK);
    const int s0 = (int)((long long)all * rank / p.split), s1 = (int)((long long)all * (rank + 1) / p.split);
    int* const status = p.status ? p.status : &mx_status_sink;
    volatile int* abort_p = &abort_flag;

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.n_stage; ++i) {
            mbar_init(smem_u32(&bar_full[i]), p.x ? 9 : 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        mbar_init(smem_u32(&bar_acc), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(p.tmem_cols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_uniform(tmem_s);
    const int acc_cols = (p.n_tile + 31) & ~31;
    const uint32_t tmem_sf = tmem + acc_cols;
    const int w_bytes = 128 * 128, a_bytes = p.n_tile * 128;

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        auto w_part = [&](int s, int i) {
            const uint32_t st = base + i * p.stage_bytes, bar = smem_u32(&bar_full[i]);
            const int spans = min(2, n_span - 2 * s);
            expect_tx_on(on, bar, w_bytes + spans * kMxPiece + (p.x ? 0 : a_bytes + spans * kMxPiece));
            tma_2d_on(on, st, &map_w, s * 128, n0, bar);
            bulk_g2s_on(on, st + w_bytes + a_bytes, p.w_scales + ((size_t)blockIdx.y * n_span + 2 * s) * kMxPiece, spans * kMxPiece, bar);
        };
        auto a_part = [&](int s, int i) {
            const uint32_t st = base + i * p.stage_bytes, bar = smem_u32(&bar_full[i]);
            const int spans = min(2, n_span - 2 * s);
            if (p.x) return;
            tma_2d_on(on, st + w_bytes, &map_a, s * 128, t0, bar);
            bulk_g2s_on(on, st + w_bytes + a_bytes + 2 * kMxPiece, p.a_scales + ((size_t)(t0 / 128) * n_span + 2 * s) * kMxPiece, spans * kMxPiece, bar);
        };
        const int early = p.w_early ? min(p.n_stage, s1 - s0) : 0;
        for (int i = 0; i < early; ++i) w_part(s0 + i, i);
        pdl_wait();
        pdl_launch_dependents();
        int s = s0, st = 0, turn = 0;
        bool ok = true;
        for (; s < s1; ++s) {
            if (turn) {
                ok = mbar_wait_warp(smem_u32(&bar_empty[st]), (turn - 1) & 1, abort_p, status);
                if (!ok) break;
            }
            if (s - s0 >= early) w_part(s, st);
            a_part(s, st);
            if (++st == p.n_stage) { st = 0; ++turn; }
        }
        ring_settle_warp(bar_full, p.n_stage, s - s0, status);
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        const uint64_t codes0 = smem_desc_sw128(base), scales0 = smem_desc_scales(base);
        const int half = t0 % 128 / 32;                                      // the second half of a piece: two columns on
        int st = 0, turn = 0;
        for (int s = s0; s < s1; ++s) {
            if (!mbar_wait_warp(smem_u32(&bar_full[st]), turn & 1, abort_p, status)) break;
            tc_fence_after();
            const uint32_t at = st * p.stage_bytes, tw = tmem_sf + st * kMmSfCols, ta = tw + 8;
            const uint64_t dw = desc_at(codes0, at), da = desc_at(codes0, at + w_bytes), ds = desc_at(scales0, at + w_bytes + a_bytes);
            const int spans = min(2, n_span - 2 * s), steps = (int)min(4ll, (kp - (long long)s * kMmStageK + 63) / 64);
            for (int h = 0; h < spans; ++h) {
                tc_cp_scales(on, tw + 4 * h, desc_at(ds, h * kMxPiece));
                tc_cp_scales(on, ta + 4 * h, desc_at(ds, (2 + h) * kMxPiece));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < steps)
                    tc_mma_mxf4(on, tmem, desc_at(dw, 32 * j), desc_at(da, 32 * j), idesc_mxf4(n_mma, (j & 1) * 2), tw + 4 * (j >> 1),
                                ta + 4 * (j >> 1) + half, s > s0 || j > 0);
            tc_commit_on(on, smem_u32(&bar_empty[st]));
            if (++st == p.n_stage) { st = 0; ++turn; }
        }
        tc_commit_on(on, smem_u32(&bar_acc));
        mbar_settle_warp(smem_u32(&bar_acc), 0, status);
    } else if (p.x) {
        // ---------------------------------------------------------------- quantisation of the CTA's part of A
        // (stage, row) pairs go to the eight warps in turn, so that a few tokens' loads are under way together as well
        pdl_wait();
        uint8_t* const smem = smem_raw + (base - smem_u32(smem_raw));
        const size_t esize = p.x_bf16 ? 2 : 4;
        for (int i = 0; i < s1 - s0; ++i) {
            const int r = (warp - 2 - i * p.m) & 7;                          // p.m <= 8: a row at most
            if (r < p.m) {
                uint8_t* st = smem + (size_t)i * p.stage_bytes + w_bytes;
                const long long col = (long long)(s0 + i) * kMmStageK + lane * 8;
                const void* row = static_cast<const uint8_t*>(p.x) + (size_t)r * p.x_stride * esize;
                float v[8];
                if (p.x_bf16) { if (p.x_vec) load8<true, true>(row, col, p.k, v); else load8<true, false>(row, col, p.k, v); }
                else { if (p.x_vec) load8<false, true>(row, col, p.k, v); else load8<false, false>(row, col, p.k, v); }
                int scale;
                const uint32_t w = mx_quantize8(v, scale);
                uint32_t word = (uint32_t)(col < kp ? scale : 0) << (((lane >> 2) & 3) * 8);
                word |= __shfl_xor_sync(0xffffffffu, word, 4);
                word |= __shfl_xor_sync(0xffffffffu, word, 8);
                *reinterpret_cast<uint32_t*>(st + r * 128 + (((lane >> 2) ^ r) << 4) + (lane & 3) * 4) = w;
                if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(st + a_bytes + 2 * kMxPiece + (lane >> 4) * kMxPiece + r * 16) = word;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_full[i]));
        }
    }
    __syncwarp();

    // -------------------------------------------------------------------- epilogue
    const int quad = warp & 3, group = (warp - 2) >> 2, row = quad * 32 + lane;   // two groups share the columns
    const bool store_row = n0 + row < p.n;
    auto put = [&](int c, float v) {
        const size_t at = (size_t)(t0 + c) * p.out_stride + n0 + row;
        if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(p.out)[at] = v;
    };
    const int pitch = n_mma + 4;                                             // floats between rows of partial sums: no bank twice
    bool done = false;
    if (warp >= 2) {
        done = mbar_wait_warp(smem_u32(&bar_acc), 0, abort_p, status) && !*abort_p;
        tc_fence_after();
        pdl_wait();                                                          // nothing is written before older kernels have ended
        if (done)
            for (int c = 16 * group; c < n_mma; c += 32) {
                float v[16];
                tc_ld16(tmem + ((uint32_t)(quad * 32) << 16) + c, v);
                if (p.split > 1) {
                    // partial sums [row][column] where the stages were: every MMA has read them
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        st_shared_v4(base + (row * pitch + c + i) * 4, __float_as_uint(v[i]), __float_as_uint(v[i + 1]),
                                     __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3]));
                } else if (store_row) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < tokens) put(c + i, v[i]);
                }
            }
        tc_fence_before();
    }
    if (p.split > 1) {
        __syncthreads();
        cluster_sync_all();
        if (warp >= 2 && done)
            for (int c = (rank * 2 + group) * 4; c < tokens; c += 8 * p.split) {   // four columns at a time, the parts in order
                float4 v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (q < p.split)
                        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                     : "=f"(v[q].x), "=f"(v[q].y), "=f"(v[q].z), "=f"(v[q].w)
                                     : "r"(mapa_u32(base + (row * pitch + c) * 4, q)));
                float4 sum = v[0];
#pragma unroll
                for (int q = 1; q < 4; ++q)
                    if (q < p.split) { sum.x += v[q].x; sum.y += v[q].y; sum.z += v[q].z; sum.w += v[q].w; }
                const float f[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (store_row && c + i < tokens) put(c + i, f[i]);
            }
        __syncwarp();
        cluster_sync_all();                                                  // no CTA ends while another reads its shared memory
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols));
    }
}

// Tiles of 128 weight rows x 256 tokens, a CTA each: every SM has one at most, since the pair kernel takes over before there
// are as many as SMs (mm_plan).  Eight warps take the accumulators into registers, 128 columns each, and store them.
constexpr int kBigThreads = 320;            // warp 0: copies, warp 1: MMA issue, warps 2-9: epilogue
constexpr int kBigTile = 256;
constexpr int kBigStages = 4;
constexpr int kBigStageBytes = 128 * 128 + kBigTile * 128 + 6 * kMxPiece;
constexpr int kBigSmem = kBigStages * kBigStageBytes + 1024;
constexpr int kBigSfCols = 24;

// 128 tokens' sums of the output column n that this lane owns.  bf16 in pairs of columns where the output's rows allow it:
// even lanes take over the pair for even tokens, odd ones for odd tokens.
__device__ __forceinline__ void store_columns(const MmArgs& p, const uint32_t (&r)[128], int n, int t0, int lane) {
    const int tokens = min(128, p.m - t0);
    if (!p.out_bf16) {
        float* o = static_cast<float*>(p.out) + (size_t)t0 * p.out_stride + n;
        if (n < p.n)
#pragma unroll
            for (int c = 0; c < 128; ++c)
                if (c < tokens) o[c * p.out_stride] = __uint_as_float(r[c]);
    } else if (p.out_pairs) {
        const int odd = lane & 1;
        uint16_t* o = static_cast<uint16_t*>(p.out) + (size_t)(t0 + odd) * p.out_stride + (n & ~1);
#pragma unroll
        for (int c = 0; c < 128; c += 2) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? r[c] : r[c + 1], 1);
            const __nv_bfloat162 v = odd ? __floats2bfloat162_rn(__uint_as_float(other), __uint_as_float(r[c + 1]))
                                         : __floats2bfloat162_rn(__uint_as_float(r[c]), __uint_as_float(other));
            if (n < p.n && c + odd < tokens) *reinterpret_cast<__nv_bfloat162*>(o + c * p.out_stride) = v;
        }
    } else {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.out) + (size_t)t0 * p.out_stride + n;
        if (n < p.n)
#pragma unroll
            for (int c = 0; c < 128; ++c)
                if (c < tokens) o[c * p.out_stride] = __float2bfloat16_rn(__uint_as_float(r[c]));
    }
}

__global__ void __launch_bounds__(kBigThreads, 1)
mx_matmul_tiles_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ MmArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bar_full[kBigStages], bar_empty[kBigStages], bar_acc;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int n_w = (p.n + 127) / 128, tt = blockIdx.x / n_w, tw = blockIdx.x - tt * n_w;
    const long long kp = (p.k + kMxBlock - 1) / kMxBlock * kMxBlock;
    const int n_span = (p.k + kMxSpan - 1) / kMxSpan, stages = (int)((kp + kMmStageK - 1) / kMmStageK);
    int* const status = p.status ? p.status : &mx_status_sink;
    volatile int* abort_p = &abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kBigStages; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        mbar_init(smem_u32(&bar_acc), 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "n"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    pdl_wait();
    pdl_launch_dependents();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_uniform(tmem_s), tmem_sf = tmem + kBigTile;
    constexpr int w_bytes = 128 * 128, a_bytes = kBigTile * 128;

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        const int pieces = min(2, (p.m - tt * kBigTile + 127) / 128);
        int s = 0, st = 0, turn = 0;
        bool ok = true;
        for (; s < stages; ++s) {
            if (turn) {
                ok = mbar_wait_warp(smem_u32(&bar_empty[st]), (turn - 1) & 1, abort_p, status);
                if (!ok) break;
            }
            const uint32_t dst = base + st * kBigStageBytes, bar = smem_u32(&bar_full[st]);
            const int bytes = min(2, n_span - 2 * s) * kMxPiece;
            expect_tx_on(on, bar, w_bytes + a_bytes + bytes * (1 + pieces));
            tma_2d_on(on, dst, &map_w, s * 128, tw * 128, bar);
            tma_2d_on(on, dst + w_bytes, &map_a, s * 128, tt * kBigTile, bar);
            bulk_g2s_on(on, dst + w_bytes + a_bytes, p.w_scales + ((size_t)tw * n_span + 2 * s) * kMxPiece, bytes, bar);
            for (int q = 0; q < pieces; ++q)
                bulk_g2s_on(on, dst + w_bytes + a_bytes + (1 + q) * 2 * kMxPiece,
                            p.a_scales + ((size_t)(tt * 2 + q) * n_span + 2 * s) * kMxPiece, bytes, bar);
            if (++st == kBigStages) { st = 0; ++turn; }
        }
        ring_settle_warp(bar_full, kBigStages, s, status);
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        const uint64_t codes0 = smem_desc_sw128(base), scales0 = smem_desc_scales(base);
        const int n_mma = (min(kBigTile, p.m - tt * kBigTile) + 15) & ~15;
        int st = 0, turn = 0;
        for (int s = 0; s < stages; ++s) {
            if (!mbar_wait_warp(smem_u32(&bar_full[st]), turn & 1, abort_p, status)) break;
            tc_fence_after();
            const uint32_t at = st * kBigStageBytes, sw = tmem_sf + st * kBigSfCols, sa = sw + 8;
            const uint64_t dw = desc_at(codes0, at), da = desc_at(codes0, at + w_bytes), ds = desc_at(scales0, at + w_bytes + a_bytes);
            const int steps = (int)min(4ll, (kp - (long long)s * kMmStageK + 63) / 64);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (2 * s + h >= n_span) break;
                tc_cp_scales(on, sw + 4 * h, desc_at(ds, h * kMxPiece));
                tc_cp_scales(on, sa + 8 * h, desc_at(ds, (2 + h) * kMxPiece));
                tc_cp_scales(on, sa + 8 * h + 4, desc_at(ds, (4 + h) * kMxPiece));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < steps)
                    tc_mma_mxf4(on, tmem, desc_at(dw, 32 * j), desc_at(da, 32 * j), idesc_mxf4(n_mma, (j & 1) * 2), sw + 4 * (j >> 1),
                                sa + 8 * (j >> 1), s > 0 || j > 0);
            tc_commit_on(on, smem_u32(&bar_empty[st]));
            if (++st == kBigStages) { st = 0; ++turn; }
        }
        tc_commit_on(on, smem_u32(&bar_acc));
        mbar_settle_warp(smem_u32(&bar_acc), 0, status);
    } else {
        // ---------------------------------------------------------------- epilogue
        const int quad = warp & 3, half = (warp - 2) >> 2, row = quad * 32 + lane;
        const bool ok = mbar_wait_warp(smem_u32(&bar_acc), 0, abort_p, status) && !*abort_p;
        tc_fence_after();
        if (ok) {
            uint32_t r[128];
#pragma unroll
            for (int q = 0; q < 4; ++q) tc_ld32_issue(tmem + ((uint32_t)(quad * 32) << 16) + half * 128 + q * 32, r + 32 * q);
            tc_wait_ld();
#pragma unroll
            for (int q = 0; q < 8; ++q) tc_reg_fence16(r + 16 * q);
            store_columns(p, r, tw * 128 + row, tt * kBigTile + half * 128, lane);
        }
        tc_fence_before();
    }
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512));
    }
}

// The same with pairs of CTAs: 256 weight rows x 256 tokens.  One CTA alone has to bring 48 KB of codes into shared memory
// and feed the MMA 48 KB out of it for every 512 cycles of MMAs, more than its 128 bytes per cycle; in a pair each CTA
// loads its own 128 weight rows but half of the tokens, whose other half the hardware reads from the partner.  The
// leader's barriers count both CTAs' copies (all of them tiled, the scales too: an untiled bulk copy cannot signal another
// CTA's barrier) and one commit frees a stage, or hands over the accumulators, in both.
constexpr int kPairStages = 6;
constexpr int kPairStageBytes = 2 * 128 * 128 + 6 * kMxPiece;
constexpr int kPairSmem = kPairStages * kPairStageBytes + 1024;

__global__ void __launch_bounds__(kBigThreads, 1)
mx_matmul_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a,
                      const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_as, const __grid_constant__ MmArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bar_full[kPairStages], bar_empty[kPairStages], bar_acc, bar_free;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int n_w = (p.n + 255) / 256, n_t = (p.m + kBigTile - 1) / kBigTile, total = n_w * n_t;
    const long long kp = (p.k + kMxBlock - 1) / kMxBlock * kMxBlock;
    const int n_span = (p.k + kMxSpan - 1) / kMxSpan, stages = (int)((kp + kMmStageK - 1) / kMmStageK);
    int* const status = p.status ? p.status : &mx_status_sink;
    volatile int* abort_p = &abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairStages; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        mbar_init(smem_u32(&bar_acc), 1);
        mbar_init(smem_u32(&bar_free), 16);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "n"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster_sync_all();                                                        // both CTAs' barriers exist
    tc_fence_after();
    pdl_wait();
    pdl_launch_dependents();
    const uint32_t tmem = warp_uniform(tmem_s), tmem_sf = tmem + kBigTile;
    constexpr int half_bytes = 128 * 128, scales_at = 2 * half_bytes;

    if (warp == 0) {
        // ---------------------------------------------------------------- copies (both CTAs)
        const uint32_t on = elect_one();
        int it = 0, st = 0, turn = 0;
        bool ok = true;
        for (int i = pair; i < total && ok; i += pairs) {
            const int tt = i / n_w, tw = (i - tt * n_w) * 2 + rank;
            for (int s = 0; s < stages; ++s, ++it) {
                if (turn) {
                    ok = mbar_wait_warp(smem_u32(&bar_empty[st]), (turn - 1) & 1, abort_p, status);
                    if (!ok) break;
                }
                const uint32_t dst = base + st * kPairStageBytes, full = mapa_u32(smem_u32(&bar_full[st]), 0);
                // the leader alone arms its barrier, for both; the partner's copies may complete on it first
                if (rank == 0) expect_tx_on(on, smem_u32(&bar_full[st]), 2 * kPairStageBytes);
                tma_2d_pair_on(on, dst, &map_w, s * 128, tw * 128, full);
                tma_2d_pair_on(on, dst + half_bytes, &map_a, s * 128, tt * kBigTile + rank * 128, full);
                tma_2d_pair_on(on, dst + scales_at, &map_ws, 0, tw * n_span + 2 * s, full);
                tma_2d_pair_on(on, dst + scales_at + 2 * kMxPiece, &map_as, 0, 2 * tt * n_span + 2 * s, full);
                tma_2d_pair_on(on, dst + scales_at + 4 * kMxPiece, &map_as, 0, (2 * tt + 1) * n_span + 2 * s, full);
                if (++st == kPairStages) { st = 0; ++turn; }
            }
        }
        // The leader's barriers count both CTAs' copies, and the partner waits for the leader below.  Where one CTA gave up and
        // the other did not, their last stages differ, and a barrier may count too little to wait for: then by the clock, a
        // hundred times what a copy takes.
        if (!ok) {
            const unsigned long long t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 200000ull) {}
        } else if (rank == 0) {
            for (int q = max(0, it - kPairStages); q < it; ++q) {
                int never = 0;
                if (!__all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_full[q % kPairStages]), (q / kPairStages) & 1, &never, status))) break;
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            // ------------------------------------------------------------ MMA issue (leader)
            const uint32_t on = elect_one();
            const uint64_t codes0 = smem_desc_sw128(base), scales0 = smem_desc_scales(base + scales_at);
            int st = 0, turn = 0, k = 0;
            bool ok = true;
            for (int i = pair; i < total && ok; i += pairs, ++k) {
                if (k) ok = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_free), (k - 1) & 1, abort_p, status));
                tc_fence_after();
                for (int s = 0; s < stages && ok; ++s) {
                    ok = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_full[st]), turn & 1, abort_p, status));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t at = st * kPairStageBytes, tw = tmem_sf + st * kBigSfCols, ta = tw + 8;
                    const uint64_t dw = desc_at(codes0, at), da = desc_at(codes0, at + half_bytes), ds = desc_at(scales0, at);
                    const int steps = (int)min(4ll, (kp - (long long)s * kMmStageK + 63) / 64);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (2 * s + h >= n_span) break;
                        tc_cp_scales_pair(on, tw + 4 * h, desc_at(ds, h * kMxPiece));
                        tc_cp_scales_pair(on, ta + 8 * h, desc_at(ds, (2 + h) * kMxPiece));
                        tc_cp_scales_pair(on, ta + 8 * h + 4, desc_at(ds, (4 + h) * kMxPiece));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps)
                            tc_mma_mxf4_pair(on, tmem, desc_at(dw, 32 * j), desc_at(da, 32 * j), idesc_mxf4_pair(kBigTile, (j & 1) * 2),
                                             tw + 4 * (j >> 1), ta + 8 * (j >> 1), s > 0 || j > 0);
                    tc_commit_pair_on(on, smem_u32(&bar_empty[st]));
                    if (++st == kPairStages) { st = 0; ++turn; }
                }
                tc_commit_pair_on(on, smem_u32(&bar_acc));
            }
            if (k) mbar_settle_warp(smem_u32(&bar_acc), (k - 1) & 1, status);
        }
    } else {
        // ---------------------------------------------------------------- epilogue (both CTAs)
        const int quad = warp & 3, half = (warp - 2) >> 2, row = quad * 32 + lane;
        bool ok = true;
        int k = 0;
        for (int i = pair; i < total && ok; i += pairs, ++k) {
            const int tt = i / n_w, tw = (i - tt * n_w) * 2 + rank;
            ok = mbar_wait_warp(smem_u32(&bar_acc), k & 1, abort_p, status);
            tc_fence_after();
            uint32_t r[128];
            if (ok) {
#pragma unroll
                for (int q = 0; q < 4; ++q) tc_ld32_issue(tmem + ((uint32_t)(quad * 32) << 16) + half * 128 + q * 32, r + 32 * q);
                tc_wait_ld();
#pragma unroll
                for (int q = 0; q < 8; ++q) tc_reg_fence16(r + 16 * q);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_u32(smem_u32(&bar_free), 0));
            if (ok) store_columns(p, r, tw * 128 + row, tt * kBigTile + half * 128, lane);
        }
    }
    // neither CTA leaves, or frees tensor memory, while the other may still touch it
    __syncwarp();
    tc_fence_before();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512));
    }
}

// ------------------------------------------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static std::atomic<EncodeTiledFn> g_mx_encode{nullptr};
static DeviceOnce g_mx_once;

static cudaError_t mx_matmul_init() {
    return once_on_device(g_mx_once, [] {
        cudaError_t e;
        if (!g_mx_encode) {
            void* fn = nullptr;
            cudaDriverEntryPointQueryResult q;
            e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
            if (e != cudaSuccess) return e;
            if (!fn || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
            g_mx_encode = (EncodeTiledFn)fn;
        }
        e = cudaFuncSetAttribute(mx_matmul_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmSmem);
        if (e != cudaSuccess) return e;
        e = cudaFuncSetAttribute(mx_matmul_tiles_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBigSmem);
        return e != cudaSuccess ? e : cudaFuncSetAttribute(mx_matmul_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
    });
}

// Codes as a byte matrix: boxes of 128 bytes (256 elements) x `box_rows` rows; what lies outside reads as zero.
static bool make_code_map(CUtensorMap* m, const void* codes, long long rows, long long cols, int box_rows) {
    const cuuint64_t pitch = (cuuint64_t)((cols + kMxBlock - 1) / kMxBlock) * 16;
    const cuuint64_t dims[2] = {pitch, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return g_mx_encode.load(std::memory_order_relaxed)(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, estr,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product is cut: decided from its sizes alone, so that saem_mx_linear knows whether A is to be quantised first.
struct MmPlan {
    bool big;                               // mx_matmul_tiles_kernel: fewer tiles of 128 x 256 than SMs
    bool pairs;                             // mx_matmul_pair_kernel
    bool fused;                             // A quantised by the product's CTAs (where it is not quantised already)
    int n_tile, split, n_stage, stage_bytes;
};
static MmPlan mm_plan(int m, int n, int k, int n_sm) {
    MmPlan p = {};
    const long long rows = (n + 127) / 128;
    const int stages = (k + kMmStageK - 1) / kMmStageK;
    // every pair of SMs has a tile of 256 x 256 at least
    p.pairs = m > 64 && (long long)((n + 255) / 256) * ((m + 255) / 256) >= n_sm / 2;
    // 64 tokens at a time while all tiles are under way at once
    p.big = p.pairs || (m > 64 && rows * ((m + 63) / 64) > 2 * n_sm);
    if (p.big) return p;
    p.n_tile = m <= 64 ? round_up(m, 16) : 64;
    const int tiles = (int)rows * ((m + p.n_tile - 1) / p.n_tile);
    p.stage_bytes = 128 * 128 + p.n_tile * 128 + 4 * kMxPiece;
    p.split = 1;
    while (p.split < 4 && tiles * p.split * 2 <= n_sm && stages >= 8 * p.split) p.split *= 2;
    const int mine = (stages + p.split - 1) / p.split;
    p.n_stage = (kMmSmem / 2 - 2048) / p.stage_bytes;                          // two CTAs per SM
    if (m <= 8 && mine <= kMmMaxStages && mine * p.stage_bytes + 1024 <= kMmSmem) {
        p.fused = true;                                                        // a place in the ring for every stage of the CTA
        p.n_stage = mine;
    }
    if (p.n_stage > mine) p.n_stage = mine;
    return p;
}

// Scales as rows of 512 bytes: two pieces of a row tile, which follow each other along k.
static bool make_scale_map(CUtensorMap* m, const void* scales, long long rows, long long cols) {
    const cuuint64_t dims[2] = {128, (cuuint64_t)((rows + 127) / 128 * ((cols + kMxSpan - 1) / kMxSpan))};
    const cuuint64_t strides[1] = {kMxPiece};
    const cuuint32_t box[2] = {128, 2};
    const cuuint32_t estr[2] = {1, 1};
    return g_mx_encode.load(std::memory_order_relaxed)(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(scales), dims, strides, box, estr,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static cudaError_t launch_mx_matmul(const MmPlan& plan, MmArgs p, const uint8_t* a_codes, const uint8_t* w_codes, int n_sm, cudaStream_t st) {
    alignas(64) CUtensorMap map_w, map_a;
    const int n_tile = plan.big ? kBigTile : plan.n_tile;
    if (!make_code_map(&map_w, w_codes, p.n, p.k, 128)) return cudaErrorInvalidValue;
    if (a_codes ? !make_code_map(&map_a, a_codes, p.m, p.k, n_tile) : (map_a = map_w, false)) return cudaErrorInvalidValue;
    p.n_tile = n_tile;
    p.out_pairs = p.out_bf16 && p.n % 2 == 0 && ((uintptr_t)p.out & 3) == 0 && (p.out_stride % 2 == 0 || p.m == 1);
    if (plan.pairs) {
        alignas(64) CUtensorMap map_ws, map_as;
        if (!make_code_map(&map_a, a_codes, p.m, p.k, 128) || !make_scale_map(&map_ws, p.w_scales, p.n, p.k) ||
            !make_scale_map(&map_as, p.a_scales, p.m, p.k))
            return cudaErrorInvalidValue;
        return launch_pdl_pairs(mx_matmul_pair_kernel, dim3((unsigned)(n_sm & ~1)), dim3(kBigThreads), (size_t)kPairSmem, st, map_w, map_a, map_ws,
                                map_as, p);
    }
    if (plan.big)
        return launch_pdl(mx_matmul_tiles_kernel, dim3((unsigned)(((p.n + 127) / 128) * ((p.m + kBigTile - 1) / kBigTile))), dim3(kBigThreads),
                          (size_t)kBigSmem, st, map_w, map_a, p);
    p.stage_bytes = plan.stage_bytes;
    p.n_stage = plan.n_stage;
    p.split = plan.split;
    const int need = round_up(p.n_tile, 32) + p.n_stage * kMmSfCols;
    p.tmem_cols = 32;
    while (p.tmem_cols < need) p.tmem_cols *= 2;
    // partial sums take the place of the stages
    const int sums = 128 * (p.n_tile + 4) * 4, ring = p.n_stage * p.stage_bytes;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.split, (p.n + 127) / 128, (p.m + p.n_tile - 1) / p.n_tile);
    cfg.blockDim = dim3(kMmThreads);
    cfg.dynamicSmemBytes = 1024 + (p.split > 1 && sums > ring ? sums : ring);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, mx_matmul_kernel, map_w, map_a, p);
}

}  // namespace saem

using namespace saem;

static int check_product(int64_t m, int64_t n, int64_t k, int out_dtype, int64_t out_stride) {
    if (out_dtype != SAEM_OUT_F32 && out_dtype != SAEM_OUT_BF16) return SAEM_ERR_INVALID_ARG;
    if (m < 0 || n < 1 || k < 1 || m > (1 << 23) || n > (1 << 22) || k > (1 << 24)) return SAEM_ERR_SHAPE;
    if (m > 1 && out_stride < n) return SAEM_ERR_SHAPE;
    return SAEM_OK;
}

extern "C" {

int saem_mx_matmul(const void* a_codes, const void* a_scales, int64_t m, const void* w_codes, const void* w_scales,
                   int64_t n, int64_t k, void* out, int out_dtype, int64_t out_stride, int32_t* status, void* stream) {
    const int s = check_product(m, n, k, out_dtype, out_stride);
    if (s != SAEM_OK) return s;
    if (m == 0) return SAEM_OK;
    if (!a_codes || !a_scales || !w_codes || !w_scales || !out) return SAEM_ERR_INVALID_ARG;
    if (((uintptr_t)a_codes | (uintptr_t)a_scales | (uintptr_t)w_codes | (uintptr_t)w_scales) & 15) return SAEM_ERR_ALIGNMENT;
    if ((uintptr_t)out % (out_dtype == SAEM_OUT_BF16 ? 2 : 4) || ((uintptr_t)status & 3)) return SAEM_ERR_ALIGNMENT;
    int n_sm;
    if (mx_matmul_init() != cudaSuccess || sm_count(&n_sm) != cudaSuccess) return SAEM_ERR_CUDA;
    MmArgs p = {};
    p.a_scales = (const uint8_t*)a_scales; p.w_scales = (const uint8_t*)w_scales; p.out = out; p.status = status; p.out_stride = out_stride;
    p.m = (int)m; p.n = (int)n; p.k = (int)k; p.out_bf16 = out_dtype == SAEM_OUT_BF16;
    return launch_mx_matmul(mm_plan(p.m, p.n, p.k, n_sm), p, (const uint8_t*)a_codes, (const uint8_t*)w_codes, n_sm, (cudaStream_t)stream) ==
                   cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}

size_t saem_mx_linear_workspace_bytes(int64_t max_rows, int64_t k) {
    const size_t c = saem_mx_codes_bytes(max_rows, k);
    if (!c) return 0;
    return 256 + (c + 255) / 256 * 256 + saem_mx_scales_bytes(max_rows, k);
}

int saem_mx_linear(const void* x, int x_dtype, int64_t m, int64_t x_stride, const void* w_codes, const void* w_scales,
                   int64_t n, int64_t k, void* out, int out_dtype, int64_t out_stride, void* workspace,
                   size_t workspace_bytes, void* stream) {
    const int s = check_product(m, n, k, out_dtype, out_stride);
    if (s != SAEM_OK) return s;
    if (m == 0) return SAEM_OK;
    if (!x || !w_codes || !w_scales || !out || !workspace) return SAEM_ERR_INVALID_ARG;
    if (((uintptr_t)w_codes | (uintptr_t)w_scales) & 15 || (uintptr_t)workspace & 255) return SAEM_ERR_ALIGNMENT;
    if ((uintptr_t)out % (out_dtype == SAEM_OUT_BF16 ? 2 : 4)) return SAEM_ERR_ALIGNMENT;
    if (workspace_bytes < saem_mx_linear_workspace_bytes(m, k)) return SAEM_ERR_WORKSPACE;
    if (x_dtype != SAEM_OUT_F32 && x_dtype != SAEM_OUT_BF16) return SAEM_ERR_INVALID_ARG;
    if (m > 1 && x_stride < k) return SAEM_ERR_SHAPE;
    const size_t esize = x_dtype == SAEM_OUT_BF16 ? 2 : 4;
    if ((uintptr_t)x % esize) return SAEM_ERR_ALIGNMENT;
    int n_sm;
    if (mx_matmul_init() != cudaSuccess || sm_count(&n_sm) != cudaSuccess) return SAEM_ERR_CUDA;
    const MmPlan plan = mm_plan((int)m, (int)n, (int)k, n_sm);
    uint8_t* codes = (uint8_t*)workspace + 256;                              // the status word stands before them
    uint8_t* scales = codes + (saem_mx_codes_bytes(m, k) + 255) / 256 * 256;
    MmArgs p = {};
    p.a_scales = scales; p.w_scales = (const uint8_t*)w_scales; p.out = out; p.status = (int*)workspace; p.out_stride = out_stride;
    p.m = (int)m; p.n = (int)n; p.k = (int)k; p.out_bf16 = out_dtype == SAEM_OUT_BF16;
    if (plan.fused) {
        p.x = x;
        p.x_stride = x_stride;
        p.x_bf16 = x_dtype == SAEM_OUT_BF16;
        p.x_vec = ((uintptr_t)x & 15) == 0 && (m == 1 || x_stride * (long long)esize % 16 == 0);
        codes = nullptr;
    } else {
        const int q = saem_mx_quantize(x, x_dtype, m, k, x_stride, codes, scales, stream);
        if (q != SAEM_OK) return q;
        p.w_early = 1;
    }
    return launch_mx_matmul(plan, p, codes, (const uint8_t*)w_codes, n_sm, (cudaStream_t)stream) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}

}  // extern "C"
