// Attention of many rows per key head over a paged cache, on tcgen05: tiles of 2 x 128 rows against tiles of 128 places.
//
// One persistent CTA per SM: a warp that walks through the CTA's range of the plan and hands its items on, a warp that copies key and
// value tiles (TMA, a box per page or part of one) into a ring, one that copies queries, one that issues the products, and two groups of
// four warps, a thread per row, that turn scores into weights.  Scores S = Q K^T come to tensor memory, a thread reads its row, and writes
// the weights back over it as the 16-bit A operand of O += P V; O stays in tensor memory.  While one group works on its scores the
// tensor cores work for the other.  Values are used as they lie in the cache (places along the rows, the MN-major form of B), so
// nothing is transposed.
//
// The maximum that a row's weights refer to is only moved, and O multiplied, where it has grown by more than 2^8: the result is the same but
// for rounding, 16-bit floats have the range, and it is rare after a row's first tiles.
//
// The weights are rounded to 16 bits, half a step each, because that is the width of the operand beside 16-bit values; their sum is of the unrounded
// ones.  A second product for what they lose would add 1024 cycles of the tensor cores, and as many conversions again, to a tile's 3300 cycles.
//
// An item of at most 128 rows (a short chunk, decoding sequences beside a prompt) is worked on by both groups, even tiles of places
// and odd ones, whose results are added up at its end.
#include "attend_plan.cuh"
#include "mx_tc.cuh"

namespace saem {

constexpr int kAtThreads = 384;             // a warpgroup that copies and issues products and looks ahead, two with rows
constexpr int kAtRegsFew = 72, kAtRegsMany = 216;                   // of 168 per thread at launch: 72 + 2 * 216 = 3 * 168
constexpr int kAtR = 256, kAtKeys = 128, kAtHead = 4, kAtSnap = 4;
constexpr int kAtMaxStages = 10;
constexpr int kAtStage = 32 * 128;          // a warp's place for 64 columns of its 32 rows' results
constexpr int kAtParts = 3;                 // items read ahead
enum { kAtBarAll = 1 };                     // named barrier of the eight warps with rows

template <int DK>
struct TilesShape {
    static constexpr int kTile = 128 * DK * 2;                      // bytes of 128 queries, keys or values
    static constexpr int kStages = DK == 128 ? 4 : 8;
    static constexpr int kSmem = 1024 + (2 + kStages) * kTile + 8 * kAtStage;
    static constexpr int kSlot = kAtR * (DK + 2);                   // floats of a partial result: maxima, sums, outputs [DK / 4][256][4]
    static_assert(kStages <= kAtMaxStages, "");
};
struct TilesArgs {
    AttendArgs a;
    int box;                                // places of a copy: divides page_size and 128
    int rows_total;                         // pages * kv_heads * page_size
};

__device__ __forceinline__ void tc_mma_f16_on(uint32_t on, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %4, 0;\n\t"
        "@p tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, q;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on) : "memory");
}
// A from tensor memory: two 16-bit elements of a row per column.
__device__ __forceinline__ void tc_mma_f16_ta_on(uint32_t on, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %4, 0;\n\t"
        "@p tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, q;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(on) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_ld32_now(uint32_t taddr, uint32_t* r) {
    tc_ld32_issue(taddr, r);
    tc_wait_ld();
    tc_reg_fence16(r);
    tc_reg_fence16(r + 16);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// A barrier at which all learn whether all are well.
__device__ __forceinline__ bool named_all(int id, int threads, bool v) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.and.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(id), "r"(threads), "r"((uint32_t)v) : "memory");
    return r != 0;
}
// Shared-memory descriptor of values as B: 64 elements of head_dim are a 128-byte row of the 128-byte swizzle, a place per row (MN-major);
// groups of eight places 1024 bytes apart, the next 64 elements a tile of 128 places on.
__device__ __forceinline__ uint64_t smem_desc_values(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 * 128 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// kind::f16, fp32 sums, M = 128, N = n; b_mn: B is MN-major.
template <bool F16>
__device__ __forceinline__ uint32_t idesc_attend(int n, bool b_mn) {
    return (1u << 4) | (F16 ? 0u : (1u << 7) | (1u << 10)) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// The limit of a wait that lasts as long as an item: a tile of places takes at most 2 us (rows with a NaN are summed again behind the last item).
__device__ __forceinline__ unsigned long long item_limit_ns(const AttendPart& p) { return kWaitLimitNs + 20000ull * (unsigned)max(0, p.key_end - p.key_begin); }

// The items that the CTA has ended, for their rows with a NaN: the walk once more, by the eight warps with rows.
template <bool F16>
__device__ __noinline__ void attend_items_again(const AttendArgs& a, const AttendPlan& plan, const int* ended, int* marks, int warp) {
    AttendWalk<kAtR, kAtKeys, kAtHead, kAtSnap> walk;
    if (a.seqs > kPlanWarpSeqs) walk.begin(a, plan);
    else walk.begin_alone<kAtHead + 1>(a);
    for (AttendPart p; walk.next(a, p);)
        if (p.whole || ended[p.slot & 1]) attend_again<F16, kAtKeys, 8, kAtBarAll>(a, p.e, p.s, p.h, p.r * kAtR, p.rows, marks, warp);
}

template <bool F16, int DK>
__global__ void __launch_bounds__(kAtThreads, 1)
attend_tiles_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TilesArgs args) {
    using Shape = TilesShape<DK>;
    constexpr int kStages = Shape::kStages, kTile = Shape::kTile, kLift = F16 ? 7 : 0;          // weights are at most 2^8
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bar_full[kStages], bar_empty[kStages], bar_tail, bar_end, bar_q[2], bar_free[2], bar_s[2], bar_p[2][2], bar_o[2], bar_part[kAtParts], bar_done[kAtParts];
    __shared__ AttendPart parts[kAtParts];  // the items at hand; one without rows ends the range
    __shared__ AttendPlan plan;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag, last_s, nan_s, ended_s[2];          // some row has a NaN; cut items (by the parity of the part's place) that this CTA has ended
    __shared__ float other_s[2][128];       // the second group's maxima and sums, where both worked on the same rows
    const AttendArgs& a = args.a;
    const uint32_t base = warp_uniform((smem_u32(smem_raw) + 1023u) & ~1023u), ring = base + 2 * kTile;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    volatile int* abort_p = &abort_flag;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
            mbar_init(smem_u32(&bar_empty[i]), 1);
        }
        mbar_init(smem_u32(&bar_tail), 1);
        mbar_init(smem_u32(&bar_end), 1);
        for (int g = 0; g < 2; ++g) {
            mbar_init(smem_u32(&bar_q[g]), 1);
            mbar_init(smem_u32(&bar_free[g]), 9);
            mbar_init(smem_u32(&bar_s[g]), 1);
            mbar_init(smem_u32(&bar_p[g][0]), 4);
            mbar_init(smem_u32(&bar_p[g][1]), 4);
            mbar_init(smem_u32(&bar_o[g]), 1);
        }
        for (int i = 0; i < kAtParts; ++i) {
            mbar_init(smem_u32(&bar_part[i]), 1);
            mbar_init(smem_u32(&bar_done[i]), 11);
        }
        abort_flag = nan_s = ended_s[0] = ended_s[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_s)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    pdl_launch_dependents();
    if (a.seqs > kPlanWarpSeqs) make_plan<kAtR, kAtKeys, kAtHead, kAtHead + 1, kAtThreads / 32>(a, plan);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_uniform(tmem_s);
    bool ok = true;
    int turn = 0;                                                   // items so far
    auto next = [&](unsigned long long limit = kWaitLimitNs) -> bool {                                     // false at the end, or when a wait has run out
        ok = ok && mbar_wait_warp(smem_u32(&bar_part[turn % kAtParts]), (turn / kAtParts) & 1, abort_p, a.status, limit);
        return ok && (int)warp_uniform(parts[turn % kAtParts].rows) > 0;
    };
    auto finished = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar_done[turn % kAtParts]));
        ++turn;
    };

    if (warp >= 4) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAtRegsMany));
        // ---------------------------------------------------------------- weights and results: a thread per row
        const int g = (warp - 4) >> 2, quarter = warp & 3, own = quarter * 32 + lane;
        const uint32_t t_lane = (uint32_t)(quarter * 32) << 16, t_s = tmem + t_lane + g * 128, t_o = tmem + t_lane + 256 + g * 128;
        float* const meet = reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw)));    // [DK / 4][128][4] over both tiles of queries
        int n_s = 0, n_o = 0;
        // all eight warps go on to an item or none: they meet at barriers there, one that has given up meanwhile too
        auto next_all = [&]() -> bool {
            next();
            ok = named_all(kAtBarAll, 256, ok);
            return ok && parts[turn % kAtParts].rows > 0;
        };
        for (; next_all(); finished()) {
            const AttendPart& p = parts[turn % kAtParts];
            const bool both = p.rows <= 128;                        // both groups on the same rows
            const int n_all = max(0, p.key_end - p.key_begin), n = both ? (n_all - g + 1) / 2 : n_all;
            const int tile_row = (both ? 0 : g * 128) + own, row0 = p.r * kAtR + (both ? 0 : g * 128);
            const bool in = tile_row < p.rows;
            const bool warp_in = (both ? 0 : g * 128) + quarter * 32 < p.rows;
            // the tiles of queries may be filled again: here, or once the sum of the two groups, which takes their place, is read
            auto free_queries = [&] {
                if (lane < 2 && n_all > (both ? lane : 0)) mbar_arrive(smem_u32(&bar_free[lane]));
            };
            if (!both) free_queries();
            int lo = 0, hi = INT_MAX;                               // rows that are none see everything: nobody reads them
            if (in) row_bounds(a, p.e, row0 + own, true, lo, hi);
            const int lo_most = __reduce_max_sync(0xffffffffu, lo), hi_least = __reduce_min_sync(0xffffffffu, hi);
            float m = -INFINITY, l = 0.f;                           // m: what the weights refer to, in scores
            for (int i = 0; i < n; ++i) {
                const int first = (p.key_begin + (both ? 2 * i + g : i)) * kAtKeys;
                ok = mbar_wait_warp(smem_u32(&bar_s[g]), n_s & 1, abort_p, a.status);
                if (!ok) break;
                ++n_s;
                if (warp_in) {
                    tc_fence_after();
                    uint32_t s[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tc_ld32_issue(t_s + c * 32, s + c * 32);
                    tc_wait_ld();
#pragma unroll
                    for (int c = 0; c < 8; ++c) tc_reg_fence16(s + c * 16);
                    if (first < lo_most || first + kAtKeys - 1 > hi_least) {
#pragma unroll
                        for (int c = 0; c < 128; ++c)
                            if (first + c < lo || first + c > hi) s[c] = 0xFF800000u;
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) mx[e] = max3(mx[e], __uint_as_float(s[c + 2 * e]), __uint_as_float(s[c + 2 * e + 1]));
                    const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                    const bool move = (top - m) * a.scale_log2 > 8.f;           // false where both are -inf
                    if (__any_sync(0xffffffffu, move)) {
                        const float to = move ? top : m, was = move ? fast_exp2((m - to) * a.scale_log2) : 1.f;
                        m = to;
                        l *= was;
                        if (i) {
#pragma unroll 1
                            for (int c = 0; c < DK / 32; ++c) {
                                uint32_t o[32];
                                tc_ld32_now(t_o + c * 32, o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * was);
                                tc_st32(t_o + c * 32, o);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m * a.scale_log2;
                    const uint64_t by = pack_f32x2(a.scale_log2, a.scale_log2), less = pack_f32x2(kLift - ref, kLift - ref);
                    uint64_t sum[2] = {0, 0};                                   // two sums each: zeros
#pragma unroll
                    for (int c = 0; c < 2; ++c) {                               // half of the places at a time: its products need not wait for the rest
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const uint64_t x = fma_f32x2(pack_b32x2(s[c * 64 + 2 * e], s[c * 64 + 2 * e + 1]), by, less);
                            const float p0 = fast_exp2(low_f32(x)), p1 = fast_exp2(high_f32(x));
                            sum[e & 1] = add_f32x2(sum[e & 1], pack_f32x2(p0, p1));
                            w[e] = pack2<F16>(p0, p1);
                        }
                        tc_st32(t_s + c * 32, w);
                        tc_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bar_p[g][c]));
                    }
                    const uint64_t both_sums = add_f32x2(sum[0], sum[1]);
                    l += low_f32(both_sums) + high_f32(both_sums);
                } else if (lane < 2) {
                    mbar_arrive(smem_u32(&bar_p[g][lane]));
                }
            }
            if (ok && n > 0) {
                ok = mbar_wait_warp(smem_u32(&bar_o[g]), n_o & 1, abort_p, a.status);
                ++n_o;
                tc_fence_after();
            }
            float ms = m * a.scale_log2;                            // in powers of two, as in the workspace
            float w_own = 1.f, w_other = 0.f;
            if (both) {
                named_sync(kAtBarAll, 256);                         // all products with the queries are done
                if (g == 1) {
                    other_s[0][own] = n > 0 ? ms : -INFINITY;
                    other_s[1][own] = l;
                    if (n > 0 && warp_in) {
#pragma unroll 1
                        for (int c = 0; c < DK / 32; ++c) {
                            uint32_t o[32];
                            tc_ld32_now(t_o + c * 32, o);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<uint4*>(meet + ((c * 8 + e) * 128 + own) * 4) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        }
                    }
                }
                named_sync(kAtBarAll, 256);
                if (g == 0) {
                    const float m2 = other_s[0][own], top = fmaxf(ms, m2), ref = top == -INFINITY ? 0.f : top;
                    w_own = fast_exp2(ms - ref);
                    w_other = fast_exp2(m2 - ref);
                    l = l * w_own + other_s[1][own] * w_other;
                    ms = top;
                }
            }
            const AttendPart e = parts[turn % kAtParts];
            const bool warp_writes = warp_in && (!both || g == 0), writes = in && warp_writes;   // this thread has a row's sum
            const bool add = both && n_all > 1;
            const int token_i = quotient(row0 + own, a.by_group), head = e.h * a.group + row0 + own - token_i * a.group;
            const long long token = e.e.first + token_i;
            uint8_t* const out = in ? a.out + (token * a.out_ts + head * a.out_hs) * 2 : nullptr;
            float* const slot = a.partials + (size_t)e.slot * Shape::kSlot;
            const uint32_t stage = base + (2 + kStages) * kTile + (warp - 4) * kAtStage;
            // 32 of the row's columns; two calls are 64, which leave in whole rows of 128 bytes: a thread's own stores would touch a row each
            auto finish = [&](const uint32_t* v, int c, float inv) {
                const uint64_t by = pack_f32x2(inv, inv);
                uint64_t any = 0;                                   // NaN if one of them is, or where infinities meet (which comes out the same again)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t w[4];
                    uint64_t sum = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint64_t x = mul_f32x2(pack_b32x2(v[8 * e + 2 * i], v[8 * e + 2 * i + 1]), by);
                        sum = add_f32x2(sum, x);
                        w[i] = pack2<F16>(low_f32(x), high_f32(x));
                    }
                    if (c * 32 + e * 8 < a.dim) any = add_f32x2(any, sum);
                    st_shared_v4(stage + lane * 128 + ((((c & 1) * 4 + e) ^ (lane & 7)) << 4), w[0], w[1], w[2], w[3]);
                }
                const float all = low_f32(any) + high_f32(any);
                if (all != all && in) nan_s = 1;
                if (c & 1) {
                    __syncwarp();
                    const int col = (c >> 1) * 64 + (lane & 7) * 8;
                    uint4 w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = i * 4 + (lane >> 3);
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                                     : "r"(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4)));
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint8_t* const to = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, (unsigned long long)out, i * 4 + (lane >> 3)));
                        if (to && col < a.dim) *reinterpret_cast<uint4*>(to + col * 2) = w[i];
                    }
                    __syncwarp();
                }
            };
            auto finish_lse = [&](float mx, float sum) {
                if (a.lse) a.lse[token * a.group * a.kv_heads + head] = log_sum_exp<kLift>(mx, sum);
            };
            if (warp_writes) {
                const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll 1
                for (int c = 0; c < DK / 32; ++c) {
                    uint32_t o[32];
                    if (n > 0) tc_ld32_now(t_o + c * 32, o);
                    else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    if (add) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 x = *reinterpret_cast<const float4*>(meet + ((c * 8 + i) * 128 + own) * 4);
                            o[4 * i] = __float_as_uint(fmaf(x.x, w_other, __uint_as_float(o[4 * i]) * w_own));
                            o[4 * i + 1] = __float_as_uint(fmaf(x.y, w_other, __uint_as_float(o[4 * i + 1]) * w_own));
                            o[4 * i + 2] = __float_as_uint(fmaf(x.z, w_other, __uint_as_float(o[4 * i + 2]) * w_own));
                            o[4 * i + 3] = __float_as_uint(fmaf(x.w, w_other, __uint_as_float(o[4 * i + 3]) * w_own));
                        }
                    }
                    if (e.whole) finish(o, c, inv);
                    else if (in) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            __stcg(reinterpret_cast<uint4*>(slot + 2 * kAtR + ((c * 8 + i) * kAtR + tile_row) * 4), make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
                    }
                }
                if (writes) {
                    if (e.whole) finish_lse(ms, l);
                    else {
                        __stcg(slot + tile_row, ms);
                        __stcg(slot + kAtR + tile_row, l);
                    }
                }
            }
            if (both) {
                __syncwarp();
                free_queries();
            }
            tc_fence_before();                                      // O is read before the next item's products
            if (!e.whole) {
                named_sync(kAtBarAll, 256);
                if (threadIdx.x == 128) {
                    __threadfence();                                // what the barrier has ordered before it, too
                    // a CTA that gave up leaves the item open
                    last_s = !*abort_p && atomicAdd(a.counters + e.first_cta, 1) == e.n_parts - 1;
                    if (last_s) {
                        a.counters[e.first_cta] = 0;
                        ended_s[e.slot & 1] = 1;
                    }
                }
                named_sync(kAtBarAll, 256);
                if (last_s) {
                    __threadfence();
                    auto part = [&](int j) { return a.partials + (size_t)part_slot(e.first_cta, j) * Shape::kSlot; };
                    if (e.rows <= 64) {
                        // few rows, and often many parts: the columns are shared out over the warps, and four parts are under way at once
                        const int blocks = e.rows <= 32 ? 1 : 2, row = (warp & (blocks - 1)) * 32 + lane, wide = DK / 32 * blocks;   // fours of columns a warp
                        const int at0 = (warp - 4) / blocks * wide, row_of_all = e.r * kAtR + row, t = quotient(row_of_all, a.by_group);
                        if (row < e.rows) {
                            const long long tok = e.e.first + t;
                            const int hd = e.h * a.group + row_of_all - t * a.group;
                            float mx = -INFINITY, sum = 0.f;
#pragma unroll 8
                            for (int j = 0; j < e.n_parts; ++j) mx = fmaxf(mx, __ldcg(part(j) + row));
                            const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll 8
                            for (int j = 0; j < e.n_parts; ++j) sum += fast_exp2(__ldcg(part(j) + row) - ref) * __ldcg(part(j) + kAtR + row);
                            const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                            float any = 0.f;
#pragma unroll 1
                            for (int c = at0; c < at0 + wide; c += 2) {
                                float4 v[2] = {};
#pragma unroll 4
                                for (int j = 0; j < e.n_parts; ++j) {
                                    const float* f = part(j);
                                    const float w = fast_exp2(__ldcg(f + row) - ref);
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        const float4 x = __ldcg(reinterpret_cast<const float4*>(f + 2 * kAtR + ((c + i) * kAtR + row) * 4));
                                        v[i].x = fmaf(x.x, w, v[i].x); v[i].y = fmaf(x.y, w, v[i].y); v[i].z = fmaf(x.z, w, v[i].z); v[i].w = fmaf(x.w, w, v[i].w);
                                    }
                                }
                                if (c * 4 < a.dim) {
                                    const uint4 w = make_uint4(pack2<F16>(v[0].x * inv, v[0].y * inv), pack2<F16>(v[0].z * inv, v[0].w * inv),
                                                               pack2<F16>(v[1].x * inv, v[1].y * inv), pack2<F16>(v[1].z * inv, v[1].w * inv));
#pragma unroll
                                    for (int i = 0; i < 2; ++i) any = fmaf(v[i].x * inv, 0.f, fmaf(v[i].y * inv, 0.f, fmaf(v[i].z * inv, 0.f, fmaf(v[i].w * inv, 0.f, any))));
                                    *reinterpret_cast<uint4*>(a.out + (tok * a.out_ts + hd * a.out_hs + c * 4) * 2) = w;
                                }
                            }
                            if (any != any) nan_s = 1;
                            if (a.lse && at0 == 0) a.lse[tok * a.group * a.kv_heads + hd] = log_sum_exp<kLift>(mx, sum);
                        }
                    } else if (warp_writes) {
                        float mx = -INFINITY, sum = 0.f;
#pragma unroll 4
                        for (int j = 0; j < e.n_parts; ++j) mx = fmaxf(mx, __ldcg(part(j) + tile_row));
                        const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll 4
                        for (int j = 0; j < e.n_parts; ++j) sum += fast_exp2(__ldcg(part(j) + tile_row) - ref) * __ldcg(part(j) + kAtR + tile_row);
                        const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
#pragma unroll 1
                        for (int c = 0; c < DK / 32; ++c) {
                            float v[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = 0.f;
#pragma unroll 2
                            for (int j = 0; j < e.n_parts; ++j) {
                                const float* f = part(j);
                                float4 x[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) x[i] = __ldcg(reinterpret_cast<const float4*>(f + 2 * kAtR + ((c * 8 + i) * kAtR + tile_row) * 4));
                                const float w = fast_exp2(__ldcg(f + tile_row) - ref);
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    v[4 * i] = fmaf(x[i].x, w, v[4 * i]); v[4 * i + 1] = fmaf(x[i].y, w, v[4 * i + 1]);
                                    v[4 * i + 2] = fmaf(x[i].z, w, v[4 * i + 2]); v[4 * i + 3] = fmaf(x[i].w, w, v[4 * i + 3]);
                                }
                            }
                            finish(reinterpret_cast<const uint32_t*>(v), c, inv);
                        }
                        if (in) finish_lse(mx, sum);
                    }
                }
            }
            named_sync(kAtBarAll, 256);                             // the groups go on together: 1 % slower if they drift apart
        }
        // no wait is left that this, which is long, could outlast
        if (ok && nan_s) attend_items_again<F16>(a, plan, ended_s, reinterpret_cast<int*>(meet), warp - 4);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAtRegsFew));
        if (warp == 0) {
            // ---------------------------------------------------------------- copies
            int pos = 0, tails = 0;                                     // tiles requested; those of them that end within
            for (; next(); finished()) {
                const AttendPart& p = parts[turn % kAtParts];
                const int n = p.key_end - p.key_begin;
                const int32_t* const table = a.table + p.s * a.table_stride;
                auto request = [&](int kt, bool values) {
                    const int st = pos % kStages;
                    if (pos >= kStages) ok = mbar_wait_warp(smem_u32(&bar_empty[st]), (pos / kStages - 1) & 1, abort_p, a.status);
                    if (!ok) return;
                    ++pos;
                    // lane l: the box of places l * box and on, if the sequence has any of them
                    const int place = kt * kAtKeys + lane * args.box, left = p.e.len - kt * kAtKeys;
                    const bool mine = lane * args.box < min(kAtKeys, left);
                    int row = args.rows_total;                          // out of the map: zeros
                    if (mine) {
                        const int entry = quotient(place, a.by_page), page = table[entry];
                        if (page >= 0 && page < a.pages) row = (page * a.kv_heads + p.h) * a.page_size + place - entry * a.page_size;
                        else atomicExch(a.status, SAEM_ERR_INVALID_ARG);
                    }
                    const bool tail = values && left < kAtKeys;
                    const uint32_t full = smem_u32(&bar_full[st]), bar = tail ? smem_u32(&bar_tail) : full, to = ring + st * kTile;
                    const int boxes = __popc(__ballot_sync(0xffffffffu, mine));
                    if (lane == 0) mbar_expect_tx(bar, boxes * args.box * DK * 2);
                    __syncwarp();
                    if (mine) {
                        const CUtensorMap* map = values ? &map_v : &map_k;
    #pragma unroll
                        for (int h = 0; h < DK / 64; ++h) tma_2d(to + h * kAtKeys * 128 + lane * args.box * 128, map, h * 64, row, bar);
                    }
                    if (tail) {
                        // values behind the sequence's last are anything, and 0 times anything may be NaN: zeros
                        ok = mbar_wait_warp(bar, tails & 1, abort_p, a.status);
                        ++tails;
                        for (int u = lane; u < (kAtKeys - left) * 8 * (DK / 64); u += 32) {
                            const int h = u / ((kAtKeys - left) * 8), at = u - h * ((kAtKeys - left) * 8);
                            st_shared_v4(to + h * kAtKeys * 128 + left * 128 + at * 16, 0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full);
                    }
                };
                if (p.rows > 128) {
                    for (int j = 0; j < n && ok; ++j) {
                        request(p.key_begin + j, false);
                        if (ok) request(p.key_begin + j, true);
                    }
                } else {
                    for (int j = 0; j < min(n, 2) && ok; ++j) request(p.key_begin + j, false);
                    for (int j = 0; j < n && ok; ++j) {
                        request(p.key_begin + j, true);
                        if (ok && j + 2 < n) request(p.key_begin + j + 2, false);
                    }
                }
            }
            ring_settle_warp(bar_full, kStages, pos, a.status);
        } else if (warp == 1) {
            // ---------------------------------------------------------------- products
            const uint32_t on = elect_one();
            const uint32_t idesc_s = idesc_attend<F16>(128, false), idesc_o = idesc_attend<F16>((a.dim + 15) & ~15, true);
            const uint64_t desc_k = smem_desc_sw128(base), desc_v = smem_desc_values(base);
            const int n_k = (a.dim + 15) / 16;
            int pos = 0, n_q[2] = {0, 0}, n_p[2] = {0, 0};
            auto take = [&](int at) {                                   // the ring's tile `at`
                ok = ok && mbar_wait_warp(smem_u32(&bar_full[at % kStages]), (at / kStages) & 1, abort_p, a.status);
                tc_fence_after();
            };
            auto give = [&](int at) { tc_commit_on(on, smem_u32(&bar_empty[at % kStages])); };
            auto scores = [&](int g, int at, bool first, bool last) {
                if (first) {
                    ok = ok && mbar_wait_warp(smem_u32(&bar_q[g]), n_q[g] & 1, abort_p, a.status);
                    ++n_q[g];
                    tc_fence_after();
                }
                if (!ok) return;
                const uint64_t dq = desc_at(desc_k, g * kTile), dk = desc_at(desc_k, 2 * kTile + at % kStages * kTile);
    #pragma unroll
                for (int k = 0; k < DK / 16; ++k)
                    if (k < n_k) {
                        const uint32_t off = k / 4 * kAtKeys * 128 + k % 4 * 32;
                        tc_mma_f16_on(on, tmem + g * 128, desc_at(dq, off), desc_at(dk, off), idesc_s, k > 0);
                    }
                if (last) tc_commit_on(on, smem_u32(&bar_free[g]));
                tc_commit_on(on, smem_u32(&bar_s[g]));
            };
            auto outputs = [&](int g, int at, bool first, bool last) {
                const uint64_t dv = desc_at(desc_v, 2 * kTile + at % kStages * kTile);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && mbar_wait_warp(smem_u32(&bar_p[g][half]), n_p[g] & 1, abort_p, a.status);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int k = half * 4; k < half * 4 + 4; ++k)
                        tc_mma_f16_ta_on(on, tmem + 256 + g * 128, tmem + g * 128 + k * 8, desc_at(dv, k * 16 * 128), idesc_o, !first || k > 0);
                }
                ++n_p[g];
                if (last) tc_commit_on(on, smem_u32(&bar_o[g]));
            };
            for (; next(); finished()) {
                const AttendPart& p = parts[turn % kAtParts];
                const int n = (int)warp_uniform(p.key_end - p.key_begin);      // operands of the products stay in uniform registers
                if (n <= 0) continue;
                if (warp_uniform(p.rows) > 128) {
                    int k_at = pos++;
                    take(k_at);
                    scores(0, k_at, true, n == 1);
                    scores(1, k_at, true, n == 1);
                    give(k_at);
                    for (int j = 0; j < n && ok; ++j) {
                        const int v_at = pos++;
                        take(v_at);
                        outputs(0, v_at, j == 0, j == n - 1);
                        if (j + 1 < n) {
                            k_at = pos++;
                            take(k_at);
                            scores(0, k_at, false, j + 2 == n);
                        }
                        outputs(1, v_at, j == 0, j == n - 1);
                        give(v_at);
                        if (j + 1 < n) {
                            scores(1, k_at, false, j + 2 == n);
                            give(k_at);
                        }
                    }
                } else {
                    for (int j = 0; j < min(n, 2) && ok; ++j) {
                        const int at = pos++;
                        take(at);
                        scores(j, at, true, j + 2 >= n);
                        give(at);
                    }
                    for (int j = 0; j < n && ok; ++j) {
                        const int v_at = pos++;
                        take(v_at);
                        outputs(j & 1, v_at, j < 2, j + 2 >= n);
                        give(v_at);
                        if (j + 2 < n) {
                            const int at = pos++;
                            take(at);
                            scores(j & 1, at, false, j + 4 >= n);
                            give(at);
                        }
                    }
                }
            }
            // whatever is under way ends before tensor memory is given back
            tc_commit_on(on, smem_u32(&bar_end));
            mbar_settle_warp(smem_u32(&bar_end), 0, a.status);
        } else if (warp == 2) {
            // ---------------------------------------------------------------- items
            AttendWalk<kAtR, kAtKeys, kAtHead, kAtSnap> walk;
            if (a.seqs > kPlanWarpSeqs) walk.begin(a, plan);
            else walk.begin_alone<kAtHead + 1>(a);
            for (bool more = true; more; ++turn) {
                const int at = turn % kAtParts;
                if (turn >= kAtParts && !mbar_wait_warp(smem_u32(&bar_done[at]), (turn / kAtParts - 1) & 1, abort_p, a.status, item_limit_ns(parts[at]))) break;
                AttendPart p;
                more = walk.next(a, p);
                if (!more) p.rows = 0;
                else if (p.e.cut() && lane == 0) atomicExch(a.status, SAEM_ERR_INVALID_ARG);
                if (lane == 0) {
                    parts[at] = p;
                    mbar_arrive(smem_u32(&bar_part[at]));
                }
                __syncwarp();
            }
        } else {
            // ---------------------------------------------------------------- queries, in the 128-byte swizzle
            int n_q[2] = {0, 0};
            unsigned long long limit = kWaitLimitNs;                    // of the longest item so far: it may be under way still
            for (; next(limit); finished()) {
                const AttendPart p = parts[turn % kAtParts];
                const bool both = p.rows <= 128;
                for (int g = 0; g < 2; ++g) {
                    if (p.key_end - p.key_begin <= (both ? g : 0)) continue;                     // the group has no tiles
                    if (n_q[g]) ok = ok && mbar_wait_warp(smem_u32(&bar_free[g]), (n_q[g] - 1) & 1, abort_p, a.status, limit);
                    if (!ok) break;
                    ++n_q[g];
                    // eight rows at a time, four lanes to a row; rows beyond the item's are left as they are, nobody reads what comes of them
                    const int skip = both ? 0 : g * 128, n_rows = min(128, p.rows - skip);
#pragma unroll 2
                    for (int r = lane >> 2; r < n_rows; r += 8) {
                        const int row = p.r * kAtR + skip + r, t = quotient(row, a.by_group), head = p.h * a.group + row - t * a.group;
                        const uint8_t* q = a.q + ((p.e.first + t) * a.q_ts + head * a.q_hs) * 2;
                        const uint32_t to = base + g * kTile + r * 128;
#pragma unroll
                        for (int j = 0; j < DK / 32; ++j) {
                            const int c = j * 4 + (lane & 3);
                            const bool in = c * 8 < a.dim;
                            cp_async16(to + c / 8 * kAtKeys * 128 + ((c % 8 ^ (r & 7)) << 4), q + (in ? c * 16 : 0), in ? 16 : 0);
                        }
                    }
                    cp_async_commit();
                    cp_async_wait<0>();
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bar_q[g]));
                }
                limit = max(limit, item_limit_ns(p));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// ------------------------------------------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static std::atomic<EncodeTiledFn> g_attend_encode{nullptr};
static DeviceOnce g_attend_once;

static cudaError_t attend_tiles_init() {
    return once_on_device(g_attend_once, [] {
        cudaError_t e;
        if (!g_attend_encode) {
            void* fn = nullptr;
            cudaDriverEntryPointQueryResult q;
            e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
            if (e != cudaSuccess) return e;
            if (!fn || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
            g_attend_encode = (EncodeTiledFn)fn;
        }
        e = cudaFuncSetAttribute(attend_tiles_kernel<false, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TilesShape<64>::kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_tiles_kernel<true, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TilesShape<64>::kSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_tiles_kernel<false, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TilesShape<128>::kSmem);
        return e != cudaSuccess ? e : cudaFuncSetAttribute(attend_tiles_kernel<true, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TilesShape<128>::kSmem);
    });
}

// A cache as rows of head_dim elements, a row per place: boxes of 64 elements (the 128-byte swizzle's row) x `box` places; what lies
// outside reads as zero.
static bool make_cache_map(CUtensorMap* m, const void* p, bool f16, int dim, long long rows, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)dim, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)dim * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return g_attend_encode.load(std::memory_order_relaxed)(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims,
                           strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t attend_tiles_partials(int dim, int n_sm) { return (size_t)2 * n_sm * (dim <= 64 ? TilesShape<64>::kSlot : TilesShape<128>::kSlot) * 4; }

cudaError_t launch_attend_tiles(const AttendArgs& a, bool f16, int n_sm, cudaStream_t st) {
    cudaError_t e = attend_tiles_init();
    if (e != cudaSuccess) return e;
    TilesArgs t = {a, 128, (int)(a.pages * a.kv_heads * a.page_size)};
    while (a.page_size % t.box) t.box /= 2;
    t.a.by_ctas = divisor_of((uint32_t)n_sm);
    alignas(64) CUtensorMap map_k, map_v;
    if (!make_cache_map(&map_k, a.k, f16, a.dim, t.rows_total, t.box) || !make_cache_map(&map_v, a.v, f16, a.dim, t.rows_total, t.box)) return cudaErrorInvalidValue;
    const dim3 grid(n_sm), block(kAtThreads);
    if (a.dim <= 64)
        return f16 ? launch_pdl(attend_tiles_kernel<true, 64>, grid, block, TilesShape<64>::kSmem, st, map_k, map_v, t)
                   : launch_pdl(attend_tiles_kernel<false, 64>, grid, block, TilesShape<64>::kSmem, st, map_k, map_v, t);
    return f16 ? launch_pdl(attend_tiles_kernel<true, 128>, grid, block, TilesShape<128>::kSmem, st, map_k, map_v, t)
               : launch_pdl(attend_tiles_kernel<false, 128>, grid, block, TilesShape<128>::kSmem, st, map_k, map_v, t);
}

}  // namespace saem
