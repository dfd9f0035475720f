// The expert FFN over microscaled 4-bit experts (SAEM_FFN_MX contexts): h = silu(Wg x) * (Wu x), y = Wd h.
//
// A decode batch reads every active expert's bytes once, so the bound is DRAM, and the arithmetic has to keep up with
// some 46 codes per cycle and SM.  The weights are the A operand of mma.sync.m16n8k16 (a decode batch's few columns
// would leave tcgen05's 128 x 8 tiles waiting for the same bytes, behind a longer start-up): a unit (16 weight rows x 128
// elements, mx_common.cuh) is two 16-byte shared-memory loads and two scale words per lane; eight codes become four f16
// pairs with one cvt each (E2M1 is exact in f16), two MMAs multiply a block of 32 elements, and the block's scale,
// different in every row, multiplies the fp32 partial sums -- four FMAs for 512 codes.  Units come through a ring of
// bulk copies (cp.async.bulk) that one producer warp keeps full across items, so that DRAM never waits for a barrier
// between the consumer warps.
//
// The activations are the B operand in f16, a run of 64 or 128 elements of a row at a time brought to [2^14, 2^15) by a
// power of two that is multiplied back in fp32.  bf16 activations stay exact unless they are 2^-28 of the run's largest;
// the hidden activations are rounded to f16's 11 bits there and nowhere else.
//
// Two forms.  Up to 8 tokens (mx_few_*): the whole step in two launches.  Every CTA routes the batch itself; the columns
// of all MMAs are the batch's tokens, so the down projection runs along one long axis over (expert, hidden unit) with
// the gate weight folded into the column's factor, and the merge over a token's experts costs nothing.  Its routing and
// its first weights do not depend on the first launch and are under way while that one drains.  More tokens (mx_rows,
// mx_ffn): the rows packed by expert, in tiles of 8..64.
#include "mx_common.cuh"
#include "route_row.cuh"
#include "tc_common.cuh"

namespace saem {

constexpr int kMoeWarps = 8;                // consumer warps; one more warp copies
constexpr int kMoeThreads = (kMoeWarps + 1) * 32;
constexpr int kStageUnits = 2 * kMoeWarps;  // units of a ring stage: two per consumer warp
constexpr int kStageWBytes = kStageUnits * kMxUnitBytes;
constexpr int kMaxStages = 8;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Barrier of the consumer warps only.
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kMoeWarps * 32) : "memory"); }

struct MxUnit {                 // one lane's part of a unit
    uint4 q0, q1;               // codes of rows g and g + 8
    uint32_t s0, s1;            // their scales
};
__device__ __forceinline__ void load_unit(MxUnit& u, const uint8_t* p, int lane) {
    u.q0 = reinterpret_cast<const uint4*>(p)[lane];
    u.q1 = reinterpret_cast<const uint4*>(p + 512)[lane];
    u.s0 = reinterpret_cast<const uint32_t*>(p + kMxUnitScales)[lane >> 2];
    u.s1 = reinterpret_cast<const uint32_t*>(p + kMxUnitScales + 32)[lane >> 2];
}

// acc[j] += unit x (8 activation rows j).  frag(j, b): the lane's 16 bytes of f16 activations (row 8 j + g, elements
// 32 b + 8 t ..); factor(j, r): the factors of rows 8 j + 2 t and + 1 for run r of RUN elements.
template <int NT, int RUN, typename Frag, typename Factor>
__device__ __forceinline__ void unit_mma(const MxUnit& u, int nt, float (&acc)[NT][4], Frag frag, Factor factor) {
    const uint32_t q0[4] = {u.q0.x, u.q0.y, u.q0.z, u.q0.w}, q1[4] = {u.q1.x, u.q1.y, u.q1.z, u.q1.w};
    float s0[4], s1[4];
    mx_scales4(u.s0, s0);
    mx_scales4(u.s1, s1);
    constexpr int kBlocks = RUN / kMxBlock;                  // blocks that share a factor
#pragma unroll
    for (int r = 0; r < 4 / kBlocks; ++r) {
        uint32_t a[kBlocks][4], c[kBlocks][4];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            mx_decode8(q0[r * kBlocks + b], a[b]);
            mx_decode8(q1[r * kBlocks + b], c[b]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (j >= nt) break;
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const int blk = r * kBlocks + b;
                const uint4 x = frag(j, blk);
                float m[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(m, a[b][0], c[b][0], a[b][1], c[b][1], x.x, x.y);
                mma_f16(m, a[b][2], c[b][2], a[b][3], c[b][3], x.z, x.w);
                part[0] += s0[blk] * m[0];
                part[1] += s0[blk] * m[1];
                part[2] += s1[blk] * m[2];
                part[3] += s1[blk] * m[3];
            }
            const float2 f = factor(j, r);
            acc[j][0] += f.x * part[0];
            acc[j][1] += f.y * part[1];
            acc[j][2] += f.x * part[2];
            acc[j][3] += f.y * part[3];
        }
    }
}

// Power of two that brings a run whose largest magnitude has these fp32 bits to [2^14, 2^15), and its inverse.  A run
// with an infinity or NaN keeps its values (factor 1): every output of that row is then not finite either.
__device__ __forceinline__ void run_scale(uint32_t amax_bits, float& up, float& down) {
    int e = (int)(amax_bits >> 23);
    e = e == 255 ? 141 : max(e, 15);                         // both powers are normal numbers
    up = __uint_as_float((uint32_t)(268 - e) << 23);
    down = __uint_as_float((uint32_t)(e - 14) << 23);
}
__device__ __forceinline__ uint2 pack_half4(const float (&v)[4], float up) {
    const __half2 lo = __floats2half2_rn(v[0] * up, v[1] * up), hi = __floats2half2_rn(v[2] * up, v[3] * up);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}
__device__ __forceinline__ uint32_t abs_max4(const float (&v)[4]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}

struct Ring {                   // shared-memory addresses; `n` stages `bytes` apart
    uint32_t full, empty;       // arrays of 8-byte barriers
    uint8_t* data;
    int n, bytes;
};
// At an abort: copies that are still under way land before the CTA ends.  `issued` stages were requested in all.
__device__ void drain(const Ring& r, int issued, volatile int* abort_flag, int* status) {
    for (int i = max(0, issued - r.n); i < issued; ++i) {
        *abort_flag = 0;
        mbar_wait(r.full + 8 * (i % r.n), (i / r.n) & 1, abort_flag, status);
        *abort_flag = 1;
    }
}

// =================================================================================================== more than 8 tokens
constexpr int kRun = 64;                    // elements that share a factor
constexpr int kTileSpans = kStageUnits / kMoeWarps;          // a stage: 8 groups of 16 weight rows x 2 spans
constexpr int kRowPitch = kTileSpans * kMxSpan * 2 + 64;     // bytes between staged rows: 64 off a multiple of 128, so that
                                                             // eight rows x 64 bytes of a fragment load meet no bank twice
constexpr int kRowFactors = kTileSpans * kMxSpan / kRun;     // floats (16 bytes) per staged row

// Factors of a row of K elements in global memory: padded so that every stage's four floats are 16-byte aligned.
__host__ __device__ inline int factor_pitch(int K) { return (K / kRun + 3) & ~3; }

// Packed rows of bf16 to f16 with a factor per 64 elements: one warp per 128 elements, a half-warp per run.
__global__ void __launch_bounds__(256)
mx_rows_kernel(const uint16_t* __restrict__ x, int rows, int K, __half* __restrict__ xh, float* __restrict__ xf) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, n_span = K / kMxSpan;
    const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (i >= (long long)rows * n_span) return;
    const int row = (int)(i / n_span), span = (int)(i % n_span);
    const size_t at = (size_t)row * K + span * kMxSpan + 4 * lane;
    const uint2 q = *reinterpret_cast<const uint2*>(x + at);
    const float v[4] = {__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16),
                        __uint_as_float(q.y & 0xFFFF0000u)};
    uint32_t m = abs_max4(v);
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    float up, down;
    run_scale(m, up, down);
    *reinterpret_cast<uint2*>(xh + at) = pack_half4(v, up);
    if ((lane & 15) == 0) xf[(size_t)row * factor_pitch(K) + span * 2 + (lane >> 4)] = down;
}

struct MoeArgs {
    const __half* x;            // gate/up: xh [rows, d]; down: hh [rows, f]
    const float* xf;            // their factors
    const int32_t* offsets;     // [E + 1], or nullptr: one segment [0, max_rows)
    int max_rows, E, d, f;
    const uint8_t* slot_region;
    size_t slot_bytes;
    __half* hh;                 // gate/up: output rows and factors
    float* hf;
    float* y;                   // down: output
    int* status;
    int n_stage;
};

// MODE 0: gate/up (x -> h), MODE 1: down (h -> y).  A CTA takes items of (expert, 8 * NT rows, 8 groups of 16 weight
// rows); each consumer warp owns a group, the activations of a stage are copied beside its units.
template <int MODE, int NT>
__global__ void __launch_bounds__(kMoeThreads)
mx_ffn_kernel(const __grid_constant__ MoeArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(128) uint8_t smem[];
    constexpr int kTileRows_ = 8 * NT;
    constexpr int kStageBytes = kStageWBytes + kTileRows_ * (kRowPitch + kRowFactors * 4);
    __shared__ alignas(8) uint64_t bars[2 * kMaxStages];
    __shared__ int first[SAEM_MAX_EXPERTS + 1], start[SAEM_MAX_EXPERTS], rows_of[SAEM_MAX_EXPERTS], warp_sum[4];
    __shared__ uint32_t red[2][kMoeWarps][kTileRows_];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int K = MODE == 0 ? a.d : a.f, n_span = K / kMxSpan, n_chunk = (n_span + kTileSpans - 1) / kTileSpans;
    const int n_gb = (MODE == 0 ? a.f / 8 : a.d / 16) / kMoeWarps;              // d, f are multiples of 128
    const Ring ring = {smem_u32(bars), smem_u32(bars + kMaxStages), smem, a.n_stage, kStageBytes};
    volatile int* abort_p = &abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < ring.n; ++i) {
            mbar_init(ring.full + 8 * i, 1);
            mbar_init(ring.empty + 8 * i, kMoeWarps);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_launch_dependents();
    // items per expert and their prefix sums (SAEM_MAX_EXPERTS = 128 = four warps)
    if (threadIdx.x < SAEM_MAX_EXPERTS) {
        const int e = threadIdx.x;
        int n = 0, lo = 0;
        if (e < a.E) {
            lo = a.offsets ? a.offsets[e] : 0;
            int hi = a.offsets ? a.offsets[e + 1] : a.max_rows;
            lo = min(max(lo, 0), a.max_rows);
            hi = min(max(hi, lo), a.max_rows);
            n = hi - lo;
            if (n > 0 && tab.slot[e] < 0) {
                if (tab.in_subset[e] && MODE == 0 && blockIdx.x == 0) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
                n = 0;
            }
        }
        start[e] = lo;
        rows_of[e] = n;
        const int items = (n + kTileRows_ - 1) / kTileRows_ * n_gb;
        int s = items;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += v;
        }
        if (lane == 31) warp_sum[warp] = s;
        first[e + 1] = s;                                                      // within the warp so far
    }
    __syncthreads();
    if (threadIdx.x < SAEM_MAX_EXPERTS) {
        int before = 0;
        for (int w = 0; w < warp; ++w) before += warp_sum[w];
        first[threadIdx.x + 1] += before;
        if (threadIdx.x == 0) first[0] = 0;
    }
    __syncthreads();
    const int total = first[SAEM_MAX_EXPERTS];

    struct Item { int e, gb, row0, rows; };
    auto item_at = [&](int i) {
        int e = 0;
#pragma unroll
        for (int step = 64; step > 0; step >>= 1)                              // the last e with first[e] <= i
            if (first[e + step] <= i) e += step;
        const int tiles = (rows_of[e] + kTileRows_ - 1) / kTileRows_, rem = i - first[e];
        const int gb = rem / tiles, tile = rem - gb * tiles;
        return Item{e, gb, start[e] + tile * kTileRows_, min(kTileRows_, rows_of[e] - tile * kTileRows_)};
    };

    if (warp == kMoeWarps) {
        // ---------------------------------------------------------------- copies
        const size_t region = MODE == 0 ? 0 : mx_gate_up_units(a.d, a.f);
        int it = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            const Item t = item_at(i);
            const uint8_t* w = a.slot_region + (size_t)tab.slot[t.e] * a.slot_bytes +
                               (region + ((size_t)t.gb * kMoeWarps + (lane & 7)) * n_span) * kMxUnitBytes;
            for (int c = 0; c < n_chunk; ++c, ++it) {
                const int st = it % ring.n, spans = min(kTileSpans, n_span - c * kTileSpans);
                if (it >= ring.n) {
                    ok = mbar_wait(ring.empty + 8 * st, (it / ring.n - 1) & 1, abort_p, a.status);
                    if (!ok) break;
                }
                const uint32_t bar = ring.full + 8 * st;
                const uint32_t dst = smem_u32(ring.data) + st * kStageBytes;
                if (lane == 0)
                    mbar_expect_tx(bar, kMoeWarps * spans * kMxUnitBytes + t.rows * (spans * kMxSpan * 2 + kRowFactors * 4));
                __syncwarp();
                if (lane < kMoeWarps)
                    bulk_g2s(dst + lane * kTileSpans * kMxUnitBytes, w + (size_t)c * kTileSpans * kMxUnitBytes, spans * kMxUnitBytes, bar);
                for (int r = lane; r < t.rows; r += 32) {
                    bulk_g2s(dst + kStageWBytes + r * kRowPitch, a.x + (size_t)(t.row0 + r) * K + c * kTileSpans * kMxSpan,
                             spans * kMxSpan * 2, bar);
                    bulk_g2s(dst + kStageWBytes + kTileRows_ * kRowPitch + r * kRowFactors * 4,
                             a.xf + (size_t)(t.row0 + r) * factor_pitch(K) + c * kRowFactors, kRowFactors * 4, bar);
                }
            }
        }
        if (!ok && lane == 0) drain(ring, it, abort_p, a.status);
        return;
    }
    // -------------------------------------------------------------------- products
    const int g = lane >> 2, t = lane & 3;
    int it = 0, buf = 0;
    bool ok = true;
    for (int i = blockIdx.x; i < total; i += gridDim.x, buf ^= 1) {
        const Item im = item_at(i);
        const int nt = (im.rows + 7) / 8;
        float acc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[j][q] = 0.f;
        for (int c = 0; c < n_chunk; ++c, ++it) {
            const int st = it % ring.n, spans = min(kTileSpans, n_span - c * kTileSpans);
            ok = ok && mbar_wait(ring.full + 8 * st, (it / ring.n) & 1, abort_p, a.status);
            const uint8_t* base = ring.data + (size_t)st * kStageBytes;
            const uint8_t* xs = base + kStageWBytes + g * kRowPitch + 16 * t;
            const float* xf = reinterpret_cast<const float*>(base + kStageWBytes + kTileRows_ * kRowPitch) + 2 * t * kRowFactors;
            if (ok)
#pragma unroll
                for (int s = 0; s < kTileSpans; ++s)
                    if (s < spans) {
                        MxUnit u;
                        load_unit(u, base + (warp * kTileSpans + s) * kMxUnitBytes, lane);
                        unit_mma<NT, kRun>(u, nt, acc,
                            [&](int j, int b) { return *reinterpret_cast<const uint4*>(xs + j * 8 * kRowPitch + s * kMxSpan * 2 + b * 64); },
                            [&](int j, int r) {
                                const float* p = xf + 8 * j * kRowFactors + s * 2 + r;
                                return make_float2(p[0], p[kRowFactors]);
                            });
                    }
            __syncwarp();
            if (lane == 0) mbar_arrive(ring.empty + 8 * st);
        }
        // lane (g, t): rows g and g + 8 of the group, activation rows 8 j + 2 t and + 1
        const int group = im.gb * kMoeWarps + warp;
        if (MODE == 1) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int r = 8 * j + 2 * t + q;
                    if (!ok || r >= im.rows) continue;
                    float* o = a.y + (size_t)(im.row0 + r) * a.d + group * 16 + g;
                    o[0] = acc[j][q];
                    o[8] = acc[j][q + 2];
                }
        } else {
            // the item's 64 hidden units are one run of every row: its largest magnitude over the eight warps
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float z = acc[j][q], v = z / (1.f + expf(-z)) * acc[j][q + 2];
                    acc[j][q] = v;
                    uint32_t m = __float_as_uint(v) & 0x7FFFFFFFu;
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 4));
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 8));
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 16));
                    if (g == 0) red[buf][warp][8 * j + 2 * t + q] = m;
                }
            consumer_sync();
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int r = 8 * j + 2 * t + q;
                    if (!ok || r >= im.rows) continue;
                    uint32_t m = 0;
#pragma unroll
                    for (int w = 0; w < kMoeWarps; ++w) m = max(m, red[buf][w][r]);
                    float up, down;
                    run_scale(m, up, down);
                    a.hh[(size_t)(im.row0 + r) * a.f + group * 8 + g] = __float2half_rn(acc[j][q] * up);
                    if (warp == 0 && g == 0) a.hf[(size_t)(im.row0 + r) * factor_pitch(a.f) + im.gb] = down;
                }
        }
    }
}

// Regions of the context's MX workspace (at lay.h): f16 rows and factors of x and of h; the two-launch form keeps its
// fp32 hidden activations there instead.
struct MoeRegions {
    size_t xh, xf, hh, hf, total;
};
static MoeRegions moe_regions(long long rows, int d, int f) {
    MoeRegions r;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    r.xh = 0;
    r.xf = up(rows * (size_t)d * 2);
    r.hh = r.xf + up(rows * (size_t)factor_pitch(d) * 4);
    r.hf = r.hh + up(rows * (size_t)f * 2);
    r.total = r.hf + up(rows * (size_t)factor_pitch(f) * 4);
    const size_t few = up((rows < 8 * SAEM_MAX_EXPERTS ? rows : 8 * SAEM_MAX_EXPERTS) * (size_t)f * 4);
    if (r.total < few) r.total = few;
    return r;
}
size_t mx_workspace_bytes(long long rows, int d, int f) { return moe_regions(rows, d, f).total; }

constexpr int kSmemPerSm = 227 * 1024;

template <int MODE, int NT>
static cudaError_t launch_one(MoeArgs a, const SlotTable& tab, long long items, int n_sm, cudaStream_t st) {
    static bool done[64];
    constexpr int kStageBytes = kStageWBytes + 8 * NT * (kRowPitch + kRowFactors * 4);
    // two CTAs per SM where each then has two stages at least, else one
    const int per_sm = (kSmemPerSm / 2 - 8 * 1024) / kStageBytes >= 2 ? 2 : 1;
    const int n = (kSmemPerSm / per_sm - 8 * 1024) / kStageBytes;
    a.n_stage = n > kMaxStages ? kMaxStages : n;
    const int smem = a.n_stage * kStageBytes;
    if (first_call_on_device(done)) {
        const cudaError_t e = cudaFuncSetAttribute(mx_ffn_kernel<MODE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    const long long most = (long long)n_sm * per_sm;
    return launch_pdl(mx_ffn_kernel<MODE, NT>, dim3((unsigned)(items < most ? items : most)), dim3(kMoeThreads), (size_t)smem, st, a, tab);
}

cudaError_t launch_mx_ffn(const FfnArgs& f, const SlotTable& tab, int max_segment, cudaStream_t st, int* n_launch) {
    uint8_t* ws = reinterpret_cast<uint8_t*>(f.h);
    const MoeRegions r = moe_regions(f.h_rows, f.d, f.f);
    MoeArgs a = {};
    a.x = reinterpret_cast<__half*>(ws + r.xh);
    a.xf = reinterpret_cast<float*>(ws + r.xf);
    a.offsets = f.offsets; a.max_rows = f.max_rows; a.E = f.E; a.d = f.d; a.f = f.f;
    a.slot_region = f.slot_region; a.slot_bytes = f.slot_bytes; a.status = f.status;
    a.hh = reinterpret_cast<__half*>(ws + r.hh);
    a.hf = reinterpret_cast<float*>(ws + r.hf);
    a.y = f.y_packed;
    MoeArgs b = a;
    b.x = a.hh;
    b.xf = a.hf;
    const long long tasks = (long long)f.max_rows * (f.d / kMxSpan);
    cudaError_t e = launch_pdl(mx_rows_kernel, dim3((unsigned)((tasks + 7) / 8)), dim3(256), 0, st, f.x_packed, f.max_rows, f.d,
                               reinterpret_cast<__half*>(ws + r.xh), reinterpret_cast<float*>(ws + r.xf));
    if (e != cudaSuccess) return e;
    const int nt = max_segment <= 8 ? 1 : max_segment <= 16 ? 2 : max_segment <= 32 ? 4 : 8;
    const long long tiles = f.max_active + f.max_rows / (8 * nt);             // an upper bound of the row tiles
    const long long ia = tiles * (f.f / 64), ib = tiles * (f.d / 128);
#define SAEM_MX_NT(NT_)                                                                       \
    e = launch_one<0, NT_>(a, tab, ia, f.n_sm, st);                                           \
    if (e == cudaSuccess) e = launch_one<1, NT_>(b, tab, ib, f.n_sm, st)
    if (nt == 1) { SAEM_MX_NT(1); }
    else if (nt == 2) { SAEM_MX_NT(2); }
    else if (nt == 4) { SAEM_MX_NT(4); }
    else { SAEM_MX_NT(8); }
#undef SAEM_MX_NT
    if (e == cudaSuccess) *n_launch += 3;
    return e;
}

// ================================================================================================ up to 8 tokens
constexpr int kFewTokens = 8;
constexpr int kFewPairs = kFewTokens * kFewTokens;           // top_k <= 8
constexpr int kFewActive = kFewPairs + 16;                   // plus the always-on experts
constexpr int kFewStages = 4;

struct FewShared {
    alignas(8) uint64_t bars[2 * kFewStages];
    int idx[kFewPairs];
    float w[kFewPairs];
    uint32_t mask[4];
    int n_active;
    int16_t expert[kFewActive];
    int8_t slot_of_token[kFewActive][kFewTokens];            // j of the token's pair with this expert, -1: none
    alignas(16) float red[2][kMoeWarps][16 * kFewTokens];    // written in pairs
    int abort_flag;
};

// Routes the batch (one consumer warp per token) and lists the active experts in ascending order, the always-on ones
// last; experts without a slot are left out (status word).  All threads call it; ends with a barrier.
__device__ void few_route(FewShared& s, const MxFewArgs& a, const SlotTable& tab, bool report) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, P = a.T * a.k;
    if (threadIdx.x < 4) s.mask[threadIdx.x] = 0;
    if (warp < a.T) route_row(a.logits + (size_t)warp * a.E, a.E, a.k, a.renorm, lane, s.idx + warp * a.k, s.w + warp * a.k);
    __syncthreads();
    if (threadIdx.x < P) {
        const int e = s.idx[threadIdx.x];
        if (tab.slot[e] >= 0) atomicOr(&s.mask[e >> 5], 1u << (e & 31));
        else if (report) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
    }
    for (int i = threadIdx.x; i < kFewActive * kFewTokens; i += kMoeThreads) (&s.slot_of_token[0][0])[i] = -1;
    __syncthreads();
    auto position = [&](int e) {
        int p = __popc(s.mask[e >> 5] & ((1u << (e & 31)) - 1u));
        for (int q = 0; q < (e >> 5); ++q) p += __popc(s.mask[q]);
        return p;
    };
    if (threadIdx.x < P) {
        const int e = s.idx[threadIdx.x];
        if (tab.slot[e] >= 0) {
            const int p = position(e);
            s.expert[p] = (int16_t)e;
            s.slot_of_token[p][threadIdx.x / a.k] = (int8_t)(threadIdx.x % a.k);
        }
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
__device__ __forceinline__ void few_init(FewShared& s, const Ring& ring) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < ring.n; ++i) {
            mbar_init(ring.full + 8 * i, 1);
            mbar_init(ring.empty + 8 * i, kMoeWarps);
        }
        s.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
}
// Row of h that holds (token t, active expert): the pair's id, the always-on experts' rows behind the pairs.
__device__ __forceinline__ int few_row(const FewShared& s, const MxFewArgs& a, int active, int t) {
    const int j = s.slot_of_token[active][t], e = s.expert[active];
    return e < a.E ? t * a.k + j : a.T * a.k + (e - a.E) * a.T + t;
}
// Elements 4 lane .. + 3 of a 128-element run to f16 at dst, its factor returned to every lane.
__device__ __forceinline__ float few_stage(const float (&v)[4], __half* dst, int lane) {
    const uint32_t m = __reduce_max_sync(0xffffffffu, abs_max4(v));
    float up, down;
    run_scale(m, up, down);
    *reinterpret_cast<uint2*>(dst + 4 * lane) = pack_half4(v, up);
    return down;
}

// Gate, and gate/up projection: items are (active expert, G groups of 8 hidden units); a stage holds 16 / G spans of
// each group, and the warps that share a group split them.  x stays in shared memory for all items.
__global__ void __launch_bounds__(kMoeThreads)
mx_few_gate_up_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ FewShared s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n_span = a.d / kMxSpan, pitch = a.d + 32;                       // f16 elements; 64 bytes off a multiple of 128
    const int G = a.groups_a, spans = kStageUnits / G, n_chunk = (n_span + spans - 1) / spans, n_groups = a.f / 8;
    const Ring ring = {smem_u32(s.bars), smem_u32(s.bars + kFewStages), smem, kFewStages, kStageWBytes};
    __half* xs = reinterpret_cast<__half*>(smem + kFewStages * kStageWBytes);  // [T][pitch]
    float* xf = reinterpret_cast<float*>(xs + (size_t)a.T * pitch);            // [n_span][8]
    volatile int* abort_p = &s.abort_flag;
    few_init(s, ring);
    pdl_wait();
    pdl_launch_dependents();
    few_route(s, a, tab, blockIdx.x == 0);
    if (blockIdx.x == 0 && threadIdx.x < a.T * a.k) {
        a.topk_idx[threadIdx.x] = s.idx[threadIdx.x];
        a.topk_w[threadIdx.x] = s.w[threadIdx.x];
    }
    const int per = n_groups / G, total = s.n_active * per;                    // n_groups is a multiple of 16
    if (warp == kMoeWarps) {
        int it = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < total && ok; i += gridDim.x) {
            const int act = i / per, group0 = (i - act * per) * G;
            const uint8_t* w = a.slot_region + (size_t)tab.slot[s.expert[act]] * a.slot_bytes +
                               (size_t)(group0 + (lane & (G - 1))) * n_span * kMxUnitBytes;
            for (int c = 0; c < n_chunk; ++c, ++it) {
                const int st = it % ring.n, now = min(spans, n_span - c * spans);
                if (it >= ring.n) {
                    ok = mbar_wait(ring.empty + 8 * st, (it / ring.n - 1) & 1, abort_p, a.status);
                    if (!ok) break;
                }
                const uint32_t bar = ring.full + 8 * st;
                if (lane == 0) mbar_expect_tx(bar, G * now * kMxUnitBytes);
                __syncwarp();
                if (lane < G)
                    bulk_g2s(smem_u32(ring.data) + st * kStageWBytes + lane * spans * kMxUnitBytes,
                             w + (size_t)c * spans * kMxUnitBytes, now * kMxUnitBytes, bar);
            }
        }
        if (!ok && lane == 0) drain(ring, it, abort_p, a.status);
        return;
    }
    for (int i = warp; i < a.T * n_span; i += kMoeWarps) {
        const int r = i / n_span, sp = i - r * n_span;
        const uint2 q = *reinterpret_cast<const uint2*>(a.x + (size_t)r * a.d + sp * kMxSpan + 4 * lane);
        const float v[4] = {__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16),
                            __uint_as_float(q.y & 0xFFFF0000u)};
        const float f = few_stage(v, xs + (size_t)r * pitch + sp * kMxSpan, lane);
        if (lane == 0) xf[sp * 8 + r] = f;
    }
    consumer_sync();
    // columns beyond the batch repeat its last token; their sums are not used
    const __half* xrow = xs + (size_t)min(g, a.T - 1) * pitch + 8 * t;
    const int c0 = min(2 * t, a.T - 1), c1 = min(2 * t + 1, a.T - 1);
    const int gl = warp & (G - 1), ks = warp / G;
    int it = 0, buf = 0;
    bool ok = true;
    for (int i = blockIdx.x; i < total; i += gridDim.x, buf ^= 1) {
        const int act = i / per, group0 = (i - act * per) * G;
        float acc[1][4] = {{0.f, 0.f, 0.f, 0.f}};
        for (int c = 0; c < n_chunk; ++c, ++it) {
            const int st = it % ring.n;
            ok = ok && mbar_wait(ring.full + 8 * st, (it / ring.n) & 1, abort_p, a.status);
            const uint8_t* base = ring.data + (size_t)st * kStageWBytes;
            if (ok)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int local = 2 * ks + q, sp = c * spans + local;
                    if (sp >= n_span) continue;
                    MxUnit u;
                    load_unit(u, base + (gl * spans + local) * kMxUnitBytes, lane);
                    unit_mma<1, kMxSpan>(u, 1, acc,
                        [&](int, int b) { return *reinterpret_cast<const uint4*>(xrow + sp * kMxSpan + b * kMxBlock); },
                        [&](int, int) { return make_float2(xf[sp * 8 + c0], xf[sp * 8 + c1]); });
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(ring.empty + 8 * st);
        }
        // [row of the group][token] sums of every warp
        float* o = &s.red[buf][warp][g * kFewTokens + 2 * t];
        *reinterpret_cast<float2*>(o) = make_float2(acc[0][0], acc[0][1]);
        *reinterpret_cast<float2*>(o + 8 * kFewTokens) = make_float2(acc[0][2], acc[0][3]);
        consumer_sync();
        // G groups x 8 hidden units x 8 tokens; the warps that share a group are added in order
        for (int q = threadIdx.x; q < G * 64; q += kMoeWarps * 32) {
            const int grp = q >> 6, unit = q & 7, tok = (q >> 3) & 7;
            if (!ok || tok >= a.T || s.slot_of_token[act][tok] < 0) continue;
            float z = 0.f, up = 0.f;
            for (int w = grp; w < kMoeWarps; w += G) {
                z += s.red[buf][w][unit * kFewTokens + tok];
                up += s.red[buf][w][(8 + unit) * kFewTokens + tok];
            }
            a.h[(size_t)few_row(s, a, act, tok) * a.f + (group0 + grp) * 8 + unit] = z / (1.f + expf(-z)) * up;
        }
    }
}

// Down projection and merge: a CTA owns 16 output columns; its k axis runs over the active experts' hidden units.
__global__ void __launch_bounds__(kMoeThreads)
mx_few_down_kernel(const __grid_constant__ MxFewArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ FewShared s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int nf = a.f / kMxSpan, chunk = a.chunk_b, pitch = chunk * kMxSpan + 32;
    const Ring ring = {smem_u32(s.bars), smem_u32(s.bars + kFewStages), smem, kFewStages, kStageWBytes};
    __half* hs = reinterpret_cast<__half*>(smem + kFewStages * kStageWBytes);  // [T][pitch]
    float* hf = reinterpret_cast<float*>(hs + (size_t)a.T * pitch);            // [chunk][8]: factor x gate weight
    volatile int* abort_p = &s.abort_flag;
    few_init(s, ring);
    // What the first launch reads is complete when this one starts (its CTAs wait for it before they let this launch
    // begin), and the weights are not written by any of them: only h has to be waited for.
    few_route(s, a, tab, false);
    const int total = s.n_active * nf, n_stage = (total + kStageUnits - 1) / kStageUnits;
    if (warp == kMoeWarps) {
        bool ok = true;
        int it = 0;
        for (; it < n_stage; ++it) {
            const int st = it % ring.n;
            if (it >= ring.n) {
                ok = mbar_wait(ring.empty + 8 * st, (it / ring.n - 1) & 1, abort_p, a.status);
                if (!ok) break;
            }
            const uint32_t bar = ring.full + 8 * st;
            const int now = min(kStageUnits, total - it * kStageUnits);
            if (lane == 0) mbar_expect_tx(bar, now * kMxUnitBytes);
            __syncwarp();
            if (lane < now) {
                const int q = it * kStageUnits + lane, act = q / nf;
                bulk_g2s(smem_u32(ring.data) + st * kStageWBytes + lane * kMxUnitBytes,
                         a.slot_region + (size_t)tab.slot[s.expert[act]] * a.slot_bytes +
                             (mx_gate_up_units(a.d, a.f) + (size_t)blockIdx.x * nf + (q - act * nf)) * kMxUnitBytes,
                         kMxUnitBytes, bar);
            }
        }
        if (!ok && lane == 0) drain(ring, it, abort_p, a.status);
        pdl_wait();
        pdl_launch_dependents();
        return;
    }
    pdl_wait();
    pdl_launch_dependents();
    const __half* hrow = hs + (size_t)min(g, a.T - 1) * pitch + 8 * t;
    const int c0 = min(2 * t, a.T - 1), c1 = min(2 * t + 1, a.T - 1);
    float acc[1][4] = {{0.f, 0.f, 0.f, 0.f}};
    bool ok = true;
    int it = 0;
    for (int q0 = 0; q0 < total; q0 += chunk) {
        const int now = min(chunk, total - q0);
        if (q0) consumer_sync();                                               // the previous chunk has been read
        for (int i = warp; i < now * a.T; i += kMoeWarps) {
            const int l = i / a.T, r = i - l * a.T, act = (q0 + l) / nf, sp = q0 + l - act * nf;
            const int j = s.slot_of_token[act][r];
            __half* dst = hs + (size_t)r * pitch + l * kMxSpan;
            if (j < 0) {
                *reinterpret_cast<uint2*>(dst + 4 * lane) = make_uint2(0u, 0u);
                if (lane == 0) hf[l * 8 + r] = 0.f;
                continue;
            }
            const float4 q = __ldcg(reinterpret_cast<const float4*>(a.h + (size_t)few_row(s, a, act, r) * a.f + sp * kMxSpan) + lane);
            const float v[4] = {q.x, q.y, q.z, q.w};
            const float f = few_stage(v, dst, lane);
            if (lane == 0) hf[l * 8 + r] = f * (s.expert[act] < a.E ? s.w[r * a.k + j] : 1.f);
        }
        consumer_sync();
        for (int u0 = 0; u0 < now; u0 += kStageUnits, ++it) {                  // chunk is a multiple of a stage
            const int st = it % ring.n;
            ok = ok && mbar_wait(ring.full + 8 * st, (it / ring.n) & 1, abort_p, a.status);
            const uint8_t* base = ring.data + (size_t)st * kStageWBytes;
            if (ok)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int l = u0 + 2 * warp + q;
                    if (l >= now) continue;
                    MxUnit u;
                    load_unit(u, base + (2 * warp + q) * kMxUnitBytes, lane);
                    unit_mma<1, kMxSpan>(u, 1, acc,
                        [&](int, int b) { return *reinterpret_cast<const uint4*>(hrow + l * kMxSpan + b * kMxBlock); },
                        [&](int, int) { return make_float2(hf[l * 8 + c0], hf[l * 8 + c1]); });
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(ring.empty + 8 * st);
        }
    }
    float* o = &s.red[0][warp][g * kFewTokens + 2 * t];
    *reinterpret_cast<float2*>(o) = make_float2(acc[0][0], acc[0][1]);
    *reinterpret_cast<float2*>(o + 8 * kFewTokens) = make_float2(acc[0][2], acc[0][3]);
    consumer_sync();
    if (threadIdx.x < 16 * kFewTokens) {
        const int row = threadIdx.x & 15, tok = threadIdx.x >> 4;
        if (ok && tok < a.T) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kMoeWarps; ++w) v += s.red[0][w][row * kFewTokens + tok];
            const size_t at = (size_t)tok * a.d + blockIdx.x * 16 + row;
            if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
            else static_cast<float*>(a.out)[at] = v;
        }
    }
}

// The staged x may take 64 KB: beyond that (8 tokens of d_model > 4096) the packed form is as fast.
bool mx_few_supported(int T, int k, int d) { return T <= kFewTokens && k <= kFewTokens && (long long)T * d <= 32768; }

cudaError_t launch_mx_few(MxFewArgs a, const SlotTable& tab, int n_sm, cudaStream_t st, int* n_launch) {
    static bool done[64];
    if (first_call_on_device(done)) {
        cudaError_t e = cudaFuncSetAttribute(mx_few_gate_up_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_few_down_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
        if (e != cudaSuccess) return e;
    }
    const int n_span = a.d / kMxSpan;
    a.groups_a = n_span >= 16 ? 1 : n_span >= 8 ? 2 : n_span >= 4 ? 4 : 8;     // a stage is no longer than the k axis
    const size_t smem_a = kFewStages * kStageWBytes + (size_t)a.T * (a.d + 32) * 2 + (size_t)n_span * 8 * 4;
    a.chunk_b = 128 / a.T / 16 * 16;                                           // 32 KB of staged hidden activations
    const size_t smem_b = kFewStages * kStageWBytes + (size_t)a.T * (a.chunk_b * kMxSpan + 32) * 2 + (size_t)a.chunk_b * 8 * 4;
    const int pairs = a.T * a.k;
    const long long items = (long long)((pairs < a.E ? pairs : a.E) + a.S) * (a.f / 8 / a.groups_a);
    int per_sm = (int)(kSmemPerSm / (smem_a + 12 * 1024));
    if (per_sm > 3) per_sm = 3;
    const long long most = (long long)n_sm * per_sm;
    cudaError_t e = launch_pdl(mx_few_gate_up_kernel, dim3((unsigned)(items < most ? items : most)), dim3(kMoeThreads), smem_a, st, a, tab);
    if (e != cudaSuccess) return e;
    *n_launch += 1;
    e = launch_pdl(mx_few_down_kernel, dim3((unsigned)(a.d / 16)), dim3(kMoeThreads), smem_b, st, a, tab);
    if (e == cudaSuccess) *n_launch += 1;
    return e;
}

}  // namespace saem
