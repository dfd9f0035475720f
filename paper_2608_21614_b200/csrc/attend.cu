// Attention of new tokens over a paged cache: o = sum_j softmax_j(scale q.k_j) v_j.  The form for few rows per key head, and the call.
//
// attend_rows_kernel: tiles of 16 rows (a decoding sequence's query heads that share a key head; further tokens are further rows) by
// mma.sync m16n8k16.  With so few rows every key and value is used for little arithmetic and the bound is the cache's bytes, so that what
// counts is how many of them are under way: each of a CTA's 4 warps (two CTAs per SM) takes every fourth chunk of 16 places through a
// ring of its own in shared memory (cp.async, no barrier between warps), with its own running maximum, sum and output; they meet at
// the end of an item.  tcgen05 takes 128 rows at least, of which a decoding sequence fills 4 or 8, and its results would have to
// cross tensor memory twice for each tile.
#include "attend_plan.cuh"
#include "tc_common.cuh"

namespace saem {

constexpr int kRowsWarps = 4, kRowsThreads = kRowsWarps * 32;
constexpr int kRowsR = 16, kRowsKeys = 16, kRowsHead = 12;
constexpr int kRowsSnap = 12;
constexpr int kRowsLeast = 8;               // units of a CTA's range at least
constexpr int kRowsPerSm = 2;               // CTAs

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Two weights as 16-bit ones and what they lose.  A bfloat16 is cut, and its rest above 0 where the weight is, so that both parts' products with an
// infinity are that infinity (0 times it, or a sum of both signs, is NaN; float16 has no exponents for that, see attend_again).
template <bool F16>
__device__ __forceinline__ uint32_t cut2(float a, float b, float2& rest) {
    const uint32_t w = F16 ? pack2<true>(a, b) : __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    const float2 got = unpack2<F16>(w);
    rest = make_float2(a - got.x, b - got.y);
    if (!F16) rest = make_float2(fmaxf(rest.x, fminf(a, 0x1p-126f)), fmaxf(rest.y, fminf(b, 0x1p-126f)));
    return w;
}

// DK: head_dim rounded up to 64 or 128.
template <int DK>
struct RowsShape {
    static constexpr int kRow = DK * 2;                             // bytes of a place in shared memory
    static constexpr int kStage = 2 * kRowsKeys * kRow;             // keys, then values
    static constexpr int kStages = DK == 128 ? 3 : 6;
    static constexpr int kRing = kRowsWarps * kStages * kStage;     // 96 KB
    static constexpr int kMeet = 8 * (DK + 2);                      // floats of eight rows of a warp: maxima, sums, outputs
    static constexpr int kSmem = kRing + kRowsWarps * kMeet * 4;
    static constexpr int kSlot = kRowsR * (DK + 2);                 // floats of a partial result: maxima, sums, outputs
};

template <bool F16, int DK>
__global__ void __launch_bounds__(kRowsThreads, kRowsPerSm)
attend_rows_kernel(const __grid_constant__ AttendArgs a) {
    using Shape = RowsShape<DK>;
    constexpr int kStages = Shape::kStages, kLift = F16 ? 15 : 0;   // weights are at most 1
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ AttendPlan plan;
    __shared__ int last_s;
    __shared__ int nan_s;                   // a row of the item has a NaN
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    AttendWalk<kRowsR, kRowsKeys, kRowsHead, kRowsSnap> walk;
    if (a.seqs <= kPlanWarpSeqs) {
        walk.begin_alone<kRowsLeast>(a);
    } else {
        make_plan<kRowsR, kRowsKeys, kRowsHead, kRowsLeast, kRowsWarps>(a, plan);
        walk.begin(a, plan);
    }
    const uint32_t ring = smem_u32(smem) + warp * kStages * Shape::kStage;
    float* const meet = reinterpret_cast<float*>(smem + Shape::kRing);          // [warp][kMeet]
    const int quad = lane >> 2, two = (lane & 3) * 2;
    const int n_k = (a.dim + 15) / 16;                              // steps of 16 of head_dim

    // ---- requests: the chunks key_begin + warp + kRowsWarps * i of the part `p`, the next one's begun before the last one's result is written
    AttendPart p = {};
    int n_chunk = 0, pages = -1;                                    // lane l: page of chunk l of the 32 at hand
    const int32_t* table = a.table;
    bool bad = false;
    auto look_up = [&](int i) {
        pages = -1;
        if (i < n_chunk) pages = table[quotient((p.key_begin + warp + kRowsWarps * i) * kRowsKeys, a.by_page)];
    };
    // A lane copies the same 16 bytes of every row that it takes.
    constexpr int kPieces = DK / 8, kRowStep = 32 / kPieces;
    const int piece = lane % kPieces, first_row = lane / kPieces;
    const bool piece_in = piece * 8 < a.dim;
    const int lane_off = piece_in ? (first_row * a.dim + piece * 8) * 2 : 0, row_off = kRowStep * a.dim * 2;
    auto request = [&](int i) {
        if (i < n_chunk) {
            if (i % 32 == 0 && i) look_up(i + lane);
            int page = __shfl_sync(0xffffffffu, pages, i % 32);
            const int place = (p.key_begin + warp + kRowsWarps * i) * kRowsKeys;
            int valid = piece_in ? p.e.len - place : 0;
            if (page < 0 || page >= a.pages) { page = 0; valid = 0; bad = true; }
            const int in_page = place - quotient(place, a.by_page) * a.page_size;
            const long long from = ((long long)page * a.kv_heads * a.page_size + p.h * a.page_size + in_page) * (a.dim * 2) + lane_off;
            const uint8_t *k = a.k + from, *v = a.v + from;
            const uint32_t to = ring + i % kStages * Shape::kStage;
#pragma unroll
            for (int j = 0; j < kRowsKeys / kRowStep; ++j) {
                const int row = first_row + j * kRowStep, bytes = row < valid ? 16 : 0;
                const uint32_t at = to + row * Shape::kRow + ((piece ^ (row & 7)) << 4);
                cp_async16(at, k + j * row_off, bytes);
                cp_async16(at + kRowsKeys * Shape::kRow, v + j * row_off, bytes);
            }
        }
        cp_async_commit();
    };
    auto begin_part = [&]() -> bool {
        if (!walk.next(a, p)) return false;
        bad |= p.e.cut();
        n_chunk = max(0, (p.key_end - p.key_begin - warp + kRowsWarps - 1) / kRowsWarps);
        table = a.table + p.s * a.table_stride;
        look_up(lane);
#pragma unroll 1
        for (int i = 0; i < kStages - 1; ++i) request(i);
        return true;
    };

    bool more = begin_part();
    if (threadIdx.x == 0) nan_s = 0;
    while (more) {
        // ---- queries, as the A operand; the bounds of the lane's two rows
        const int row0 = p.r * kRowsR, rows = p.rows, head0 = p.h * a.group, s_now = p.s, h_now = p.h;
        const SeqExtent ext = p.e;
        uint32_t qf[DK / 16][4];
        int lo[2], hi[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int row = row0 + quad + 8 * b, i = quotient(row, a.by_group);
            const bool in = quad + 8 * b < rows;
            const uint8_t* q = a.q + ((ext.first + i) * a.q_ts + (head0 + row - i * a.group) * a.q_hs + two) * 2;
            row_bounds(a, ext, row, in, lo[b], hi[b]);
#pragma unroll
            for (int k = 0; k < DK / 16; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    qf[k][b + 2 * c] = in && k * 16 + c * 8 < a.dim ? *reinterpret_cast<const uint32_t*>(q + (k * 16 + c * 8) * 2) : 0u;
        }
        // An item of at most 8 rows leaves half of a tile's rows free: they take what the weights lose to 16 bits, and are added at the end (1 % of a
        // call).  An item of more rows has its weights in 16 bits: a second product for what they lose took 4 to 8 %.
        const bool half = rows <= 8;
        float o[DK / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int d = 0; d < DK / 8; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][i] = 0.f;

#pragma unroll 1
        for (int i = 0; i < n_chunk; ++i) {
            __syncwarp();                                           // the stage that the next request overwrites is read
            request(i + kStages - 1);
            cp_async_wait<kStages - 1>();
            __syncwarp();
            const uint32_t kt = ring + i % kStages * Shape::kStage, vt = kt + kRowsKeys * Shape::kRow;
            float sc[2][4] = {};
#pragma unroll
            for (int k = 0; k < DK / 16; ++k) {
                if (k < n_k) {
                    // matrices: places 0-7 and elements 0-7, places 0-7 and 8-15, places 8-15 and 0-7, places 8-15 and 8-15
                    const int row = (lane & 7) + (lane >> 4) * 8, c = 2 * k + ((lane >> 3) & 1);
                    uint32_t f[4];
                    ldmatrix4(f, kt + row * Shape::kRow + ((c ^ (row & 7)) << 4));
                    mma16816<F16>(sc[0], qf[k], f[0], f[1]);
                    mma16816<F16>(sc[1], qf[k], f[2], f[3]);
                }
            }
            const int place = (p.key_begin + warp + kRowsWarps * i) * kRowsKeys;
            float mx[2] = {m[0], m[1]};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = place + t * 8 + two + (e & 1), b = e >> 1;
                    sc[t][e] = j >= lo[b] && j <= hi[b] ? sc[t][e] * a.scale_log2 : -INFINITY;
                    mx[b] = fmaxf(mx[b], sc[t][e]);
                }
            float was[2], base[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                mx[b] = fmaxf(mx[b], __shfl_xor_sync(0xffffffffu, mx[b], 1));
                mx[b] = fmaxf(mx[b], __shfl_xor_sync(0xffffffffu, mx[b], 2));
                base[b] = mx[b] == -INFINITY ? 0.f : mx[b];
                was[b] = fast_exp2(m[b] - base[b]);
                m[b] = mx[b];
                l[b] *= was[b];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[t][e] = fast_exp2(sc[t][e] - (base[e >> 1] - kLift));
                    l[e >> 1] += sc[t][e];
                }
            if (half) was[1] = was[0];
            if (__any_sync(0xffffffffu, was[0] != 1.f || was[1] != 1.f)) {
#pragma unroll
                for (int d = 0; d < DK / 8; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][e] *= was[e >> 1];
            }
            uint32_t w[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float2 rest;
                const uint32_t most = cut2<F16>(sc[t][0], sc[t][1], rest);
                w[2 * t] = half ? most : pack2<F16>(sc[t][0], sc[t][1]);
                w[2 * t + 1] = pack2<F16>(half ? rest.x : sc[t][2], half ? rest.y : sc[t][3]);
            }
#pragma unroll
            for (int k = 0; k < DK / 16; ++k) {
                if (k < n_k) {
                    // transposed: places 0-7 and 8-15 of elements 16k .. 16k + 7, then of the eight behind them
                    const int row = (lane & 7) + ((lane >> 3) & 1) * 8, c = 2 * k + (lane >> 4);
                    uint32_t f[4];
                    ldmatrix4_t(f, vt + row * Shape::kRow + ((c ^ (row & 7)) << 4));
                    mma16816<F16>(o[2 * k], w, f[0], f[1]);
                    mma16816<F16>(o[2 * k + 1], w, f[2], f[3]);
                }
            }
        }
        cp_async_wait<0>();
        __syncwarp();
        if (half) {
#pragma unroll
            for (int d = 0; d < DK / 8; ++d) {
                o[d][0] += o[d][2];
                o[d][1] += o[d][3];
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            l[b] += __shfl_xor_sync(0xffffffffu, l[b], 1);
            l[b] += __shfl_xor_sync(0xffffffffu, l[b], 2);
        }
        const bool whole = p.whole;
        const int first_cta = p.first_cta, n_parts = p.n_parts, slot_i = p.slot;
        more = begin_part();

        // ---- the warps meet, eight rows at a time, while the next part's first places are on their way
        constexpr int kCols = DK / 4;
        const int col = threadIdx.x % kCols * 4;
        float* const slot = a.partials + (size_t)slot_i * Shape::kSlot;
        auto finish = [&](int row, float4 v, float mx, float sum) {
            const int i = quotient(row0 + row, a.by_group), head = head0 + row0 + row - i * a.group;
            const long long token = ext.first + i;
            const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
            v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
            if (v.x != v.x || v.y != v.y || v.z != v.z || v.w != v.w) nan_s = 1;
            if (col < a.dim) *reinterpret_cast<uint2*>(a.out + (token * a.out_ts + head * a.out_hs + col) * 2) = make_uint2(pack2<F16>(v.x, v.y), pack2<F16>(v.z, v.w));
            if (a.lse && col == 0) a.lse[token * a.group * a.kv_heads + head] = log_sum_exp<kLift>(mx, sum);
        };
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (b * 8 >= rows) break;
            if (quad + b * 8 < rows) {
                float* const mine = meet + warp * Shape::kMeet;
                if (two == 0) { mine[quad] = m[b]; mine[8 + quad] = l[b]; }
#pragma unroll
                for (int d = 0; d < DK / 8; ++d)
                    *reinterpret_cast<float2*>(mine + 16 + quad * DK + d * 8 + two) = make_float2(o[d][2 * b], o[d][2 * b + 1]);
            }
            __syncthreads();
#pragma unroll 1
            for (int r = threadIdx.x / kCols; r < min(8, rows - b * 8); r += kRowsThreads / kCols) {
                float w[kRowsWarps], top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int j = 0; j < kRowsWarps; ++j) {
                    w[j] = meet[j * Shape::kMeet + r];
                    top = fmaxf(top, w[j]);
                }
                const float base = top == -INFINITY ? 0.f : top;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int j = 0; j < kRowsWarps; ++j) {
                    w[j] = fast_exp2(w[j] - base);
                    sum = fmaf(meet[j * Shape::kMeet + 8 + r], w[j], sum);
                    const float4 x = *reinterpret_cast<const float4*>(meet + j * Shape::kMeet + 16 + r * DK + col);
                    v.x = fmaf(x.x, w[j], v.x); v.y = fmaf(x.y, w[j], v.y); v.z = fmaf(x.z, w[j], v.z); v.w = fmaf(x.w, w[j], v.w);
                }
                const int row = b * 8 + r;
                if (whole) {
                    finish(row, v, top, sum);
                } else {
                    if (col == 0) { __stcg(slot + row, top); __stcg(slot + kRowsR + row, sum); }
                    __stcg(reinterpret_cast<float4*>(slot + 2 * kRowsR + row * DK + col), v);
                }
            }
            __syncthreads();
        }
        if (!whole) {
            if (threadIdx.x == 0) {
                __threadfence();                                    // what the barrier has ordered before it, too
                last_s = atomicAdd(a.counters + first_cta, 1) == n_parts - 1;
                if (last_s) a.counters[first_cta] = 0;
            }
            __syncthreads();
            if (last_s) {
                __threadfence();
                constexpr int kAhead = 12;                          // parts whose loads are under way together
#pragma unroll 1
                for (int row = threadIdx.x / kCols; row < rows; row += kRowsThreads / kCols) {
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    float mx = -INFINITY, sum = 0.f;
#pragma unroll 1
                    for (int j0 = 0; j0 < n_parts; j0 += kAhead) {
                        float pm[kAhead], pl[kAhead];
                        float4 po[kAhead];
#pragma unroll
                        for (int j = 0; j < kAhead; ++j) {
                            const float* f = a.partials + (size_t)part_slot(first_cta, j0 + j) * Shape::kSlot;
                            const bool there = j0 + j < n_parts;
                            pm[j] = there ? __ldcg(f + row) : -INFINITY;
                            pl[j] = there ? __ldcg(f + kRowsR + row) : 0.f;
                            po[j] = there ? __ldcg(reinterpret_cast<const float4*>(f + 2 * kRowsR + row * DK + col)) : make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                        float top = mx;
#pragma unroll
                        for (int j = 0; j < kAhead; ++j) top = fmaxf(top, pm[j]);
                        const float base = top == -INFINITY ? 0.f : top, was = fast_exp2(mx - base);
                        mx = top;
                        sum *= was;
                        v = make_float4(v.x * was, v.y * was, v.z * was, v.w * was);
#pragma unroll
                        for (int j = 0; j < kAhead; ++j) {
                            const float w = fast_exp2(pm[j] - base);
                            sum = fmaf(pl[j], w, sum);
                            v.x = fmaf(po[j].x, w, v.x); v.y = fmaf(po[j].y, w, v.y); v.z = fmaf(po[j].z, w, v.z); v.w = fmaf(po[j].w, w, v.w);
                        }
                    }
                    finish(row, v, mx, sum);
                }
                __syncthreads();
            }
        }
        // the barriers above order this after the first results, and its own the next item's after it
        if (nan_s) {
            attend_again<F16, kRowsKeys, kRowsWarps, 0>(a, ext, s_now, h_now, row0, rows, reinterpret_cast<int*>(meet), warp);
            if (threadIdx.x == 0) nan_s = 0;
            __syncthreads();
        }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) atomicExch(a.status, SAEM_ERR_INVALID_ARG);
}

// Both forms have their partial results at the same place: calls that share a workspace are ordered.
static size_t partials_bytes(int dim, int n_sm) {
    const size_t rows = (size_t)2 * kRowsPerSm * n_sm * RowsShape<kHeadDimMax>::kSlot * 4, tiles = attend_tiles_partials(dim, n_sm);
    return rows > tiles ? rows : tiles;
}
// Which form, by the most rows of a sequence and key head and by the rows of all heads together (times in us: few, many).  Up to 16 rows read
// the cache once either way: 64 sequences of 2000 places 94, 110.  More read it once per 16 rows, from L2, but there are more items to
// share out, which is what counts while there are few in all: 60 tokens of 8 heads over 700 places 14.4, 24.0, 10 of 32 heads in each
// of 2 sequences of 1000 16.6, 20.3 (of 200 13.5, 11.1), 16 of 32 heads over 4000 22.7, 25.9 (over 16000 44.7, 35.4); and
// beyond: 5 of 32 heads in each of 8 sequences of 500 19.1, 15.3, of 16000 175, 98.
static bool rows_are_few(long long rows, long long all_rows) { return rows <= 16 || all_rows <= 768; }

template <bool F16, int DK>
static cudaError_t launch_rows_typed(AttendArgs a, int n_sm, cudaStream_t st) {
    static DeviceOnce once;
    const cudaError_t e = once_on_device(once, [] {
        return cudaFuncSetAttribute(attend_rows_kernel<F16, DK>, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsShape<DK>::kSmem);
    });
    if (e != cudaSuccess) return e;
    a.by_ctas = divisor_of((uint32_t)(kRowsPerSm * n_sm));
    return launch_pdl(attend_rows_kernel<F16, DK>, dim3(kRowsPerSm * n_sm), dim3(kRowsThreads), RowsShape<DK>::kSmem, st, a);
}
static cudaError_t launch_rows(const AttendArgs& a, bool f16, int n_sm, cudaStream_t st) {
    if (a.dim <= 64) return f16 ? launch_rows_typed<true, 64>(a, n_sm, st) : launch_rows_typed<false, 64>(a, n_sm, st);
    return f16 ? launch_rows_typed<true, 128>(a, n_sm, st) : launch_rows_typed<false, 128>(a, n_sm, st);
}

}  // namespace saem

using namespace saem;

extern "C" size_t saem_attend_workspace_bytes(const saem_kv_cache* c) {
    int n_sm;
    if (!c) return 0;
    const int r = cache_status(*c);
    if (r != SAEM_OK || sm_count(&n_sm) != cudaSuccess || kRowsPerSm * n_sm > kAttendMaxCtas) return 0;
    return SAEM_ATTEND_HEAD_BYTES + partials_bytes(c->head_dim, n_sm);
}

extern "C" int saem_attend(const saem_attend_config* c, const saem_kv_cache* cache, const saem_batch* b, const void* q, void* out,
                           float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (!c || !cache || !b) return SAEM_ERR_INVALID_ARG;
    int r = cache_status(*cache);
    if (r == SAEM_OK) r = batch_shape(*b);
    if (r != SAEM_OK) return r;
    if (!(c->scale > 0.f) || !isfinite(c->scale)) return SAEM_ERR_INVALID_ARG;
    if (c->q_heads < 1 || c->q_heads % cache->kv_heads || c->q_heads / cache->kv_heads > 128 || c->window < 0 || b->tokens > 0x7FFFFFFF / c->q_heads)
        return SAEM_ERR_SHAPE;
    if (b->tokens == 0 || b->seqs == 0) return SAEM_OK;
    r = batch_status(*b);
    if (r != SAEM_OK) return r;
    if (!q || !out || !workspace) return SAEM_ERR_INVALID_ARG;
    const int64_t strides[4] = {b->tokens > 1 ? c->q_token_stride : 0, c->q_heads > 1 ? c->q_head_stride : 0,
                                b->tokens > 1 ? c->out_token_stride : 0, c->q_heads > 1 ? c->out_head_stride : 0};
    if (strides[0] < 0 || strides[1] < 0 || !heads_apart(b->tokens, c->q_heads, cache->head_dim, c->out_token_stride, c->out_head_stride)) return SAEM_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)out) % 16 || (uintptr_t)lse % 4 || (uintptr_t)workspace % 1024) return SAEM_ERR_ALIGNMENT;
    for (int64_t s : strides)
        if (s % 8) return SAEM_ERR_ALIGNMENT;
    int n_sm;
    if (sm_count(&n_sm) != cudaSuccess || kRowsPerSm * n_sm > kAttendMaxCtas) return SAEM_ERR_CUDA;
    if (workspace_bytes < SAEM_ATTEND_HEAD_BYTES + partials_bytes(cache->head_dim, n_sm)) return SAEM_ERR_WORKSPACE;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    AttendArgs a = {};
    a.q = static_cast<const uint8_t*>(q); a.out = static_cast<uint8_t*>(out); a.lse = lse;
    a.q_ts = strides[0]; a.q_hs = strides[1]; a.out_ts = strides[2]; a.out_hs = strides[3];
    a.k = static_cast<const uint8_t*>(cache->k); a.v = static_cast<const uint8_t*>(cache->v);
    a.pages = cache->pages; a.page_size = cache->page_size; a.kv_heads = cache->kv_heads; a.dim = cache->head_dim;
    a.group = c->q_heads / cache->kv_heads;
    a.by_page = divisor_of(cache->page_size); a.by_group = divisor_of(a.group);
    a.offsets = b->offsets; a.lengths = b->lengths; a.table = b->table; a.table_stride = b->table_stride;
    a.seqs = b->seqs; a.tokens = b->tokens; a.max_pages = b->max_pages;
    a.causal = c->causal != 0; a.window = c->window; a.scale_log2 = c->scale * 1.4426950408889634f;
    a.status = reinterpret_cast<int*>(ws);
    a.counters = reinterpret_cast<int*>(ws + kAttendCounters);
    a.partials = reinterpret_cast<float*>(ws + SAEM_ATTEND_HEAD_BYTES);
    const bool f16 = cache->dtype == SAEM_OUT_F16, few = rows_are_few((long long)b->max_new * a.group, (long long)b->tokens * c->q_heads);
    const cudaError_t e = few ? launch_rows(a, f16, n_sm, (cudaStream_t)stream) : launch_attend_tiles(a, f16, n_sm, (cudaStream_t)stream);
    return e == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
}
