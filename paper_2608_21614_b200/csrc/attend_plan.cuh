// How the work of an attention call is dealt out, on the device alone: lengths, offsets and pages are never read on the host.
//
// An item is a tile of R rows of one sequence and one key head (row = token * group + query head within the group); its units are the
// tiles of KEYS places that any of its rows may see, one at least, so that rows that see nothing are written too, behind HEAD units
// for what an item costs by itself (queries, first bytes, the result).  All units of a call, in the order sequence, key head, row
// tile, are cut into as many equal ranges as there are CTAs: long and short sequences, few and many rows load the SMs alike.  A cut
// within an item's first HEAD units moves to its beginning, and one within SNAP units (or a third of a range, if that is less) of either
// end of an item moves there, because a cut costs about as much; an item of up to 2 HEAD units is not cut at all.  An item that is still
// cut leaves sums of its parts in the workspace, and the CTA that arrives last adds them up in the order of the parts, so that two runs
// give the same bits.
#ifndef SAEM_ATTEND_PLAN_CUH_
#define SAEM_ATTEND_PLAN_CUH_

#include <limits.h>

#include "attend_common.cuh"

namespace saem {

constexpr int kAttendMaxCtas = 640;         // SMs x CTAs per SM at most

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Weights are multiplied by 2^LIFT before they are rounded to float16, and so is their sum: the largest is then close to 65504 and the last bit
// of a small one is 2^-24 of that, not of 1.  Without it small weights beside a large one of the same CTA came out 4 % off (2^-20.6) or not at all (2^-25.2).
template <int LIFT>
__device__ __forceinline__ float log_sum_exp(float top, float sum) {           // top in powers of two
    return top == -INFINITY ? -INFINITY : top * 0.69314718056f + logf(sum * (1.f / (1 << LIFT)));
}

struct AttendArgs {
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    long long q_ts, q_hs, out_ts, out_hs;   // strides in elements
    const uint8_t* k;
    const uint8_t* v;
    long long pages;
    int page_size, kv_heads, dim, group;
    Divisor by_page, by_group, by_ctas;     // by_ctas: the grid's
    const int32_t* offsets;
    const int32_t* lengths;
    const int32_t* table;
    long long table_stride;
    int seqs, tokens, max_pages;
    int causal, window;
    float scale_log2;                       // scale * log2(e)
    int* status;
    int* counters;                          // [kAttendMaxCtas], zero between calls
    float* partials;                        // two slots per CTA
};
// The form for many rows per key head (attend_tiles.cu), and the bytes that its partial results take.
cudaError_t launch_attend_tiles(const AttendArgs& a, bool f16, int n_sm, cudaStream_t st);
size_t attend_tiles_partials(int dim, int n_sm);
constexpr size_t kAttendCounters = 256;     // byte offset of the counters in the workspace
static_assert(kAttendCounters + 4 * kAttendMaxCtas <= SAEM_ATTEND_HEAD_BYTES, "");

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
struct SeqExtent {
    int first, n;                           // first row of the call's tokens, new tokens
    int len, before;                        // places that can be read, which the table cuts; place of the first new token (may be negative), which it does not
    __device__ __forceinline__ bool cut() const { return before + n > len; }                // a token's own place is not in the table
};
__device__ __forceinline__ SeqExtent seq_extent(const AttendArgs& a, int s) {
    const int end = a.offsets[s + 1], lo = min(max(a.offsets[s], 0), a.tokens), hi = min(max(end, lo), a.tokens), length = max(a.lengths[s], 0);
    const long long most = min((long long)a.max_pages * a.page_size, 0x7FFF0000ll);      // sums of places stay within 32 bits
    return {lo, hi - lo, (int)min((long long)length, most), hi > lo ? length - (end - lo) : 0};
}
// The places that rows [row0, row1] may see, in tiles of KEYS.
template <int KEYS>
__device__ __forceinline__ void key_tiles(const AttendArgs& a, const SeqExtent& e, int row0, int row1, int& begin, int& end) {
    const int stop = a.causal ? min(e.before + quotient(row1, a.by_group) + 1, e.len) : e.len;
    const int first = e.before + quotient(row0, a.by_group) + 1, start = a.window && first > a.window ? first - a.window : 0;
    begin = start / KEYS;
    end = stop > start ? (stop - 1) / KEYS + 1 : begin;
}
template <int R>
__device__ __forceinline__ int row_tiles(const AttendArgs& a, const SeqExtent& e) { return (int)(((uint32_t)(e.n * a.group) + (R - 1)) / R); }
template <int R, int KEYS, int HEAD>
__device__ __forceinline__ int item_units(const AttendArgs& a, const SeqExtent& e, int r) {
    int b, t;
    const int rows = e.n * a.group;
    key_tiles<KEYS>(a, e, r * R, min(rows - r * R, R) + r * R - 1, b, t);
    return HEAD + max(1, t - b);
}

// x / d where the quotient is below 2^20: an estimate in fp32, off by one at most, and a look at the rest.
__device__ __forceinline__ int small_quotient(long long x, long long d) {
    int q = (int)__fdividef((float)x, (float)d);
    const long long rest = x - q * d;
    return rest < 0 ? q - 1 : rest >= d ? q + 1 : q;
}
// The units of a range, LEAST at least.
template <int LEAST>
__device__ __forceinline__ long long range_units(const AttendArgs& a, long long total) {
    const long long per = total < 0x7FFF0000 ? (long long)quotient((int)total + a.by_ctas.d - 1, a.by_ctas) : (total + gridDim.x - 1) / gridDim.x;
    return max(per, (long long)LEAST);
}
// Units of one key head of the sequence that the lane holds (all lanes of a warp; the row tiles of a sequence with more than one are shared
// out over the warp).
template <int R, int KEYS, int HEAD>
__device__ __forceinline__ long long head_units(const AttendArgs& a, const SeqExtent& e, int lane) {
    const int tiles = row_tiles<R>(a, e);
    long long u = tiles == 1 ? item_units<R, KEYS, HEAD>(a, e, 0) : 0;
    for (uint32_t many = __ballot_sync(0xffffffffu, tiles > 1); many; many &= many - 1) {
        const int src = __ffs(many) - 1;
        const SeqExtent o = {0, __shfl_sync(0xffffffffu, e.n, src), __shfl_sync(0xffffffffu, e.len, src), __shfl_sync(0xffffffffu, e.before, src)};
        const int t = __shfl_sync(0xffffffffu, tiles, src);
        long long sum = 0;
        for (int r = lane; r < t; r += 32) sum += item_units<R, KEYS, HEAD>(a, o, r);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == src) u = sum;
    }
    return u;
}
template <class T>
__device__ __forceinline__ T inclusive_sum(T v, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T o = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += o;
    }
    return v;
}

constexpr int kPlanWarpSeqs = 32;           // so many sequences are planned by each warp for itself (AttendWalk::begin_alone)
struct AttendPlan {                         // in shared memory
    long long per;                          // units of a range
    long long begin, seq_begin, per_head;   // first unit of this CTA's range, that of the sequence s that it lies in, units of one of its heads
    int s;                                  // seqs: the CTA has no range
    long long scan[12];                     // a warp each
};

// For more sequences than that: all threads of the CTA (WARPS whole warps).
template <int R, int KEYS, int HEAD, int LEAST, int WARPS>
__device__ __forceinline__ void make_plan(const AttendArgs& a, AttendPlan& p) {
    static_assert(WARPS <= 12, "");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int kStep = WARPS * 32;
    auto units_of = [&](int s) { return head_units<R, KEYS, HEAD>(a, s < a.seqs ? seq_extent(a, s) : SeqExtent{}, lane) * a.kv_heads; };
    if (threadIdx.x == 0) p.s = a.seqs;
    long long mine = units_of(warp * 32 + lane), incl = inclusive_sum(mine, lane), sum = __shfl_sync(0xffffffffu, incl, 31);
    for (int s = kStep + warp * 32; s < a.seqs; s += kStep) sum += __shfl_sync(0xffffffffu, inclusive_sum(units_of(s + lane), lane), 31);
    if (lane == 0) p.scan[warp] = sum;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) total += p.scan[w];
    const long long per = range_units<LEAST>(a, total), begin = per * blockIdx.x;
    if (begin >= total) return;
    long long before = 0;
    for (int s0 = 0; before <= begin; s0 += kStep) {
        if (a.seqs > kStep) {               // the sums are not those of this step's sequences
            if (s0) incl = inclusive_sum(mine = units_of(s0 + warp * 32 + lane), lane);
            __syncthreads();
            if (lane == 31) p.scan[warp] = incl;
            __syncthreads();
        }
        long long base = before;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) base += p.scan[w];
            before += p.scan[w];
        }
        if (base + incl - mine <= begin && begin < base + incl) { p.per = per; p.begin = begin; p.seq_begin = base + incl - mine; p.per_head = mine / a.kv_heads; p.s = s0 + warp * 32 + lane; }
    }
    __syncthreads();
}

// A part of an item: what one CTA does of it between two looks at the plan.
struct AttendPart {
    SeqExtent e;
    int s, h, r;
    int rows;                               // of the tile
    int key_begin, key_end;                 // tiles of KEYS places; none where the rows see nothing
    bool whole;                             // the item is not cut
    int first_cta, n_parts, slot;           // where it is: the CTA of its first part, the parts, and this one's place in the workspace
};
// The places in the workspace: a CTA has at most two parts of cut items, one that begins its item and one that does not.
__device__ __forceinline__ int part_slot(int first_cta, int j) { return 2 * (first_cta + j) + (j == 0 ? 1 : 0); }

// Walks through a CTA's range; every warp for itself, alike in all lanes.
template <int R, int KEYS, int HEAD, int SNAP>
struct AttendWalk {
    long long item, per;                    // first unit of the item at hand; units of a range
    int snap, low;
    int s, h, r, tiles;
    SeqExtent e;
    __device__ __forceinline__ void begin(const AttendArgs& a, const AttendPlan& p) {
        s = p.s;
        if (s >= a.seqs) return;
        per = p.per;
        e = seq_extent(a, s);
        find(a, p.begin, p.seq_begin, p.per_head);
    }
    // Up to kPlanWarpSeqs sequences, a lane each: the plan without shared memory or barriers (it is what a short call waits for first).
    template <int LEAST>
    __device__ __forceinline__ void begin_alone(const AttendArgs& a) {
        const int lane = threadIdx.x & 31;
        const SeqExtent mine = lane < a.seqs ? seq_extent(a, lane) : SeqExtent{};
        const long long per_head = head_units<R, KEYS, HEAD>(a, mine, lane), units = per_head * a.kv_heads;
        // sums of 32 of them fit into 32 bits, but for uncommon calls
        const long long incl = __any_sync(0xffffffffu, units >> 26) ? inclusive_sum(units, lane) : (long long)inclusive_sum((uint32_t)units, lane);
        const long long total = __shfl_sync(0xffffffffu, incl, 31);
        per = range_units<LEAST>(a, total);
        const long long at = per * blockIdx.x;
        const uint32_t past = __ballot_sync(0xffffffffu, incl > at);
        s = a.seqs;
        if (!past) return;
        s = __ffs(past) - 1;
        e.first = __shfl_sync(0xffffffffu, mine.first, s);
        e.n = __shfl_sync(0xffffffffu, mine.n, s);
        e.len = __shfl_sync(0xffffffffu, mine.len, s);
        e.before = __shfl_sync(0xffffffffu, mine.before, s);
        find(a, at, __shfl_sync(0xffffffffu, incl - units, s), __shfl_sync(0xffffffffu, per_head, s));
    }
    // The item of sequence s that holds unit `at`: the head by division, the row tile by a warp's scan.
    __device__ __forceinline__ void find(const AttendArgs& a, long long at, long long seq_begin, long long per_head) {
        snap = per < 3 * SNAP ? (int)per / 3 : SNAP;
        low = max(HEAD, snap);
        tiles = row_tiles<R>(a, e);
        r = 0;
        h = small_quotient(at - seq_begin, per_head);
        item = seq_begin + h * per_head;
        if (tiles == 1) return;
        const int lane = threadIdx.x & 31;
        for (int t0 = 0; t0 < tiles; t0 += 32) {
            // 32 tiles of 16 rows over 2^31 - 2^16 places have fewer than 2^32 units
            const uint32_t u = t0 + lane < tiles ? item_units<R, KEYS, HEAD>(a, e, t0 + lane) : 0, incl = inclusive_sum(u, lane);
            const uint32_t past = __ballot_sync(0xffffffffu, item + incl > at);
            if (past) {
                const int l = __ffs(past) - 1;
                r = t0 + l;
                item += __shfl_sync(0xffffffffu, incl - u, l);
                break;
            }
            item += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    __device__ __forceinline__ bool next(const AttendArgs& a, AttendPart& p) {
        const int me = blockIdx.x;
        while (s < a.seqs) {
            const int row0 = r * R, row1 = row0 + min(e.n * a.group - row0, R) - 1;
            int b, t;
            key_tiles<KEYS>(a, e, row0, row1, b, t);
            const int units = HEAD + max(1, t - b);
            // its parts begin with the item and at the cuts between item + low and item + units - snap
            const int first = small_quotient(item + min(low, units - 1), per), last = units <= 2 * HEAD ? first : max(first, small_quotient(item + units - snap - 1, per));
            if (first > me) return false;
            const bool mine = me <= last;
            if (mine) {
                p.e = e; p.s = s; p.h = h; p.r = r;
                p.rows = row1 - row0 + 1;
                p.key_begin = me == first ? b : b + (int)(per * me - item) - HEAD;
                p.key_end = me == last ? t : b + (int)(per * (me + 1) - item) - HEAD;
                p.whole = first == last;
                p.first_cta = first;
                p.n_parts = last - first + 1;
                p.slot = part_slot(first, me - first);
                if (me < last) { s = a.seqs; return true; }
            }
            item += units;
            if (++r == tiles) {
                r = 0;
                if (++h == a.kv_heads) {
                    h = 0;
                    do e.n = 0;
                    while (++s < a.seqs && (e = seq_extent(a, s)).n == 0);
                    tiles = row_tiles<R>(a, e);
                }
            }
            if (mine) return true;
        }
        return false;
    }
};

// The rows' bounds: row (of the item) sees places lo .. hi.
__device__ __forceinline__ void row_bounds(const AttendArgs& a, const SeqExtent& e, int row, bool in, int& lo, int& hi) {
    const int place = e.before + quotient(row, a.by_group);
    hi = !in ? -1 : a.causal ? min(place, e.len - 1) : e.len - 1;
    lo = a.window && place + 1 > a.window ? place + 1 - a.window : 0;
}

// Rows with a NaN, once more.  In a product of tiles a weight of 0 meets what other rows see, and 0 times an infinity or NaN there is NaN; so it
// is with float16 weights where a row sees an infinity itself and its weight rounds to 0.  The first comes of the few places of an item's tiles that
// some of its rows do not see, the second of any; a NaN that a row sees is one of its result and needs no second sum.  One token over 131072
// places, one with a NaN: 99 us as without (bfloat16), 1.5 ms (float16, where all values are looked at); a row that is summed again takes 1.5 us for 16 places.
constexpr int kAgain = 16;                  // places at a time: of one page, as they are multiples of 16
constexpr int kAgainMarks = 4 * kHeadDimMax;
__device__ __forceinline__ int again_page(const AttendArgs& a, int s, int j0) { return a.table[s * a.table_stride + quotient(j0, a.by_page)]; }
// The lane's four columns of kAgain places from j0 on (zeros of a page outside the cache): all of a page may be read, whatever it holds.
__device__ __forceinline__ void again_load(const AttendArgs& a, const uint8_t* cache, int page, int h, int j0, int at, uint2 (&w)[kAgain]) {
#pragma unroll
    for (int i = 0; i < kAgain; ++i) w[i] = make_uint2(0, 0);
    if (at < a.dim && page >= 0 && page < a.pages) {
        const uint8_t* p = cache + ((((long long)page * a.kv_heads + h) * a.page_size + j0 - quotient(j0, a.by_page) * a.page_size) * a.dim + at) * 2;
#pragma unroll
        for (int i = 0; i < kAgain; ++i) w[i] = *reinterpret_cast<const uint2*>(p + i * a.dim * 2);
    }
}

// One row, by one warp, out of the cache and the places that it sees alone; of its results those are written whose bit is set in `need` (of the
// lane's four columns).
template <bool F16>
__device__ __noinline__ void attend_row_again(const AttendArgs& a, const SeqExtent& e, int s, int h, int row, uint32_t need) {
    const int lane = threadIdx.x & 31, at = lane * 4;
    const bool here = at < a.dim;
    int lo, hi;
    row_bounds(a, e, row, true, lo, hi);
    const long long token = e.first + row / a.group;
    const int head = h * a.group + row % a.group;
    float q[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    auto four = [&](uint2 w, float* v) {
        const float2 x = unpack2<F16>(w.x), y = unpack2<F16>(w.y);
        v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
    };
    if (here) four(*reinterpret_cast<const uint2*>(a.q + (token * a.q_ts + head * a.q_hs + at) * 2), q);
    int j0 = lo & ~(kAgain - 1), page = j0 <= hi ? again_page(a, s, j0) : -1;
    for (; j0 <= hi; j0 += kAgain) {
        uint2 kw[kAgain], vw[kAgain];
        float d[kAgain];
        again_load(a, a.k, page, h, j0, at, kw);
        again_load(a, a.v, page, h, j0, at, vw);
        if (j0 + kAgain <= hi) page = again_page(a, s, j0 + kAgain);
#pragma unroll
        for (int i = 0; i < kAgain; ++i)    // what the row does not see is anything
            if (j0 + i < lo || j0 + i > hi) vw[i] = make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < kAgain; ++i) {
            float x[4];
            four(kw[i], x);
            d[i] = q[0] * x[0] + q[1] * x[1] + q[2] * x[2] + q[3] * x[3];
        }
        // sums over the warp, halving the places that a lane has: lanes 2i and 2i + 1 end with place i's
#pragma unroll
        for (int n = kAgain / 2; n > 0; n /= 2) {
            const bool upper = lane & 2 * n;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float give = upper ? d[i] : d[i + n];
                d[i] = (upper ? d[i + n] : d[i]) + __shfl_xor_sync(0xffffffffu, give, 2 * n);
            }
        }
        d[0] += __shfl_xor_sync(0xffffffffu, d[0], 1);
        const int mine = j0 + (lane >> 1);
        const float x = mine >= lo && mine <= hi ? d[0] * a.scale_log2 : -INFINITY;
        if (__any_sync(0xffffffffu, x != x || x == INFINITY)) {                 // so is the whole row
            l = NAN;
            break;
        }
        float top = fmaxf(m, x);
#pragma unroll
        for (int d = 2; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float base = top == -INFINITY ? 0.f : top, was = fast_exp2(m - base), p = fast_exp2(x - base);
        m = top;
        l = l * was + (lane & 1 ? 0.f : p);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= was;
#pragma unroll
        for (int i = 0; i < kAgain; ++i) {
            const float w = __shfl_sync(0xffffffffu, p, 2 * i);
            float x[4];
            four(vw[i], x);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(w, x[c], o[c]);
        }
        bool open = false;                  // columns that are not NaN for good
#pragma unroll
        for (int c = 0; c < 4; ++c) open |= (need >> c & 1) && o[c] == o[c];
        if (!__any_sync(0xffffffffu, open)) break;
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    uint16_t* const to = reinterpret_cast<uint16_t*>(a.out) + token * a.out_ts + head * a.out_hs + at;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (need >> c & 1) to[c] = (uint16_t)pack2<F16>(o[c] * inv, 0.f);
}

// The rows row0 .. row0 + rows - 1 of an item whose results are written, by WARPS warps that meet at the barrier BAR; marks: kAgainMarks ints in
// shared memory, free for it.
template <bool F16, int KEYS, int WARPS, int BAR>
__device__ __noinline__ void attend_again(const AttendArgs& a, const SeqExtent& e, int s, int h, int row0, int rows, int* marks, int warp) {
    constexpr int kThreads = WARPS * 32;
    const int lane = threadIdx.x & 31, at = lane * 4;
    int* const nan_first = marks, *const nan_last = marks + kHeadDimMax, *const inf_first = marks + 2 * kHeadDimMax, *const inf_last = marks + 3 * kHeadDimMax;
    for (int i = warp * 32 + lane; i < kAgainMarks; i += kThreads) marks[i] = i & kHeadDimMax ? -1 : INT_MAX;
    named_sync(BAR, kThreads);
    // ---- of each column, the first and the last place with a NaN and with an infinity
    constexpr uint32_t kExp = F16 ? 0x7C00u : 0x7F80u, kUnit = F16 ? 0x0400u : 0x0080u;
    int b, t, lo, hi, lo_last, hi_first;
    key_tiles<KEYS>(a, e, row0, row0 + rows - 1, b, t);
    row_bounds(a, e, row0, true, lo, hi_first);
    row_bounds(a, e, row0 + rows - 1, true, lo_last, hi);
    const int begin = b * KEYS, end = min(t * KEYS, e.len);
    auto look = [&](int from, int to) {
        constexpr int kGroups = 4, kStep = WARPS * kAgain;          // groups of places whose loads are under way
        int pages = -1;                     // lane l: of the l-th of 32 groups
        for (int j0 = (from & ~(kAgain - 1)) + warp * kAgain, n = 0; j0 < to; j0 += kGroups * kStep, n += kGroups) {
            uint2 w[kGroups][kAgain];
            uint32_t found = 0;
            if (n % 32 == 0) pages = (long long)j0 + lane * kStep < to ? again_page(a, s, j0 + lane * kStep) : -1;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) again_load(a, a.v, __shfl_sync(0xffffffffu, pages, (n + g) % 32), h, j0 + g * kStep, at, w[g]);
#pragma unroll
            for (int i = 0; i < kGroups * kAgain; ++i) {
                const uint2 x = w[i / kAgain][i % kAgain];
                found |= ((x.x & kExp * 0x10001u) + kUnit * 0x10001u) | ((x.y & kExp * 0x10001u) + kUnit * 0x10001u);
            }
            if (!(found & 0x80008000u)) continue;
#pragma unroll
            for (int i = 0; i < kGroups * kAgain; ++i) {
                const uint2 x = w[i / kAgain][i % kAgain];
                const int j = j0 + i / kAgain * kStep + i % kAgain;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t y = (c < 2 ? x.x : x.y) >> (c & 1) * 16 & 0x7FFFu;
                    if (y >= kExp && j < end) {
                        atomicMin((y > kExp ? nan_first : inf_first) + at + c, j);
                        atomicMax((y > kExp ? nan_last : inf_last) + at + c, j);
                    }
                }
            }
        }
    };
    if (F16) look(begin, end);
    else {                                  // all rows see the places lo_last .. hi_first
        look(begin, min(lo_last, end));
        look(max(hi_first + 1, begin), end);
    }
    named_sync(BAR, kThreads);
    for (int r = warp; r < rows; r += WARPS) {
        row_bounds(a, e, row0 + r, true, lo, hi);
        const int i = quotient(row0 + r, a.by_group), head = h * a.group + row0 + r - i * a.group;
        uint2 x = make_uint2(0, 0);
        if (at < a.dim) x = *reinterpret_cast<const uint2*>(a.out + ((e.first + i) * a.out_ts + head * a.out_hs + at) * 2);
        uint32_t need = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t y = (c < 2 ? x.x : x.y) >> (c & 1) * 16 & 0x7FFFu;
            if (y <= kExp) continue;
            const int n0 = nan_first[at + c], n1 = nan_last[at + c], i0 = inf_first[at + c], i1 = inf_last[at + c];
            const bool unseen = min(n0, i0) < lo || max(n1, i1) > hi, lost = F16 && i0 <= hi && i1 >= lo;
            const bool own = (n0 >= lo && n0 <= hi) || (n1 >= lo && n1 <= hi);
            if ((unseen || lost) && !own) need |= 1u << c;
        }
        if (__any_sync(0xffffffffu, need != 0)) attend_row_again<F16>(a, e, s, h, row0 + r, need);
    }
    named_sync(BAR, kThreads);
}

}  // namespace saem

#endif  // SAEM_ATTEND_PLAN_CUH_
