// The expert FFN over microscaled 4-bit experts (SAEM_FFN_MX contexts): h = silu(Wg x) * (Wu x), y = Wd h with the
// weights read as MXFP4 units (mx_common.cuh) straight from their slots into registers.
//
// A decode batch reads every active expert's bytes once, so the bound is DRAM; the arithmetic has to keep up with
// 46 codes per cycle and SM.  A unit (16 weight rows x 128 elements) is two 16-byte loads and two scale words per lane;
// eight codes become four f16 pairs with one cvt each (E2M1 is exact in f16), two mma.sync.m16n8k16 multiply a block of
// 32 elements, and the block's scale, different in every row, multiplies the fp32 partial sums of the block -- four
// FMAs for 512 codes.  The activations are the MMA's B operand in f16, each 128-element span of a row brought to
// [2^14, 2^15) by a power of two that is multiplied back in fp32: bf16 values stay exact unless they are 2^-28 of the
// span's largest; the hidden activations, kept in fp32 between the two launches, are rounded to 11 bits here and
// nowhere else.
#include "mx_common.cuh"
#include "tc_common.cuh"

namespace saem {

constexpr int kMoeWarps = 8;
constexpr int kMoeChunk = 512;              // elements of k staged at a time
constexpr int kMoeSpans = kMoeChunk / kMxSpan;
constexpr int kMoePitch = kMoeChunk + 32;   // f16 elements between staged rows: 64 bytes off a multiple of 128, so that the
                                            // eight rows x 64 bytes of a fragment load fall into different banks

struct MoeArgs {
    const void* x;              // gate/up: bf16 [rows, d]; down: fp32 h [rows, f]
    const int32_t* offsets;     // [E + 1], or nullptr: one segment [0, max_rows)
    int max_rows, E, d, f;
    const uint8_t* slot_region;
    size_t slot_bytes;
    float* out;                 // gate/up: h [rows, f]; down: y [rows, d]
    int* status;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct MxUnit {                 // one lane's part of a unit
    uint4 q0, q1;               // codes of rows g and g + 8
    uint32_t s0, s1;            // their scales
};
__device__ __forceinline__ void load_unit(MxUnit& u, const uint8_t* p, int lane) {
    u.q0 = __ldcs(reinterpret_cast<const uint4*>(p) + lane);
    u.q1 = __ldcs(reinterpret_cast<const uint4*>(p + 512) + lane);
    u.s0 = __ldcs(reinterpret_cast<const uint32_t*>(p + kMxUnitScales) + (lane >> 2));
    u.s1 = __ldcs(reinterpret_cast<const uint32_t*>(p + kMxUnitScales + 32) + (lane >> 2));
}

// acc[j] += unit x (8 activation rows j): `xs` is the span's f16 activations in shared memory (row pitch kMoePitch),
// `xf` the rows' factors for this span.
template <int NT>
__device__ __forceinline__ void unit_mma(const MxUnit& u, const __half* xs, const float* xf, int lane, int nt, float (&acc)[NT][4]) {
    const int g = lane >> 2, t = lane & 3;
    const uint32_t q0[4] = {u.q0.x, u.q0.y, u.q0.z, u.q0.w}, q1[4] = {u.q1.x, u.q1.y, u.q1.z, u.q1.w};
    float s0[4], s1[4];
    mx_scales4(u.s0, s0);
    mx_scales4(u.s1, s1);
    float part[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[j][i] = 0.f;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        uint32_t a[4], c[4];
        mx_decode8(q0[b], a);
        mx_decode8(q1[b], c);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (j >= nt) break;
            const uint4 x = *reinterpret_cast<const uint4*>(xs + (size_t)(8 * j + g) * kMoePitch + b * kMxBlock + 8 * t);
            float m[4] = {0.f, 0.f, 0.f, 0.f};
            mma_f16(m, a[0], c[0], a[1], c[1], x.x, x.y);
            mma_f16(m, a[2], c[2], a[3], c[3], x.z, x.w);
            part[j][0] += s0[b] * m[0];
            part[j][1] += s0[b] * m[1];
            part[j][2] += s1[b] * m[2];
            part[j][3] += s1[b] * m[3];
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if (j >= nt) break;
        const float2 f = *reinterpret_cast<const float2*>(xf + 8 * j + 2 * t);
        acc[j][0] += f.x * part[j][0];
        acc[j][1] += f.y * part[j][1];
        acc[j][2] += f.x * part[j][2];
        acc[j][3] += f.y * part[j][3];
    }
}

// One warp brings 128 elements of a row to f16: power of two from the largest magnitude (as an integer comparison of
// the bits), the reciprocal factor to *factor.  A span with an infinity or NaN keeps its values (factor 1): every
// output of that row is then not finite either.
__device__ __forceinline__ void stage_span(const float (&v)[4], __half* dst, float* factor, int lane) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = __reduce_max_sync(0xffffffffu, m);
    int e = (int)(m >> 23);                                  // biased exponent of the largest
    e = e == 255 ? 127 + 14 : max(e, 15);                    // both 2^(141 - e) and 2^(e - 141) are normal numbers
    const float up = __uint_as_float((uint32_t)(127 + 141 - e) << 23);
    const __half2 lo = __floats2half2_rn(v[0] * up, v[1] * up), hi = __floats2half2_rn(v[2] * up, v[3] * up);
    uint2 w;
    w.x = *reinterpret_cast<const uint32_t*>(&lo);
    w.y = *reinterpret_cast<const uint32_t*>(&hi);
    *reinterpret_cast<uint2*>(dst + 4 * lane) = w;
    if (lane == 0) *factor = __uint_as_float((uint32_t)(e - 14) << 23);
}

// MODE 0: gate/up (rows of x -> h), MODE 1: down (h -> y).  A CTA takes items of (expert, 8 * NT rows, 8 groups of 16
// weight rows); each warp streams the units of its own group along k, the activations are staged for all of them.
template <int MODE, int NT>
__global__ void __launch_bounds__(kMoeWarps * 32)
mx_ffn_kernel(const __grid_constant__ MoeArgs a, const __grid_constant__ SlotTable tab) {
    extern __shared__ __align__(16) uint8_t smem[];
    __half* xs = reinterpret_cast<__half*>(smem);                              // [8 NT][kMoePitch]
    float* xf = reinterpret_cast<float*>(smem + (size_t)8 * NT * kMoePitch * 2);   // [kMoeSpans][8 NT]
    __shared__ int first[SAEM_MAX_EXPERTS + 1], start[SAEM_MAX_EXPERTS], rows_of[SAEM_MAX_EXPERTS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int K = MODE == 0 ? a.d : a.f, n_span = K / kMxSpan;
    const int groups = MODE == 0 ? a.f / 8 : a.d / 16, n_gb = groups / kMoeWarps;   // d, f are multiples of 128
    pdl_wait();
    pdl_launch_dependents();
    for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
        int lo = a.offsets ? a.offsets[e] : 0, hi = a.offsets ? a.offsets[e + 1] : a.max_rows;
        lo = min(max(lo, 0), a.max_rows);
        hi = min(max(hi, lo), a.max_rows);
        int n = hi - lo;
        if (n > 0 && tab.slot[e] < 0) {
            if (tab.in_subset[e] && MODE == 0 && blockIdx.x == 0) atomicExch(a.status, SAEM_ERR_NOT_RESIDENT);
            n = 0;
        }
        start[e] = lo;
        rows_of[e] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int s = 0;
        for (int e = 0; e < a.E; ++e) {
            first[e] = s;
            s += (rows_of[e] + 8 * NT - 1) / (8 * NT) * n_gb;
        }
        first[a.E] = s;
    }
    __syncthreads();
    const int total = first[a.E];
    for (int item = blockIdx.x; item < total; item += gridDim.x) {
        int e = 0;
        for (int step = 64; step > 0; step >>= 1)                              // the last e with first[e] <= item
            if (e + step < a.E && first[e + step] <= item) e += step;
        const int tiles = (rows_of[e] + 8 * NT - 1) / (8 * NT), rem = item - first[e];
        const int gb = rem / tiles, tile = rem % tiles;
        const int row0 = start[e] + tile * 8 * NT, rows = min(8 * NT, rows_of[e] - tile * 8 * NT);
        const int nt = (rows + 7) / 8;
        const int group = gb * kMoeWarps + warp;
        const uint8_t* w = a.slot_region + (size_t)tab.slot[e] * a.slot_bytes +
                           ((MODE == 0 ? 0 : mx_gate_up_units(a.d, a.f)) + (size_t)group * n_span) * kMxUnitBytes;
        float acc[NT][4];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
        for (int s0 = 0; s0 < n_span; s0 += kMoeSpans) {
            const int spans = min(kMoeSpans, n_span - s0);
            MxUnit u[kMoeSpans];
#pragma unroll
            for (int s = 0; s < kMoeSpans; ++s)
                if (s < spans) load_unit(u[s], w + (size_t)(s0 + s) * kMxUnitBytes, lane);
            __syncthreads();                                                   // the previous chunk has been read
            for (int i = warp; i < nt * 8 * spans; i += kMoeWarps) {
                const int r = i / spans, s = i % spans;
                float v[4] = {0.f, 0.f, 0.f, 0.f};
                if (r < rows) {
                    const size_t at = (size_t)(row0 + r) * K + (s0 + s) * kMxSpan + 4 * lane;
                    if (MODE == 0) {
                        const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.x) + at);
                        v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
                        v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
                    } else {
                        const float4 q = *reinterpret_cast<const float4*>(static_cast<const float*>(a.x) + at);
                        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
                    }
                }
                stage_span(v, xs + (size_t)r * kMoePitch + s * kMxSpan, xf + s * 8 * NT + r, lane);
            }
            __syncthreads();
#pragma unroll
            for (int s = 0; s < kMoeSpans; ++s)
                if (s < spans) unit_mma<NT>(u[s], xs + s * kMxSpan, xf + s * 8 * NT, lane, nt, acc);
        }
        // lane (g, t): rows g and g + 8 of the group, activation rows 8 j + 2 t and + 1
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 8 * j + 2 * t + i;
                if (r >= rows) continue;
                if (MODE == 0) {
                    const float z = acc[j][i], up = acc[j][i + 2];
                    a.out[(size_t)(row0 + r) * a.f + group * 8 + g] = z / (1.f + expf(-z)) * up;
                } else {
                    float* o = a.out + (size_t)(row0 + r) * a.d + group * 16 + g;
                    o[0] = acc[j][i];
                    o[8] = acc[j][i + 2];
                }
            }
    }
}

template <int MODE, int NT>
static cudaError_t launch_one(const MoeArgs& a, const SlotTable& tab, long long items, int n_sm, cudaStream_t st) {
    static bool done[64];
    const size_t smem = (size_t)8 * NT * kMoePitch * 2 + (size_t)kMoeSpans * 8 * NT * 4;
    if (first_call_on_device(done)) {
        const cudaError_t e = cudaFuncSetAttribute(mx_ffn_kernel<MODE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    const long long most = (long long)n_sm * (NT <= 2 ? 4 : 2);
    return launch_pdl(mx_ffn_kernel<MODE, NT>, dim3((unsigned)(items < most ? items : most)), dim3(kMoeWarps * 32), smem, st, a, tab);
}

cudaError_t launch_mx_ffn(const FfnArgs& f, const SlotTable& tab, int max_segment, cudaStream_t st, int* n_launch) {
    MoeArgs a = {f.x_packed, f.offsets, f.max_rows, f.E, f.d, f.f, f.slot_region, f.slot_bytes, reinterpret_cast<float*>(f.h), f.status};
    MoeArgs b = a;
    b.x = f.h;
    b.out = f.y_packed;
    const int nt = max_segment <= 8 ? 1 : max_segment <= 16 ? 2 : max_segment <= 32 ? 4 : 8;
    const long long tiles = f.max_active + f.max_rows / (8 * nt);             // an upper bound of the row tiles
    const long long ia = tiles * (f.f / 64), ib = tiles * (f.d / 128);
    cudaError_t e;
#define SAEM_MX_NT(NT_)                                                                       \
    e = launch_one<0, NT_>(a, tab, ia, f.n_sm, st);                                           \
    if (e == cudaSuccess) e = launch_one<1, NT_>(b, tab, ib, f.n_sm, st)
    if (nt == 1) { SAEM_MX_NT(1); }
    else if (nt == 2) { SAEM_MX_NT(2); }
    else if (nt == 4) { SAEM_MX_NT(4); }
    else { SAEM_MX_NT(8); }
#undef SAEM_MX_NT
    if (e == cudaSuccess) *n_launch += 2;
    return e;
}

}  // namespace saem
