// Top-k gating (Background, "Mixture-of-Experts Inference": the router selects the top-k experts
// per token).  One warp per token; each lane keeps up to four logits in registers (experts lane,
// lane+32, ...); k rounds of a warp-wide arg-max by shuffles on a packed 64-bit key whose high
// word orders the logit and whose low word prefers the lower expert id; softmax over the k
// winners in registers.
#include "route_row.cuh"
#include "tc_common.cuh"

namespace saem {

constexpr int kRouteWarps = 4;

__global__ void __launch_bounds__(kRouteWarps * 32)
route_kernel(const float* __restrict__ logits, int T, int E, int k, int renorm, int32_t* __restrict__ idx,
             float* __restrict__ w) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int t = blockIdx.x * kRouteWarps + (threadIdx.x >> 5);
    if (t >= T) return;
    route_row(logits + (size_t)t * E, E, k, renorm, lane, idx + (size_t)t * k, w + (size_t)t * k);
}

// Router projection fused with the gate: a CTA (or a cluster of eight) per token computes logits[e] = <x_t, W_r[e]> in
// fp32 (16-byte loads of bf16, one warp per expert in turn, warp-shuffle reduction), keeps the
// row in shared memory and lets warp 0 run the same top-k / softmax.  Saves a launch and the
// logits' round trip through HBM on the latency-bound decode shapes.
constexpr int kRouterWarps = 8;

// SPLIT: the experts of a token are shared out over a cluster of that many CTAs, whose logits meet in the first one's
// shared memory (the same sums, so the same bits; 1 token, 128 experts, d 2048: 51 us with one CTA, 9 us with eight).
constexpr int kRouterSplit = 8;

template <int SPLIT>
__global__ void __launch_bounds__(kRouterWarps * 32)
route_fused_kernel(const uint16_t* __restrict__ x, const uint16_t* __restrict__ w_router, int T, int E, int d, int k,
                   int renorm, float* __restrict__ logits_out, int32_t* __restrict__ idx, float* __restrict__ w) {
    __shared__ float row[SAEM_MAX_EXPERTS];
    pdl_wait();
    pdl_launch_dependents();
    const int t = blockIdx.x / SPLIT, rank = blockIdx.x % SPLIT, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint4* xr = reinterpret_cast<const uint4*>(x + (size_t)t * d);
    if (SPLIT > 1) cluster_sync_all();                     // the first CTA is there
    for (int e = rank * kRouterWarps + warp; e < E; e += SPLIT * kRouterWarps) {
        const uint4* wr = reinterpret_cast<const uint4*>(w_router + (size_t)e * d);
        float acc = 0.f;
        for (int c = lane; c < d / 8; c += 32) {
            const uint4 a = xr[c], b = wr[c];
            const uint32_t av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc = fmaf(__uint_as_float(av[q] << 16), __uint_as_float(bv[q] << 16), acc);
                acc = fmaf(__uint_as_float(av[q] & 0xFFFF0000u), __uint_as_float(bv[q] & 0xFFFF0000u), acc);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
        if (lane == 0) {
            if (SPLIT > 1)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_u32(smem_u32(&row[e]), 0)), "f"(acc) : "memory");
            else
                row[e] = acc;
            if (logits_out) logits_out[(size_t)t * E + e] = acc;
        }
    }
    __syncthreads();
    if (SPLIT > 1) cluster_sync_all();
    if (rank == 0 && warp == 0) route_row(row, E, k, renorm, lane, idx + (size_t)t * k, w + (size_t)t * k);
}

cudaError_t launch_route(const float* logits, int T, int E, int k, int renorm, int32_t* idx, float* w,
                         cudaStream_t st) {
    int blocks = (T + kRouteWarps - 1) / kRouteWarps;
    return launch_pdl(route_kernel, dim3(blocks), dim3(kRouteWarps * 32), 0, st, logits, T, E, k, renorm, idx, w);
}

}  // namespace saem

namespace saem {
cudaError_t launch_route_fused(const uint16_t* x, const uint16_t* w_router, int T, int E, int d, int k, int renorm,
                               float* logits_out, int32_t* idx, float* w, cudaStream_t st) {
    // few tokens of many experts: one CTA per token would leave the SMs idle
    if (T > 16 || E < 4 * kRouterWarps)
        return launch_pdl(route_fused_kernel<1>, dim3(T), dim3(kRouterWarps * 32), 0, st, x, w_router, T, E, d, k, renorm, logits_out, idx, w);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kRouterSplit;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(T * kRouterSplit);
    cfg.blockDim = dim3(kRouterWarps * 32);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, route_fused_kernel<kRouterSplit>, x, w_router, T, E, d, k, renorm, logits_out, idx, w);
}
}  // namespace saem
