// Product of two MXFP4 matrices on the block-scaled tensor cores: out[m, n] = sum_k A[m, k] W[n, k].
//
// tcgen05.mma kind::mxf4 multiplies E2M1 operands out of shared memory, takes the scale of every 32 elements from
// tensor memory and accumulates in fp32 (an E2M1 product times a power of two is exact; the sum's rounding is the only
// one before the output's).  The weights' rows are the MMA's M (128 lanes of tensor memory), the tokens its N (16..256
// columns), so that one instruction shape serves one token and thousands, and a warp's stores of the result are
// consecutive n.  A stage is 256 elements of k: 128-byte rows of codes under the 128-byte swizzle (TMA) and the scales'
// 512-byte pieces (plain bulk copies, moved to tensor memory by tcgen05.cp as they are).
//
// Few tokens: the weights' bytes are the bound, and n / 128 tiles are too few for the SMs.  The k range is then split
// over a cluster of 2, 4 or 8 CTAs, whose partial sums meet in distributed shared memory in a fixed order (two runs give
// the same bits; no workspace, no second launch).
#include "mx_tc.cuh"

namespace saem {

constexpr int kMmThreads = 192;             // warp 0: copies, warp 1: MMA issue, warps 2-5: epilogue
constexpr int kMmStageK = 256;              // elements of k per stage (128 bytes of codes)
constexpr int kMmMaxStages = 12;
constexpr int kMmSmem = 226 * 1024;         // dynamic shared memory: one CTA per SM

__device__ int mx_status_sink;              // where a run-out wait is noted when the caller gave no status word

struct MmArgs {
    const uint8_t* a_scales;
    const uint8_t* w_scales;
    void* out;
    int* status;
    long long out_stride;
    int m, n, k;
    int n_tile;                             // tokens per tile
    int pieces;                             // 128-row pieces of the token tile's scales
    int n_stage;                            // stages of the ring
    int stage_bytes;
    int tmem_cols;
    int split;                              // CTAs of the cluster
    int out_bf16;
    int w_early;                            // the launch before this one wrote only A: W may be read before it is complete
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
    const int n0 = blockIdx.y * 128, t0 = blockIdx.z * p.n_tile;
    const int tokens = min(p.n_tile, p.m - t0);
    const int n_mma = (tokens + 15) & ~15;
    const long long kp = (p.k + kMxBlock - 1) / kMxBlock * kMxBlock;        // padded with zeros to whole blocks
    const int n_span = (p.k + kMxSpan - 1) / kMxSpan;
    const int all = (int)((kp + kMmStageK - 1) / kMmStageK);
    const int s0 = (int)((long long)all * rank / p.split), s1 = (int)((long long)all * (rank + 1) / p.split);
    int* const status = p.status ? p.status : &mx_status_sink;
    volatile int* abort_p = &abort_flag;

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.n_stage; ++i) {
            mbar_init(smem_u32(&bar_full[i]), 1);
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
    const uint32_t tmem_sf = tmem + acc_cols;                                // per stage: 8 columns for W, 8 per piece for A
    const int sf_cols = 8 + 8 * p.pieces;
    const int w_bytes = 128 * 128, a_bytes = p.n_tile * 128;

    if (warp == 0) {
        // ---------------------------------------------------------------- copies
        const uint32_t on = elect_one();
        const int pieces = min(p.pieces, (tokens + 127) / 128);
        const int piece_t = t0 / 128, piece_w = n0 / 128;
        auto w_part = [&](int s) {
            const int i = (s - s0) % p.n_stage;
            const uint32_t st = base + i * p.stage_bytes, bar = smem_u32(&bar_full[i]);
            const int spans = min(2, n_span - 2 * s);
            expect_tx_on(on, bar, w_bytes + a_bytes + spans * kMxPiece * (1 + pieces));
            tma_2d_on(on, st, &map_w, s * 128, n0, bar);
            bulk_g2s_on(on, st + w_bytes + a_bytes, p.w_scales + ((size_t)piece_w * n_span + 2 * s) * kMxPiece, spans * kMxPiece, bar);
        };
        auto a_part = [&](int s) {
            const int i = (s - s0) % p.n_stage;
            const uint32_t st = base + i * p.stage_bytes, bar = smem_u32(&bar_full[i]);
            const int spans = min(2, n_span - 2 * s);
            tma_2d_on(on, st + w_bytes, &map_a, s * 128, t0, bar);
            for (int q = 0; q < pieces; ++q)
                bulk_g2s_on(on, st + w_bytes + a_bytes + (1 + q) * 2 * kMxPiece,
                         p.a_scales + ((size_t)(piece_t + q) * n_span + 2 * s) * kMxPiece, spans * kMxPiece, bar);
        };
        int early = 0;
        if (p.w_early)
            for (; early < p.n_stage && s0 + early < s1; ++early) w_part(s0 + early);
        pdl_wait();
        pdl_launch_dependents();
        int s = s0;
        bool ok = true;
        for (; s < s1; ++s) {
            const int it = s - s0;
            if (it >= p.n_stage) {
                ok = mbar_wait_warp(smem_u32(&bar_empty[it % p.n_stage]), (it / p.n_stage - 1) & 1, abort_p, status);
                if (!ok) break;
            }
            if (it >= early) w_part(s);
            a_part(s);
        }
        if (!ok && lane == 0)                                                // copies still under way land before the CTA ends
            for (int q = max(s0, s - p.n_stage); q < s; ++q) {
                abort_flag = 0;
                mbar_wait(smem_u32(&bar_full[(q - s0) % p.n_stage]), ((q - s0) / p.n_stage) & 1, abort_p, status);
                abort_flag = 1;
            }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issue
        const uint32_t on = elect_one();
        for (int s = s0; s < s1; ++s) {
            const int it = s - s0, i = it % p.n_stage;
            if (!mbar_wait_warp(smem_u32(&bar_full[i]), (it / p.n_stage) & 1, abort_p, status)) break;
            tc_fence_after();
            const uint32_t st = base + i * p.stage_bytes, sf = st + w_bytes + a_bytes;
            const uint32_t tw = tmem_sf + i * sf_cols, ta = tw + 8;
            const int spans = min(2, n_span - 2 * s);
            for (int h = 0; h < spans; ++h) {
                tc_cp_scales(on, tw + 4 * h, smem_desc_scales(sf + h * kMxPiece));
                for (int q = 0; q < p.pieces; ++q)
                    tc_cp_scales(on, ta + 4 * (h * p.pieces + q), smem_desc_scales(sf + ((1 + q) * 2 + h) * kMxPiece));
            }
            const int steps = (int)min(4ll, (kp - (long long)s * kMmStageK + 63) / 64);
            const uint64_t dw = smem_desc_sw128(st), da = smem_desc_sw128(st + w_bytes);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < steps) tc_mma_mxf4(on, tmem, dw + 2 * j, da + 2 * j, idesc_mxf4(n_mma, (j & 1) * 2), tw + 4 * (j >> 1),
                            ta + 4 * (j >> 1) * p.pieces, s > s0 || j > 0);
            tc_commit_on(on, smem_u32(&bar_empty[i]));
        }
        tc_commit_on(on, smem_u32(&bar_acc));
    }
    __syncwarp();

    // -------------------------------------------------------------------- epilogue
    const int quad = warp & 3, row = quad * 32 + lane;
    const bool store_row = n0 + row < p.n;
    auto put = [&](int c, float v) {
        const size_t at = (size_t)(t0 + c) * p.out_stride + n0 + row;
        if (p.out_bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(p.out)[at] = v;
    };
    bool done = false;
    if (warp >= 2) {
        done = mbar_wait(smem_u32(&bar_acc), 0, abort_p, status) && !*abort_p;
        tc_fence_after();
        pdl_wait();                                                          // nothing is written before older kernels have ended
        if (done)
            for (int c = 0; c < n_mma; c += 16) {
                float v[16];
                tc_ld16(tmem + ((uint32_t)(quad * 32) << 16) + c, v);
                if (p.split > 1) {
                    // partial sums [column][row] where the stages were: every MMA has read them
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(base + ((c + i) * 128 + row) * 4), "f"(v[i]) : "memory");
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
            for (int c = rank; c < tokens; c += p.split) {
                float sum = 0.f;
                for (int q = 0; q < p.split; ++q) {
                    float v;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];"
                                 : "=f"(v) : "r"(mapa_u32(base + (c * 128 + row) * 4, q)) : "memory");
                    sum += v;
                }
                if (store_row) put(c, sum);
            }
        cluster_sync_all();                                                  // no CTA ends while another reads its shared memory
    } else {
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols));
    }
}

// ------------------------------------------------------------------------------------------------------------- host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn g_mx_encode = nullptr;
static bool g_mx_done[64];

static cudaError_t mx_matmul_init() {
    if (!g_mx_encode) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
        if (e != cudaSuccess) return e;
        if (!fn || q != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
        g_mx_encode = (EncodeTiledFn)fn;
    }
    if (!first_call_on_device(g_mx_done)) return cudaSuccess;
    return cudaFuncSetAttribute(mx_matmul_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmSmem);
}

// Codes as a byte matrix: boxes of 128 bytes (256 elements) x `box_rows` rows; what lies outside reads as zero.
static bool make_code_map(CUtensorMap* m, const void* codes, long long rows, long long cols, int box_rows) {
    const cuuint64_t pitch = (cuuint64_t)((cols + kMxBlock - 1) / kMxBlock) * 16;
    const cuuint64_t dims[2] = {pitch, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {pitch};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return g_mx_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, estr,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static cudaError_t launch_mx_matmul(const uint8_t* a_codes, const uint8_t* a_scales, int m, const uint8_t* w_codes,
                                    const uint8_t* w_scales, int n, int k, void* out, int out_bf16, long long out_stride,
                                    int* status, int w_early, cudaStream_t st) {
    cudaError_t e = mx_matmul_init();
    if (e != cudaSuccess) return e;
    int dev, n_sm;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if ((e = cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
    MmArgs p = {};
    p.a_scales = a_scales; p.w_scales = w_scales; p.out = out; p.status = status; p.out_stride = out_stride;
    p.m = m; p.n = n; p.k = k; p.out_bf16 = out_bf16; p.w_early = w_early;
    p.n_tile = m <= 256 ? round_up(m, 16) : 256;
    p.pieces = (p.n_tile + 127) / 128;
    p.stage_bytes = 128 * 128 + p.n_tile * 128 + 2 * kMxPiece * (1 + p.pieces);
    p.stage_bytes = round_up(p.stage_bytes, 1024);
    p.n_stage = (kMmSmem - 1024) / p.stage_bytes;
    if (p.n_stage > kMmMaxStages) p.n_stage = kMmMaxStages;
    const int need = round_up(p.n_tile, 32) + p.n_stage * (8 + 8 * p.pieces);
    p.tmem_cols = 32;
    while (p.tmem_cols < need) p.tmem_cols *= 2;
    if (p.tmem_cols > 512) return cudaErrorInvalidValue;
    const int stages = (k + kMmStageK - 1) / kMmStageK;
    const long long tiles = (long long)((n + 127) / 128) * ((m + p.n_tile - 1) / p.n_tile);
    p.split = 1;
    while (p.split < 8 && tiles * p.split * 2 <= n_sm && p.split * 2 <= stages) p.split *= 2;
    alignas(64) CUtensorMap map_w, map_a;
    if (!make_code_map(&map_w, w_codes, n, k, 128) || !make_code_map(&map_a, a_codes, m, k, p.n_tile))
        return cudaErrorInvalidValue;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.split, (n + 127) / 128, (m + p.n_tile - 1) / p.n_tile);
    cfg.blockDim = dim3(kMmThreads);
    cfg.dynamicSmemBytes = kMmSmem;
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
    return launch_mx_matmul((const uint8_t*)a_codes, (const uint8_t*)a_scales, (int)m, (const uint8_t*)w_codes,
                            (const uint8_t*)w_scales, (int)n, (int)k, out, out_dtype == SAEM_OUT_BF16, out_stride, status, 0,
                            (cudaStream_t)stream) == cudaSuccess ? SAEM_OK : SAEM_ERR_CUDA;
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
    uint8_t* codes = (uint8_t*)workspace + 256;                              // the status word stands before them
    uint8_t* scales = codes + (saem_mx_codes_bytes(m, k) + 255) / 256 * 256;
    const int q = saem_mx_quantize(x, x_dtype, m, k, x_stride, codes, scales, stream);
    if (q != SAEM_OK) return q;
    return launch_mx_matmul(codes, scales, (int)m, (const uint8_t*)w_codes, (const uint8_t*)w_scales, (int)n, (int)k, out,
                            out_dtype == SAEM_OUT_BF16, out_stride, (int*)workspace, 1, (cudaStream_t)stream) == cudaSuccess
               ? SAEM_OK : SAEM_ERR_CUDA;
}

}  // extern "C"
