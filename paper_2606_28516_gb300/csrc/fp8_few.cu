// Products of matrices in 8-bit blocks with few rows of activations (1 to FP8_FEW_MAX): reading the weights once is
// all there is to it, and at most 16 columns would leave a tcgen05 tile mostly empty. One CTA per 16 rows of W for all
// rows of A, eight warps splitting K, weights from global memory straight to the registers of warp-level MMAs
// (few.cuh); a step of 64 columns lies in one block, whose two scales multiply its fp32 sum.
#include <cstdint>

#include "common.cuh"
#include "few.cuh"
#include "fp8_gemm.cuh"
#include "internal.h"

namespace cm {

namespace {

template <int NT>
__global__ void __launch_bounds__(FEW_THREADS, 2) fp8_few_kernel(const __grid_constant__ Fp8GemmArgs a) {
    extern __shared__ float red[];  // the partial sums; then scale bytes: the tile's rows' [nkb], A's rows' [M][nkb]
    __shared__ uint32_t s_nan[FEW_WARPS];  // bit 0: a NaN scale among the tile's rows', bit 1 + m: among those of A's row m
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(red) + FewT<FEWV_W8A8, NT, 2>::SMEM;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = blockIdx.x * 16, M = (int)a.M, ldq = a.nkb * 128;
    FewTile<FEWV_W8A8, NT, 2> t;
    t.set_weights(a.w, ldq, r0, a.N, ldq);
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    t.start_w();
    float acc[NT][4], sums[4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        t.set_row(j, static_cast<const char*>(a.x) + (int64_t)min(8 * j + (lane >> 2), M - 1) * ldq);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    t.start_x();
    const uint8_t* sw = a.sb[0] + (int64_t)(r0 / 128) * a.lds;
    uint32_t nan = 0;
    for (int i = threadIdx.x; i < (M + 1) * a.nkb; i += FEW_THREADS) {
        const int row = i / a.nkb, b = i - row * a.nkb;
        const uint8_t s = row == 0 ? __ldcg(sw + b) : __ldcg(a.sa + (int64_t)(row - 1) * a.lds + b);
        s_scale[i] = s;
        if (s == 255) nan |= 1u << row;
    }
    nan = __reduce_or_sync(0xFFFFFFFFu, nan);
    if (lane == 0) s_nan[warp] = nan;
    __syncthreads();
    few_product<FEWV_W8A8, NT, 2, false>(acc, sums, t, s_scale, s_scale + a.nkb, a.nkb, M);
    few_stage<NT>(red, acc, warp, lane);
    __syncthreads();
    nan = 0;
#pragma unroll
    for (int w = 0; w < FEW_WARPS; ++w) nan |= s_nan[w];
    for (int i = threadIdx.x; i < M * 16; i += FEW_THREADS) {
        const int m = i >> 4, n = r0 + (i & 15);
        if (n >= a.N) continue;
        float s = few_sum<8 * NT>(red, m, i & 15);
        if (nan & (1u | 2u << m)) s = __uint_as_float(0x7FC00000u);
        if (a.bias)
            s += a.bias_bf16 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(a.bias) + n)) : __ldcg(static_cast<const float*>(a.bias) + n);
        if (a.act == CLEARMOE_ACT_GELU) s = gelu_erf(s);
        if (a.act == CLEARMOE_ACT_RELU) s = s < 0.f ? 0.f : s;  // NaN stays NaN
        if (a.out_kind == FP8_OUT_BF16)
            static_cast<uint16_t*>(a.out)[(int64_t)m * a.ldo + n] = f32_to_bf16(s);
        else
            static_cast<float*>(a.out)[(int64_t)m * a.ldo + n] = s;
    }
}

template <int NT>
cudaError_t launch_nt(const Fp8GemmArgs& a, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((a.N + 15) / 16);
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = FewT<FEWV_W8A8, NT, 2>::SMEM + FP8_FEW_SCALES;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fp8_few_kernel<NT>, a);
}

}  // namespace

cudaError_t launch_fp8_few(const Fp8GemmArgs& a, cudaStream_t s) {
    return a.M <= 8 ? launch_nt<1>(a, s) : launch_nt<2>(a, s);
}

}  // namespace cm
