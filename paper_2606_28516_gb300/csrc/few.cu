// A whole folded layer for a few tokens (1 to 64): y_t = W_comb[a_t] GELU(W1 x_t + b1) (+ b2), in two launches.
//
//   fc1 kernel      one CTA per 16 rows of W1 for every token, and one CTA per token for its routing;
//   expert kernel   one CTA per 16 output rows and group (expert, or the class tokens' dense path), for the
//                   tokens of that group; a group without tokens is not read.
//
// What bounds them is reading the weights once, W1 and the matrices of the experts that are taken, at these
// sizes mostly the time until the first bytes come. So a CTA's weights go from global memory straight to the
// registers they are multiplied from, all loads of a lane issued ahead of the products, and the eight warps of a
// CTA split K. The products are 16 x 8 x k warp-level MMAs (weights 16 rows, tokens 8 columns): with so few
// columns the tcgen05 tiles of the other forwards would be a sixteenth full, and their operands would first
// have to cross shared memory. The order of K within a sum is free as long as weights and tokens agree, so lane
// (g, c) of a warp takes 16 consecutive bytes of weight rows g and g + 8 and the same columns of token g, and
// feeds them to the MMA as its fragments. Partial sums of the warps are added in warp order in shared memory.
//
// Element types (WT): bf16 weights with bf16 tokens; fp32 with fp32, each operand split into a TF32 part and the
// remainder, three products; 8-bit blocks with bf16 tokens, each weight widened to bf16 exactly and the block's
// scale applied to the fp32 sum.
#include <cstdint>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace cm {

namespace {

constexpr int FEW_WARPS = 8;
constexpr int FEW_THREADS = FEW_WARPS * 32;
enum FewType { FEW_F32 = 0, FEW_BF16 = 1, FEW_FP8 = 2 };

// Weight columns per lane and step (16 bytes), and per step of a warp.
template <int WT>
struct FewT {
    static constexpr int LANE = WT == FEW_F32 ? 4 : WT == FEW_BF16 ? 8 : 16;
    static constexpr int STEP = 4 * LANE;
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// v rounded to TF32 (to nearest, ties away from zero) and the exact remainder
__device__ __forceinline__ void tf32_split(uint32_t v, uint32_t& h, uint32_t& l) {
    h = (v + 0x1000u) & 0xFFFFE000u;
    l = __float_as_uint(__uint_as_float(v) - __uint_as_float(h));
}
// Two e4m3 values as a pair of bf16, exactly
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t v) {
    const float2 f = fp8_unpack2(v & 0xFFFFu);
    return pack_bf16(f.x, f.y);
}

// Weight matrix of a CTA: rows of `pitch` elements, K columns in use.
struct FewMat {
    const void* w;
    const uint8_t* s;  // FEW_FP8: scales of the CTA's 16 rows (one block of 128 rows)
    int64_t pitch;
    int K;
};

// acc[j] += the warp's share of W[r0 .. r0 + 16) x token tile j: steps warp, warp + 8, ... of K. Token column
// 8 j + g is row tok[j] (a pointer per lane, its own g) of the activations, K elements. sums (LN): += W 1.
template <int WT, int NT, bool LN>
__device__ __forceinline__ void few_product(float (&acc)[NT][4], float (&sums)[4], const FewMat& m, int r0, int rows,
                                            const char* const (&tok)[NT], int nt, int warp, int lane) {
    using F = FewT<WT>;
    const int g = lane >> 2, c = lane & 3;
    const int esz = WT == FEW_F32 ? 4 : WT == FEW_BF16 ? 2 : 1;
    const int xsz = WT == FEW_F32 ? 4 : 2;
    const char* w0 = static_cast<const char*>(m.w) + (int64_t)min(r0 + g, rows - 1) * m.pitch * esz;
    const char* w1 = static_cast<const char*>(m.w) + (int64_t)min(r0 + g + 8, rows - 1) * m.pitch * esz;
    const int steps = (m.K + F::STEP - 1) / F::STEP;
#pragma unroll 4
    for (int st = warp; st < steps; st += FEW_WARPS) {
        const int k = st * F::STEP + c * F::LANE;
        const bool in = k < m.K;  // K is a multiple of a lane's columns
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (in) {
            a = __ldg(reinterpret_cast<const uint4*>(w0 + (int64_t)k * esz));
            b = __ldg(reinterpret_cast<const uint4*>(w1 + (int64_t)k * esz));
        }
        const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
        float part[WT == FEW_FP8 ? NT : 1][4];
        if (WT == FEW_FP8) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[j][i] = 0.f;
        }
        float scale = 1.f;
        float psum[4] = {0.f, 0.f, 0.f, 0.f};
        if (WT == FEW_FP8) scale = fp8_scale(m.s[k / 128]);
        if constexpr (WT == FEW_F32) {
            uint32_t ah[4], al[4], bh[4], bl[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tf32_split(wa[i], ah[i], al[i]);
                tf32_split(wb[i], bh[i], bl[i]);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (j < nt) {
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (in) x = __ldcg(reinterpret_cast<const uint4*>(tok[j] + (int64_t)k * xsz));
                    const uint32_t xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // columns 2 h, 2 h + 1 of the lane's four
                        uint32_t xh[2], xl[2];
                        tf32_split(xv[2 * h], xh[0], xl[0]);
                        tf32_split(xv[2 * h + 1], xh[1], xl[1]);
                        const uint32_t fh[4] = {ah[2 * h], bh[2 * h], ah[2 * h + 1], bh[2 * h + 1]};
                        const uint32_t fl[4] = {al[2 * h], bl[2 * h], al[2 * h + 1], bl[2 * h + 1]};
                        mma_tf32(acc[j], fl, xh[0], xh[1]);
                        mma_tf32(acc[j], fh, xl[0], xl[1]);
                        mma_tf32(acc[j], fh, xh[0], xh[1]);
                    }
                }
            }
            if (LN) {
                const uint32_t one = __float_as_uint(1.f);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t fh[4] = {ah[2 * h], bh[2 * h], ah[2 * h + 1], bh[2 * h + 1]};
                    const uint32_t fl[4] = {al[2 * h], bl[2 * h], al[2 * h + 1], bl[2 * h + 1]};
                    mma_tf32(sums, fl, one, one);
                    mma_tf32(sums, fh, one, one);
                }
            }
        } else {
            constexpr int NS = F::LANE / 4;  // MMAs of 16 columns per step: four of the lane's columns each
            uint32_t f[NS][4];
#pragma unroll
            for (int h = 0; h < NS; ++h) {
                if (WT == FEW_BF16) {
                    f[h][0] = wa[(2 * h) & 3], f[h][1] = wb[(2 * h) & 3];
                    f[h][2] = wa[(2 * h + 1) & 3], f[h][3] = wb[(2 * h + 1) & 3];
                } else {
                    f[h][0] = fp8x2_to_bf16x2(wa[h & 3]), f[h][1] = fp8x2_to_bf16x2(wb[h & 3]);
                    f[h][2] = fp8x2_to_bf16x2(wa[h & 3] >> 16), f[h][3] = fp8x2_to_bf16x2(wb[h & 3] >> 16);
                }
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (j < nt) {
                    uint32_t xv[2 * NS];
#pragma unroll
                    for (int h = 0; h < NS / 2; ++h) {
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (in) x = __ldcg(reinterpret_cast<const uint4*>(tok[j] + (int64_t)k * xsz) + h);
                        xv[4 * h] = x.x, xv[4 * h + 1] = x.y, xv[4 * h + 2] = x.z, xv[4 * h + 3] = x.w;
                    }
#pragma unroll
                    for (int h = 0; h < NS; ++h) {
                        if (WT == FEW_FP8)
                            mma_bf16(part[WT == FEW_FP8 ? j : 0], f[h][0], f[h][1], f[h][2], f[h][3], xv[2 * h], xv[2 * h + 1]);
                        else
                            mma_bf16(acc[j], f[h][0], f[h][1], f[h][2], f[h][3], xv[2 * h], xv[2 * h + 1]);
                    }
                    if (WT == FEW_FP8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(part[WT == FEW_FP8 ? j : 0][i], scale, acc[j][i]);
                    }
                }
            }
            if (LN) {
                const uint32_t one = 0x3F803F80u;  // a pair of bf16 ones
#pragma unroll
                for (int h = 0; h < NS; ++h) mma_bf16(psum, f[h][0], f[h][1], f[h][2], f[h][3], one, one);
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[i] = fmaf(psum[i], scale, sums[i]);
            }
        }
    }
}

// The warps' partial sums, [warp][token column][16 rows], and where column n, row r of a warp's lie.
template <int NT>
__device__ __forceinline__ void few_stage(float* red, const float (&acc)[NT][4], int nt, int warp, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        if (j < nt) {
            float* p = red + ((warp * NT + j) * 8 + 2 * c) * 16;
            p[g] = acc[j][0];
            p[16 + g] = acc[j][1];
            p[g + 8] = acc[j][2];
            p[16 + g + 8] = acc[j][3];
        }
    }
}

template <int WT>
__device__ __forceinline__ float few_load(const void* p, int64_t i) {
    return WT == FEW_F32 ? __ldcg(static_cast<const float*>(p) + i)
                         : bf16_to_f32(__ldcg(static_cast<const uint16_t*>(p) + i));
}
template <int WT>
__device__ __forceinline__ void few_store(void* p, int64_t i, float v) {
    if (WT == FEW_F32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
}

// Mean and 1 / sqrt(biased variance + 1e-6) of a row, by one warp, two passes over the row in registers or L1.
template <int WT>
__device__ __forceinline__ float2 few_row_stats(const void* x, int64_t row, int d, int lane) {
    float s = 0.f;
    for (int k = lane; k < d; k += 32) s += few_load<WT>(x, row * d + k);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    const float mean = s / (float)d;
    float q = 0.f;
    for (int k = lane; k < d; k += 32) {
        const float v = few_load<WT>(x, row * d + k) - mean;
        q = fmaf(v, v, q);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
    return make_float2(mean, 1.f / sqrtf(q / (float)d + 1e-6f));
}

// The routing of token t by one CTA: a warp per expert, the logits in fp32, lowest index on ties.
template <int WT>
__device__ __forceinline__ void few_route(const FewArgs& a, int t, float* s_logit, int warp, int lane) {
    if (a.cls_stride > 0 && t % a.cls_stride == 0) {
        if (threadIdx.x == 0) a.idx[t] = a.E;
        return;
    }
    float2 st = make_float2(0.f, 1.f);
    if (a.ln) st = few_row_stats<WT>(a.x, t, a.d, lane);
    for (int e = warp; e < a.E; e += FEW_WARPS) {
        float s = 0.f;
        for (int k = lane; k < a.d; k += 32) {
            float v = few_load<WT>(a.x, (int64_t)t * a.d + k);
            if (a.ln) v = (v - st.x) * st.y;
            s = fmaf(v, few_load<WT>(a.Wg, (int64_t)e * a.d + k), s);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane == 0) s_logit[e] = s + few_load<WT>(a.bg, e);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int best = 0;
        for (int e = 1; e < a.E; ++e)
            if (s_logit[e] > s_logit[best]) best = e;
        a.idx[t] = best;
    }
}

template <int WT, int NT, bool LN>
__global__ void __launch_bounds__(FEW_THREADS) few_fc1_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];  // [warp][NT * 8 columns][16 rows], and the row sums' [warp][16]
    __shared__ float2 s_stats[CLEARMOE_FEW_MAX];
    __shared__ float s_logit[16];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tiles = (a.H + 15) / 16;
    if ((int)blockIdx.x >= tiles) {
        few_route<WT>(a, blockIdx.x - tiles, s_logit, warp, lane);
        return;
    }
    const int r0 = blockIdx.x * 16;
    const int nt = (a.T + 7) / 8;
    float acc[NT][4], sums[4] = {0.f, 0.f, 0.f, 0.f};
    const char* tok[NT];
    const int xsz = WT == FEW_F32 ? 4 : 2;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        tok[j] = static_cast<const char*>(a.x) + (int64_t)min(8 * j + (lane >> 2), a.T - 1) * a.d * xsz;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    FewMat m = {a.W1, a.W1_s, a.d, a.d};
    if (WT == FEW_FP8) {
        m.s += (int64_t)(r0 / 128) * fp8_lds(a.d);
        m.pitch = fp8_ldq(a.d);
    }
    if (LN)
        for (int t = warp; t < a.T; t += FEW_WARPS) {
            const float2 st = few_row_stats<WT>(a.x, t, a.d, lane);
            if (lane == 0) s_stats[t] = st;
        }
    few_product<WT, NT, LN>(acc, sums, m, r0, a.H, tok, nt, warp, lane);
    few_stage<NT>(red, acc, nt, warp, lane);
    float* red_sum = red + FEW_WARPS * NT * 128;
    if (LN && (lane & 3) == 0) {  // column 0 of the ones
        red_sum[warp * 16 + (lane >> 2)] = sums[0];
        red_sum[warp * 16 + (lane >> 2) + 8] = sums[2];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += FEW_THREADS) {
        const int t = i >> 4, r = i & 15;
        if (r0 + r >= a.H) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) s += red[(w * NT * 8 + t) * 16 + r];
        if (LN) {  // W LN(y) = rstd (W y - mean W 1)
            float c = 0.f;
#pragma unroll
            for (int w = 0; w < FEW_WARPS; ++w) c += red_sum[w * 16 + r];
            const float2 st = s_stats[t];
            s = st.y * (s - st.x * c);
        }
        few_store<WT>(a.z, (int64_t)t * a.H + r0 + r, gelu_erf(s + few_load<WT>(a.b1, r0 + r)));
    }
}

template <int WT, int NT>
__global__ void __launch_bounds__(FEW_THREADS) few_expert_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];
    __shared__ int s_tok[CLEARMOE_FEW_MAX];
    __shared__ int s_n;
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int e = blockIdx.y, r0 = blockIdx.x * 16;
    pdl_wait();
    if (warp == 0) {  // the group's tokens in order
        int n = 0;
        for (int t0 = 0; t0 < a.T; t0 += 32) {
            const bool mine = t0 + lane < a.T && __ldcg(a.idx + t0 + lane) == e;
            const uint32_t b = __ballot_sync(0xFFFFFFFFu, mine);
            if (mine) s_tok[n + __popc(b & ((1u << lane) - 1))] = t0 + lane;
            n += __popc(b);
        }
        if (lane == 0) s_n = n;
    } else if (warp == 1 && blockIdx.x == 0) {  // counts, offsets and perm, as the other forwards leave them
        int before = 0, n = 0;
        for (int t0 = 0; t0 < a.T; t0 += 32) {
            const int v = t0 + lane < a.T ? __ldcg(a.idx + t0 + lane) : a.G;
            before += __popc(__ballot_sync(0xFFFFFFFFu, v < e));
            n += __popc(__ballot_sync(0xFFFFFFFFu, v == e));
        }
        int at = before;
        for (int t0 = 0; t0 < a.T; t0 += 32) {
            const bool mine = t0 + lane < a.T && __ldcg(a.idx + t0 + lane) == e;
            const uint32_t b = __ballot_sync(0xFFFFFFFFu, mine);
            if (mine) a.perm[at + __popc(b & ((1u << lane) - 1))] = t0 + lane;
            at += __popc(b);
        }
        if (lane == 0) {
            a.counts[e] = n;
            a.offsets[e] = before;
            if (e + 1 == a.G) a.offsets[a.G] = a.T;
        }
    }
    __syncthreads();
    const int n = s_n;
    if (n == 0) return;
    const int nt = (n + 7) / 8;
    float acc[NT][4], sums[4];
    const char* tok[NT];
    const int xsz = WT == FEW_F32 ? 4 : 2;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        tok[j] = static_cast<const char*>(a.z) + (int64_t)s_tok[min(8 * j + (lane >> 2), n - 1)] * a.H * xsz;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    FewMat m = {a.Wc[e], a.Wc_s[e], a.H, a.H};
    if (WT == FEW_FP8) {
        m.s += (int64_t)(r0 / 128) * fp8_lds(a.H);
        m.pitch = fp8_ldq(a.H);
    }
    few_product<WT, NT, false>(acc, sums, m, r0, a.d, tok, nt, warp, lane);
    few_stage<NT>(red, acc, nt, warp, lane);
    __syncthreads();
    for (int i = threadIdx.x; i < n * 16; i += FEW_THREADS) {
        const int j = i >> 4, r = i & 15;
        if (r0 + r >= a.d) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) s += red[(w * NT * 8 + j) * 16 + r];
        if (a.b2) s += few_load<WT>(a.b2, r0 + r);
        few_store<WT>(a.out, (int64_t)s_tok[j] * a.d + r0 + r, s);
    }
}

template <typename K>
cudaError_t few_launch(K kernel, dim3 grid, int smem, const FewArgs& a, cudaStream_t s) {
    if (smem > 48 * 1024) {
        const cudaError_t e = smem_attr_once((const void*)kernel, smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(FEW_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int WT, int NT>
cudaError_t few_run(const FewArgs& a, cudaStream_t s) {
    const int smem = FEW_WARPS * NT * 128 * 4;
    const dim3 g1((a.H + 15) / 16 + a.T), g2((a.d + 15) / 16, a.G);
    const cudaError_t e = a.ln ? few_launch(few_fc1_kernel<WT, NT, true>, g1, smem + FEW_WARPS * 64, a, s)
                               : few_launch(few_fc1_kernel<WT, NT, false>, g1, smem, a, s);
    return e != cudaSuccess ? e : few_launch(few_expert_kernel<WT, NT>, g2, smem, a, s);
}

template <int WT>
cudaError_t few_type(const FewArgs& a, cudaStream_t s) {
    const int nt = (a.T + 7) / 8;
    return nt <= 1 ? few_run<WT, 1>(a, s) : nt <= 2 ? few_run<WT, 2>(a, s) : nt <= 4 ? few_run<WT, 4>(a, s) : few_run<WT, 8>(a, s);
}

}  // namespace

cudaError_t launch_few(const FewArgs& a, int num_sms, cudaStream_t s) {
    (void)num_sms;
    return a.f32 ? few_type<FEW_F32>(a, s) : a.fp8 ? few_type<FEW_FP8>(a, s) : few_type<FEW_BF16>(a, s);
}

}  // namespace cm
