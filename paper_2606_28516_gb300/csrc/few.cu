// A whole folded layer for a few tokens (1 to 64): y_t = W_comb[a_t] GELU(W1 x_t + b1) (+ b2), in two launches.
//
//   fc1 kernel      one CTA per 16 rows of W1 for every token, and one CTA per token for its routing;
//   expert kernel   one CTA per 16 output rows and group (expert, or the class tokens' dense path), for the
//                   tokens of that group; a group without tokens is not read.
//
// What bounds them is reading the weights once, W1 and the matrices of the experts that are taken, at these
// sizes mostly the time until the first bytes come: so the first loads of weights are issued before the wait for
// the previous kernel (W1's always, an expert's when most experts will have a token), and the product is a
// warp-level MMA on registers (few.cuh): with at most 64 columns the tcgen05 tiles of the other forwards would be
// mostly empty, and the weights would first have to cross shared memory.
//
// Element types: bf16 weights with bf16 tokens; fp32 with fp32, each operand split into a TF32 part and the
// remainder, three products; 8-bit blocks with bf16 tokens, each weight widened to bf16 exactly and the block's
// scale applied to the fp32 sum. z is stored in the layer's dtype, as in the other forwards.
#include <cstdint>
#include <type_traits>

#include "common.cuh"
#include "few.cuh"
#include "internal.h"

namespace cm {

namespace {

template <int V>
__device__ __forceinline__ float few_get(const void* p, int64_t i) {
    return V == FEWV_F32 ? __ldcg(static_cast<const float*>(p) + i) : bf16_to_f32(__ldcg(static_cast<const uint16_t*>(p) + i));
}
template <int V>
__device__ __forceinline__ void few_put(void* p, int64_t i, float v) {
    if (V == FEWV_F32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
}

// A row of d <= 1024 (bf16) or 512 (fp32) elements over a warp, 16 bytes a lane and piece; pieces past d are zero.
constexpr int FEW_PIECES = 4;
template <int V>
struct FewRow {
    static constexpr int PER = V == FEWV_F32 ? 4 : 8;
    float v[FEW_PIECES][PER];
    __device__ __forceinline__ void load(const void* x, int64_t row, int d, int lane) {
        uint4 u[FEW_PIECES];
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p) {
            const int k = (p * 32 + lane) * PER;
            u[p] = make_uint4(0, 0, 0, 0);
            if (k < d) u[p] = few_ld_token(static_cast<const char*>(x) + (row * d + k) * (16 / PER));
        }
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p) {
            const uint32_t w[4] = {u[p].x, u[p].y, u[p].z, u[p].w};
#pragma unroll
            for (int i = 0; i < PER; ++i)
                v[p][i] = V == FEWV_F32 ? __uint_as_float(w[i & 3]) : (i & 1) ? bf16_hi(w[(i >> 1) & 3]) : bf16_lo(w[(i >> 1) & 3]);
        }
    }
    // (mean, 1 / sqrt(biased variance + 1e-6)), the variance from the differences to the mean
    __device__ __forceinline__ float2 stats(int d, int lane) const {
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p)
#pragma unroll
            for (int i = 0; i < PER; ++i) s += v[p][i];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        const float mean = s / (float)d;
        float q = 0.f;
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p)
            if ((p * 32 + lane) * PER < d) {
#pragma unroll
                for (int i = 0; i < PER; ++i) q = fmaf(v[p][i] - mean, v[p][i] - mean, q);
            }
#pragma unroll
        for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
        return make_float2(mean, 1.f / sqrtf(q / (float)d + 1e-6f));
    }
};

// The routing of token t by one CTA: a warp per expert, the logits in fp32, lowest index on ties.
template <int V>
__device__ __forceinline__ void few_route(const FewArgs& a, int t, float* s_logit, int warp, int lane) {
    if (a.cls_stride > 0 && t % a.cls_stride == 0) {
        if (threadIdx.x == 0) a.idx[t] = a.E;
        return;
    }
    FewRow<V> x, w;
    x.load(a.x, t, a.d, lane);
    float2 st = make_float2(0.f, 1.f);
    if (a.ln) st = x.stats(a.d, lane);
    for (int e = warp; e < a.E; e += FEW_WARPS) {
        w.load(a.Wg, e, a.d, lane);  // zeros past d
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p)
#pragma unroll
            for (int i = 0; i < FewRow<V>::PER; ++i) s = fmaf((x.v[p][i] - st.x) * st.y, w.v[p][i], s);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane == 0) s_logit[e] = s + few_get<V>(a.bg, e);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int best = 0;
        for (int e = 1; e < a.E; ++e)
            if (s_logit[e] > s_logit[best]) best = e;
        a.idx[t] = best;
    }
}

template <int V, int NT, bool LN>
__global__ void __launch_bounds__(FEW_THREADS, 2) few_fc1_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];  // [warp][NT * 8 columns][16 rows], and the row sums' [warp][16]
    __shared__ float2 s_stats[CLEARMOE_FEW_MAX];
    __shared__ float s_logit[16];
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x < a.T) {  // first, as the expert kernel's work depends on them all
        pdl_wait();
        few_route<V>(a, blockIdx.x, s_logit, warp, lane);
        return;
    }
    const int r0 = (blockIdx.x - a.T) * 16;
    FewRound<V, NT> w;
    const FewTile m = few_tile<V>(a.W1, a.W1_s, V >= FEWV_W8A16 ? fp8_ldq(a.d) : a.d, fp8_lds(a.d), r0, a.H, a.d, lane);
    few_load<V, NT>(w, m, 0, warp, lane);
    pdl_wait();
    float acc[NT][4], sums[4] = {0.f, 0.f, 0.f, 0.f};
    const char* tok[NT];
    const uint8_t* none[NT][2] = {};
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        tok[j] = static_cast<const char*>(a.x) + (int64_t)min(8 * j + (lane >> 2), a.T - 1) * a.d * FewT<V, NT>::XSZ;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    few_product<V, NT, LN>(acc, sums, m, w, tok, none, warp, lane);
    few_stage<NT>(red, acc, warp, lane);
    float* red_sum = red + FEW_WARPS * NT * 128;
    if (LN) {
        if ((lane & 3) == 0) {  // column 0 of the ones
            red_sum[warp * 16 + (lane >> 2)] = sums[0];
            red_sum[warp * 16 + (lane >> 2) + 8] = sums[2];
        }
        for (int t = warp; t < a.T; t += FEW_WARPS) {
            FewRow<V> x;
            x.load(a.x, t, a.d, lane);
            const float2 st = x.stats(a.d, lane);
            if (lane == 0) s_stats[t] = st;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += FEW_THREADS) {
        const int t = i >> 4, r = i & 15;
        if (r0 + r >= a.H) continue;
        float s = few_sum<NT>(red, t, r);
        if (LN) {  // W LN(y) = rstd (W y - mean W 1)
            float c = 0.f;
#pragma unroll
            for (int q = 0; q < FEW_WARPS; ++q) c += red_sum[q * 16 + r];
            const float2 st = s_stats[t];
            s = st.y * (s - st.x * c);
        }
        few_put<V>(a.z, (int64_t)t * a.H + r0 + r, gelu_erf(s + few_get<V>(a.b1, r0 + r)));
    }
}

// The CTA's tile for the n tokens of its group, at most 8 NT; ROUND0: the first round's weights are in w.
template <int V, int NT>
__device__ __forceinline__ void few_expert(const FewArgs& a, const FewTile& m, FewRound<V, NT>& w, float* red, const int* s_tok,
                                           int n, int r0, int warp, int lane) {
    float acc[NT][4], sums[4];
    const char* tok[NT];
    const uint8_t* none[NT][2] = {};
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        tok[j] = static_cast<const char*>(a.z) + (int64_t)s_tok[min(8 * j + (lane >> 2), n - 1)] * a.H * FewT<V, NT>::XSZ;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    few_product<V, NT, false>(acc, sums, m, w, tok, none, warp, lane);
    few_stage<NT>(red, acc, warp, lane);
    __syncthreads();
    for (int i = threadIdx.x; i < n * 16; i += FEW_THREADS) {
        const int j = i >> 4, r = i & 15;
        if (r0 + r >= a.d) continue;
        float s = few_sum<NT>(red, j, r);
        if (a.b2) s += few_get<V>(a.b2, r0 + r);
        few_put<V>(a.out, (int64_t)s_tok[j] * a.d + r0 + r, s);
    }
}

template <int V, int NT>
__global__ void __launch_bounds__(FEW_THREADS, 2) few_expert_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];
    __shared__ int s_tok[CLEARMOE_FEW_MAX];
    __shared__ int s_n;
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int e = blockIdx.y, r0 = blockIdx.x * 16;
    const FewTile m = few_tile<V>(a.Wc[e], a.Wc_s[e], V >= FEWV_W8A16 ? fp8_ldq(a.H) : a.H, fp8_lds(a.H), r0, a.d, a.H, lane);
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
    // as many token tiles as the group needs
    auto run = [&](auto tiles) {
        constexpr int N = decltype(tiles)::value;
        FewRound<V, N> w;
        few_load<V, N>(w, m, 0, warp, lane);
        few_expert<V, N>(a, m, w, red, s_tok, n, r0, warp, lane);
    };
    if (NT == 1 || n <= 8) return run(std::integral_constant<int, 1>());
    if (NT == 2 || n <= 16) return run(std::integral_constant<int, (NT < 2 ? NT : 2)>());
    if (NT == 4 || n <= 32) return run(std::integral_constant<int, (NT < 4 ? NT : 4)>());
    run(std::integral_constant<int, NT>());
}

template <typename K>
cudaError_t few_launch(K kernel, dim3 grid, int smem, const FewArgs& a, cudaStream_t s) {
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

template <int V, int NT>
cudaError_t few_run(const FewArgs& a, cudaStream_t s) {
    const dim3 g1((a.H + 15) / 16 + a.T), g2((a.d + 15) / 16, a.G);
    const cudaError_t e = a.ln ? few_launch(few_fc1_kernel<V, NT, true>, g1, few_smem(NT) + FEW_WARPS * 64, a, s)
                               : few_launch(few_fc1_kernel<V, NT, false>, g1, few_smem(NT), a, s);
    return e != cudaSuccess ? e : few_launch(few_expert_kernel<V, NT>, g2, few_smem(NT), a, s);
}

template <int V>
cudaError_t few_type(const FewArgs& a, cudaStream_t s) {
    return a.T <= 8 ? few_run<V, 1>(a, s) : a.T <= 16 ? few_run<V, 2>(a, s) : a.T <= 32 ? few_run<V, 4>(a, s) : few_run<V, 8>(a, s);
}

}  // namespace

cudaError_t launch_few(const FewArgs& a, cudaStream_t s) {
    return a.f32 ? few_type<FEWV_F32>(a, s) : a.fp8 ? few_type<FEWV_W8A16>(a, s) : few_type<FEWV_BF16>(a, s);
}

}  // namespace cm
