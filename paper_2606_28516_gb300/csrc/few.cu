// A whole folded layer for a few tokens (1 to 64): y_t = W_comb[a_t] GELU(W1 x_t + b1) (+ b2), in two launches.
//
//   fc1 kernel      one CTA per 16 rows of W1 for every token, and one CTA per token for its routing;
//   expert kernel   one CTA per 16 output rows and group (expert, or the class tokens' dense path), for the
//                   tokens of that group; of a group without tokens at most the first steps are.
//
// What bounds them is reading the weights once, W1 and the matrices of the experts that are taken, at these
// sizes mostly the time until the first bytes come: so the first loads of weights are issued before the wait for
// the previous kernel (W1's always, an expert's when most experts will have a token), and the product is a
// warp-level MMA on registers (few.cuh): with at most 64 columns the tcgen05 tiles of the other forwards would be
// mostly empty, and the weights would first have to cross shared memory.
//
// Element types: bf16 weights with bf16 tokens; fp32 with fp32, each operand split into a TF32 part and the
// remainder, three products; 8-bit blocks with bf16 tokens, each weight widened to bf16 exactly and the block's
// scale applied to the fp32 sum. Between the kernels z is stored in the layer's dtype, as in the other forwards; of up to
// 16 tokens of bf16 layers as two bf16 matrices, z rounded and the remainder rounded (16 bits of significand): rounded to
// bf16 alone it adds as much to the output's error as the output's own rounding (0.0024 instead of 0.0017 of its norm).
// The parts are neighbouring columns of the expert's product, which has columns to spare there, and their sums are added
// in fp32. (Beyond, they would double the columns and the reads of z: 64 tokens, d = 768, 18.2 us without, 21.1 with, on one
// expert, d = 1,024, 19.1 and 27.0; 13 tokens 14.4 and 14.6.)
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
            if (k < d) u[p] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const char*>(x) + (row * d + k) * (16 / PER)));
        }
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p) {
            const uint32_t w[4] = {u[p].x, u[p].y, u[p].z, u[p].w};
#pragma unroll
            for (int i = 0; i < PER; ++i)
                v[p][i] = V == FEWV_F32 ? __uint_as_float(w[i & 3]) : (i & 1) ? bf16_hi(w[(i >> 1) & 3]) : bf16_lo(w[(i >> 1) & 3]);
        }
    }
    // (mean, what it lacks, 1 / sqrt(biased variance + 1e-6)), the variance from the differences to the mean. fp32: the
    // mean of those differences is what the rounded mean lacks, without which a mean of many deviations would be off by as
    // many 2^-24 of them; bf16 tokens have no such means (0).
    __device__ __forceinline__ float3 stats(int d, int lane) const {
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p)
#pragma unroll
            for (int i = 0; i < PER; ++i) s += v[p][i];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        const float mean = s / (float)d;
        float rest = 0.f, q = 0.f;
        if (V == FEWV_F32) {
#pragma unroll
            for (int p = 0; p < FEW_PIECES; ++p)
                if ((p * 32 + lane) * PER < d) {
#pragma unroll
                    for (int i = 0; i < PER; ++i) rest += v[p][i] - mean;
                }
#pragma unroll
            for (int o = 16; o; o >>= 1) rest += __shfl_xor_sync(0xFFFFFFFFu, rest, o);
            rest /= (float)d;
        }
#pragma unroll
        for (int p = 0; p < FEW_PIECES; ++p)
            if ((p * 32 + lane) * PER < d) {
#pragma unroll
                for (int i = 0; i < PER; ++i) q = fmaf(v[p][i] - mean - rest, v[p][i] - mean - rest, q);
            }
#pragma unroll
        for (int o = 16; o; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
        return make_float3(mean, rest, 1.f / sqrtf(q / (float)d + 1e-6f));
    }
};

template <int V>
__device__ __forceinline__ int64_t few_pitch(int K) {  // bytes
    return V == FEWV_W8A16 ? fp8_ldq(K) : (int64_t)K * FewT<V, 1, 2>::WSZ;
}

// The routing of tokens TOK block .. TOK block + TOK - 1 by one CTA: a warp per expert (two above 8), its row of W_g in registers
// before the tokens may be read; the logits in fp32, lowest index on ties. (Eight tokens a CTA, one after the other,
// took longer than fc1: 9.3 us instead of 7.1 for 64 tokens, d = 192. With up to 16 tokens one a CTA: one token, 3.9 us
// against 4.5 with two; now 3.7.)
template <int V, int TOK>
__device__ __forceinline__ void few_route(const FewArgs& a, int block, float (*s_logit)[16], int warp, int lane) {
    FewRow<V> w[2], x[TOK];
#pragma unroll
    for (int q = 0; q < 2; ++q)
        if (warp + 8 * q < a.E) w[q].load(a.Wg, warp + 8 * q, a.d, lane);  // zeros past d
    pdl_wait();
    pdl_launch_dependents();
#pragma unroll
    for (int i = 0; i < TOK; ++i) x[i].load(a.x, min(TOK * block + i, a.T - 1), a.d, lane);
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        float3 st = make_float3(0.f, 0.f, 1.f);
        if (a.ln) st = x[i].stats(a.d, lane);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (warp + 8 * q >= a.E) break;
            float s = 0.f;
#pragma unroll
            for (int p = 0; p < FEW_PIECES; ++p)
#pragma unroll
                for (int c = 0; c < FewRow<V>::PER; ++c) s = fmaf((x[i].v[p][c] - st.x - st.y) * st.z, w[q].v[p][c], s);
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            if (lane == 0) s_logit[i][warp + 8 * q] = s + few_get<V>(a.bg, warp + 8 * q);
        }
    }
    __syncthreads();
    const int t = TOK * block + (int)threadIdx.x;  // a thread per token
    if (threadIdx.x >= TOK || t >= a.T) return;
    int best = 0;
    for (int e = 1; e < a.E; ++e)
        if (s_logit[threadIdx.x][e] > s_logit[threadIdx.x][best]) best = e;
    a.idx[t] = a.cls_stride > 0 && t % a.cls_stride == 0 ? a.E : best;
}

constexpr int few_route_tokens(int nt) { return nt <= 2 ? 1 : 2; }

// Tokens that a CTA of fc1 multiplies at a time.
constexpr int few_chunk(int nt) { return 8 * nt; }

// Parts that z is stored in, by the kernels' token tiles (four: more than 16 tokens), and tokens of NT column tiles.
constexpr int few_parts(int v, int nt) { return v == FEWV_F32 || nt > 2 ? 1 : 2; }
constexpr int few_pass(int parts, int nt) { return 8 * nt / parts; }

// Scale bytes of a tile's rows (8-bit weights) to shared memory; the caller synchronises.
template <int V>
__device__ __forceinline__ void few_scales(uint8_t* dst, const uint8_t* s, int r0, int K) {
    if (V != FEWV_W8A16) return;
    s += (int64_t)(r0 / 128) * fp8_lds(K);
    for (int i = threadIdx.x; i < (K + 127) / 128; i += blockDim.x) dst[i] = __ldg(s + i);
}

// The LayerNorm's statistics of tokens t0 .. t0 + rows - 1, a warp a token.
template <int V>
__device__ __forceinline__ void few_stats(const FewArgs& a, float3* s_stats, int t0, int rows, int warp, int lane) {
    for (int r = warp; r < rows; r += FEW_WARPS) {
        FewRow<V> x;
        x.load(a.x, t0 + r, a.d, lane);
        const float3 st = x.stats(a.d, lane);
        if (lane == 0) s_stats[r] = st;
    }
}

// LN, 8-bit and bf16 weights: W LN(y) = rstd (W y - mean W 1), y as it is in bf16 and W 1 of the same products. fp32: W LN(y)
// with each y normalised as it is split, because W y and mean W 1, with the TF32 products' error, would cancel (5 tokens,
// d = 64, means 3,000 times the deviation: 4e-5 of the output's norm; 24 tokens, d = 384, 13.7 us so, 14.2 normalised).
template <int V, int NT, int CTAS, bool LN>
__global__ void __launch_bounds__(FEW_THREADS, CTAS) few_fc1_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];  // the partial sums; then the scale bytes
    __shared__ float3 s_stats[few_chunk(NT)];
    __shared__ float s_logit[2][16];
    __shared__ float s_rows[FEW_WARPS][16];  // LN: the warps' row sums of W
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(red) + FewT<V, NT, CTAS>::SMEM;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int TOK = few_route_tokens(NT);
    const int routers = (a.T + TOK - 1) / TOK;
    if ((int)blockIdx.x < routers) {  // first, as the expert kernel's work depends on them all
        if (blockIdx.y == 0) few_route<V, TOK>(a, blockIdx.x, s_logit, warp, lane);
        return;
    }
    const int r0 = (blockIdx.x - routers) * 16;
    const int t0 = blockIdx.y * few_chunk(NT), rows = min(few_chunk(NT), a.T - t0);  // the CTA's tokens
    FewTile<V, NT, CTAS> t;
    t.set_weights(a.W1, few_pitch<V>(a.d), r0, a.H, a.d);
    t.start_w();
    few_scales<V>(s_scale, a.W1_s, r0, a.d);
    pdl_wait();
    // the expert kernel reads weights before its own wait: whatever wrote them before this call's predecessor has completed
    pdl_launch_dependents();
    float acc[NT][4], sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        t.set_row(j, static_cast<const char*>(a.x) + (int64_t)(t0 + min(8 * j + (lane >> 2), rows - 1)) * a.d * FewT<V, NT, CTAS>::XSZ);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    t.start_x();
    if (LN && V == FEWV_F32) {  // the statistics first, while the weights come
        few_stats<V>(a, s_stats, t0, rows, warp, lane);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) t.norm[j] = s_stats[min(8 * j + (lane >> 2), rows - 1)];
    }
    if (V == FEWV_W8A16) __syncthreads();
    few_product<V, NT, CTAS, LN>(acc, sums, t, s_scale, nullptr, 0, rows);
    few_stage<NT>(red, acc, warp, lane);
    if (LN && V != FEWV_F32) {
        if ((lane & 3) == 0) {  // column 0 of the ones
            s_rows[warp][lane >> 2] = sums[0];
            s_rows[warp][(lane >> 2) + 8] = sums[2];
        }
        few_stats<V>(a, s_stats, t0, rows, warp, lane);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * 16; i += FEW_THREADS) {
        const int m = i >> 4, r = i & 15;
        if (r0 + r >= a.H) continue;
        float s = few_sum<8 * NT>(red, m, r);
        if (LN && V != FEWV_F32) {
            float c = 0.f;
#pragma unroll
            for (int q = 0; q < FEW_WARPS; ++q) c += s_rows[q][r];
            const float3 st = s_stats[m];
            s = st.z * (s - st.x * c);
        }
        const float z = gelu_erf(s + few_get<V>(a.b1, r0 + r));
        few_put<V>(a.z, (int64_t)(t0 + m) * a.H + r0 + r, z);
        if (few_parts(V, NT) == 2) {  // what an infinity leaves is nothing
            const float hi = bf16_to_f32(f32_to_bf16(z));
            few_put<V>(a.z, (int64_t)(a.T + t0 + m) * a.H + r0 + r, isinf(hi) ? 0.f : z - hi);
        }
    }
}

// A tile's product for tokens s_tok[0 .. n), n <= few_pass(PARTS, NT), into their output rows. early: the weights of its first steps,
// already asked for (HAVE of them).
constexpr int FEW_EARLY = 4;
template <int V, int NT, int PARTS, int CTAS, int HAVE>
__device__ __forceinline__ void few_expert(const FewArgs& a, int e, int r0, const int* s_tok, int n, float* red, const uint8_t* s_scale,
                                           const uint4 (&early)[2][FEW_EARLY], int warp, int lane) {
    FewTile<V, NT, CTAS> t;
    t.set_weights(a.Wc[e], few_pitch<V>(a.H), r0, a.d, a.H);
#pragma unroll
    for (int d = 0; d < FewT<V, NT, CTAS>::DW; ++d) {
        if (d < HAVE)
            t.a[d] = early[0][d], t.b[d] = early[1][d];
        else
            t.load_w(d, d);
    }
    float acc[NT][4], sums[4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int col = 8 * j + (lane >> 2), part = col % PARTS;
        t.set_row(j, static_cast<const char*>(a.z) + (int64_t)(part * a.T + s_tok[min(col / PARTS, n - 1)]) * a.H * FewT<V, NT, CTAS>::XSZ);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    }
    t.start_x();
    if (V == FEWV_W8A16) __syncthreads();  // the scales
    few_product<V, NT, CTAS, false>(acc, sums, t, s_scale, nullptr, 0, n);
    if constexpr (PARTS == 2)
        few_stage_pairs<NT>(red, acc, warp, lane);
    else
        few_stage<NT>(red, acc, warp, lane);
    __syncthreads();
    for (int i = threadIdx.x; i < n * 16; i += FewT<V, NT, CTAS>::THREADS) {
        const int j = i >> 4, r = i & 15;
        if (r0 + r >= a.d) continue;
        float s = few_sum<few_pass(PARTS, NT), FewT<V, NT, CTAS>::WARPS>(red, j, r);
        if (a.b2) s += few_get<V>(a.b2, r0 + r);
        few_put<V>(a.out, (int64_t)s_tok[j] * a.d + r0 + r, s);
    }
}

// One CTA per 16 output rows and group, NT token tiles at most at a time; more tokens than that go through in turns, the
// weights then coming from L2. GUESS (as many tokens as groups or more): the first weights are asked for before the
// routing is known, beside fc1, as if the group had tokens.
template <int V, int NT, int CTAS, bool GUESS>
__global__ void __launch_bounds__(FewT<V, NT, CTAS>::THREADS, CTAS) few_expert_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float red[];  // the partial sums; then the scale bytes
    __shared__ int s_tok[CLEARMOE_FEW_MAX];
    __shared__ int s_n;
    uint8_t* s_scale = reinterpret_cast<uint8_t*>(red) + FewT<V, NT, CTAS>::SMEM;
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int e = blockIdx.y, r0 = blockIdx.x * 16;
    // z in two parts halves a pass; where the registers of one CTA an SM allow it, twice the tiles make up for it
    constexpr int PARTS = few_parts(V, NT), WIDE = PARTS == 2 && NT == 2 && CTAS == 1 ? 4 : NT;
    // the steps that every width of the product starts with
    constexpr int HAVE = !GUESS ? 0 : FewT<V, WIDE, CTAS>::DW < FEW_EARLY ? FewT<V, WIDE, CTAS>::DW : FEW_EARLY;
    uint4 early[2][FEW_EARLY];
    if (GUESS) {
        FewTile<V, 1, CTAS> t;
        t.set_weights(a.Wc[e], few_pitch<V>(a.H), r0, a.d, a.H);
#pragma unroll
        for (int d = 0; d < HAVE; ++d) {
            t.load_w(d, d);
            early[0][d] = t.a[d], early[1][d] = t.b[d];
        }
    }
    few_scales<V>(s_scale, a.Wc_s[e], r0, a.H);
    pdl_wait();
    if (warp == 0) {  // the group's tokens in order, two a lane; their number before it
        const int v0 = lane < a.T ? __ldcg(a.idx + lane) : a.G, v1 = lane + 32 < a.T ? __ldcg(a.idx + lane + 32) : a.G;
        const uint32_t b0 = __ballot_sync(0xFFFFFFFFu, v0 == e), b1 = __ballot_sync(0xFFFFFFFFu, v1 == e);
        const uint32_t below = (1u << lane) - 1;
        const int at0 = __popc(b0 & below), at1 = __popc(b0) + __popc(b1 & below), n = __popc(b0) + __popc(b1);
        if (v0 == e) s_tok[at0] = lane;
        if (v1 == e) s_tok[at1] = lane + 32;
        if (lane == 0) s_n = n;
        if (blockIdx.x == 0) {  // counts, offsets and perm, as the other forwards leave them
            const int before = __popc(__ballot_sync(0xFFFFFFFFu, v0 < e)) + __popc(__ballot_sync(0xFFFFFFFFu, v1 < e));
            if (v0 == e) a.perm[before + at0] = lane;
            if (v1 == e) a.perm[before + at1] = lane + 32;
            if (lane == 0) {
                a.counts[e] = n;
                a.offsets[e] = before;
                if (e + 1 == a.G) a.offsets[a.G] = a.T;
            }
        }
    }
    __syncthreads();
    constexpr int PASS = few_pass(PARTS, WIDE), P = few_pass(PARTS, 1);
    int n = min(PASS, s_n);
    if (n == 0) return;
    if (NT == 1 || n <= P)
        few_expert<V, 1, PARTS, CTAS, HAVE>(a, e, r0, s_tok, n, red, s_scale, early, warp, lane);
    else if (WIDE == 2 || n <= 2 * P)
        few_expert<V, NT < 2 ? NT : 2, PARTS, CTAS, HAVE>(a, e, r0, s_tok, n, red, s_scale, early, warp, lane);
    else
        few_expert<V, WIDE, PARTS, CTAS, HAVE>(a, e, r0, s_tok, n, red, s_scale, early, warp, lane);
    for (int m0 = PASS; m0 < s_n; m0 += PASS) {
        __syncthreads();  // red is read
        n = min(PASS, s_n - m0);
        few_expert<V, WIDE, PARTS, CTAS, 0>(a, e, r0, s_tok + m0, n, red, s_scale, early, warp, lane);
    }
}

template <typename K, typename... A>
cudaError_t few_launch(K kernel, dim3 grid, int threads, int smem, cudaStream_t s, const A&... a) {
    const cudaError_t e = smem_attr_once((const void*)kernel, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a...);
}

template <int V, int NT, int CTAS>
cudaError_t few_fc1(const FewArgs& a, cudaStream_t s) {
    const dim3 grid((a.H + 15) / 16 + (a.T + few_route_tokens(NT) - 1) / few_route_tokens(NT), (a.T + few_chunk(NT) - 1) / few_chunk(NT));
    const int smem = FewT<V, NT, CTAS>::SMEM + (V == FEWV_W8A16 ? (a.d + 127) / 128 : 0);
    return a.ln ? few_launch(few_fc1_kernel<V, NT, CTAS, true>, grid, FEW_THREADS, smem, s, a)
                : few_launch(few_fc1_kernel<V, NT, CTAS, false>, grid, FEW_THREADS, smem, s, a);
}
template <int V, int NT, int CTAS>
cudaError_t few_experts(const FewArgs& a, cudaStream_t s) {
    const dim3 grid((a.d + 15) / 16, a.G);
    const int smem = FewT<V, NT, CTAS>::SMEM + (V == FEWV_W8A16 ? (a.H + 127) / 128 : 0);
    constexpr int threads = FewT<V, NT, CTAS>::THREADS;
    static_assert(CM_MAX_E <= 16);
    if constexpr (NT < 4)  // four tiles: more than 16 tokens, as many as groups or more
        if (a.T < a.G) return few_launch(few_expert_kernel<V, NT, CTAS, false>, grid, threads, smem, s, a);
    return few_launch(few_expert_kernel<V, NT, CTAS, true>, grid, threads, smem, s, a);
}

template <int V>
cudaError_t few_type(const FewArgs& a, cudaStream_t s) {
    const cudaError_t e = a.T <= 8 ? few_fc1<V, 1, 2>(a, s) : a.T <= 16 ? few_fc1<V, 2, 2>(a, s) : few_fc1<V, 4, 2>(a, s);
    if (e != cudaSuccess) return e;
    if (a.T <= 4) return few_experts<V, 1, 2>(a, s);
    const bool lone = (int64_t)((a.d + 15) / 16) * (a.T < a.G ? a.T : a.G) <= a.num_sms;  // an SM for each CTA with work
    // us, lone CTAs of 16 warps against two or three of 8 an SM: 8 tokens, d = 384, 4 experts, bf16 4.5 / 4.9; 24, d = 384, 6, fp32
    // 9.3 / 10.2; 16, d = 768, 3, bf16 7.0 / 10.1; more CTAs than SMs: 13, d = 768, 9, bf16 16.5 / 12.8; 64, 8 19.8 / 18.4
    if (lone) return a.T <= 16 ? few_experts<V, 2, 1>(a, s) : few_experts<V, 4, 1>(a, s);
    if constexpr (few_parts(V, 2) == 1)
        if (a.T <= 8) return few_experts<V, 1, 3>(a, s);
    return a.T <= 16 ? few_experts<V, 2, 3>(a, s) : few_experts<V, 4, 2>(a, s);
}

}  // namespace

cudaError_t launch_few(const FewArgs& a, cudaStream_t s) {
    return a.f32 ? few_type<FEWV_F32>(a, s) : a.fp8 ? few_type<FEWV_W8A16>(a, s) : few_type<FEWV_BF16>(a, s);
}

}  // namespace cm
