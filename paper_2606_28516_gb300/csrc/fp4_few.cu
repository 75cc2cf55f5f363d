// Products of matrices in 4-bit blocks with few rows of activations (1 to FP4_FEW_MAX): reading the weights once is all
// there is to it, and an output tile of 128 rows would be mostly empty. So the operands change places: 128 rows of W are the
// MMA's M, the NT rows of A its N, and a cluster of CTAs splits K, so that every SM reads weights. Each CTA asks for all the
// stages it has room for at once; its sums go to shared memory, and CTA r of the cluster adds the parts of every KS-th row
// of A in CTA order (the result does not depend on which comes first) and finishes it.
//
//   4 warps      epilogue: TMEM lane quarters (32 columns of the output each) to shared memory, then the sums over the cluster,
//                a row a warp, four columns a lane
//   1 warp       TMEM allocation, tcgen05.cp of the scales, tcgen05.mma and commits
//   1 warp       TMA producer
// Waits are bounded as in fp4_gemm.cu; a CTA that gave up still takes part in the cluster's two barriers.
#include <cstdint>

#include "common.cuh"
#include "fp4.cuh"
#include "fp4_gemm.cuh"
#include "internal.h"
#include "pair.cuh"

namespace cm {

namespace {

constexpr int FEW_PREFETCH = 16;  // stages

template <int NT_>
struct FewCfg {
    static constexpr int NT = NT_;
    static constexpr int THREADS = 192;
    static constexpr int W_BYTES = 128 * 128, X_BYTES = NT * 128;
    static constexpr int STAGE_BYTES = W_BYTES + X_BYTES + 2 * F4_SF;
    static constexpr int STAGES = 108 * 1024 / STAGE_BYTES;  // two CTAs an SM
    static constexpr int SF_COL = NT;
    static constexpr int TMEM_COLS = NT + 16 <= 32 ? 32 : NT + 16 <= 64 ? 64 : NT + 16 <= 128 ? 128 : 256;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + 8 * (2 * STAGES + 1) + 16;
    static_assert(128 * NT * 4 <= STAGES * STAGE_BYTES);  // the sums, once the stages are read
    static_assert(SMEM <= 113 * 1024);
};

__device__ __forceinline__ void umma_few(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
                                         uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr_cluster) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr_cluster) : "memory");
    return v;
}

// The sums of row m and columns n .. n + 3, four a lane, to the output; vec: its rows are in whole pieces of four.
template <int KIND>
__device__ __forceinline__ void finish(const Fp4GemmArgs<1>& a, float4 s, const float4& bias, int m, int n, bool vec, int lane) {
    float v[4] = {s.x + bias.x, s.y + bias.y, s.z + bias.z, s.w + bias.w};
    if (a.act == CLEARMOE_ACT_GELU) {
        if constexpr (KIND == FP8_OUT_F32) {  // f8_act's of the tiles' epilogues
            const float2 p = gelu_pair_f32(make_float2(v[0], v[1])), q = gelu_pair_f32(make_float2(v[2], v[3]));
            v[0] = p.x, v[1] = p.y, v[2] = q.x, v[3] = q.y;
        } else {
            gelu_pairs_bf16<2>(v);
        }
    } else if (a.act == CLEARMOE_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];  // NaN stays NaN
    }
    if constexpr (KIND == FP4_OUT_FP4) {  // eight lanes' columns are a block
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i >= a.N) v[i] = 0.f;
        float top = max_abs3(max_abs(v[0], v[1]), v[2], v[3]);
#pragma unroll
        for (int o = 4; o; o >>= 1) top = max_abs(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        const uint32_t scale = fp4_scale_byte(abs_bits(top));
        const float inv = fp8_inverse_scale(scale);
        if (n / 2 >= a.ldo) return;
        *reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(a.out) + (int64_t)m * a.ldo + n / 2) =
            (uint16_t)fp4_pack8(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv, 0.f, 0.f, 0.f, 0.f);
        if ((lane & 7) == 0) a.out_scale[fp4_scale_word(m, n >> 7, a.ldos) + (n >> 5 & 3)] = (uint8_t)scale;
    } else {
        constexpr bool BF16 = KIND == FP8_OUT_BF16;
        uint16_t* b = static_cast<uint16_t*>(a.out) + (int64_t)m * a.ldo + n;
        float* f = static_cast<float*>(a.out) + (int64_t)m * a.ldo + n;
        if (vec && n + 4 <= a.N) {
            if constexpr (BF16)
                *reinterpret_cast<uint2*>(b) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
            else
                *reinterpret_cast<float4*>(f) = make_float4(v[0], v[1], v[2], v[3]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= a.N) break;
            if constexpr (BF16)
                b[i] = f32_to_bf16(v[i]);
            else
                f[i] = v[i];
        }
    }
}

template <int NT_, int KIND>
__global__ void __launch_bounds__(FewCfg<NT_>::THREADS, 2) fp4_few_kernel(const __grid_constant__ Fp4GemmArgs<1> a, const int split) {
    using C = FewCfg<NT_>;
    constexpr int NT = C::NT, STAGES = C::STAGES;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    float* s_sum = reinterpret_cast<float*>(sm);  // [row of A][column], over the stages
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + STAGES * C::STAGE_BYTES);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = warp_uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), n0 = (int)(blockIdx.x / split) * 128;
    const int kb0 = (int)((int64_t)a.nkb * rank / split), kb1 = (int)((int64_t)a.nkb * (rank + 1) / split);
    const uint32_t bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    const uint32_t done_bar = bar0 + 8u * (2 * STAGES);
    const uint64_t lim = (uint64_t)a.wait_limit_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 4 && lane == 0) f4_prefetch_maps(a);
    if (warp == 5) tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    if (warp == 0 && kb1 - kb0 > STAGES) {  // weights enough that their time counts (3 x 8,192 x 8,192 behind a norm: 11.5 -> 10.2 us)
        for (int kb = kb0; kb < min(kb1, kb0 + FEW_PREFETCH); ++kb) {
            l2_prefetch_2d(&a.tmB[0], kb * 64, n0);
            l2_prefetch_2d(&a.tmSB[0], kb * 256, n0 >> 7);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();  // everything below may read the previous kernel's results
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    const uint32_t tmem = warp_uniform(*tmem_slot);

    if (warp == 4) {
        // ------------------------------------------------ TMA producer
        int stage = 0;
        uint32_t ph = 0, issued = 0, par = 0;  // bit s: stage s has had a load; parity of its last
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait_warp(empty_bar(stage), ph ^ 1, abort_flag, a.status, lim)) break;
            const uint32_t sW = smem_u32(sm + stage * C::STAGE_BYTES), sX = sW + C::W_BYTES, sF = sX + C::X_BYTES;
            mbar_arrive_expect_tx_warp(full_bar(stage), C::STAGE_BYTES);
            // coordinates in the maps' elements: 16-bit ones of four columns, 32-bit ones of four scales
            tma_load_2d(sW, &a.tmB[0], kb * 64, n0, full_bar(stage));
            tma_load_2d(sF, &a.tmSB[0], kb * 256, n0 >> 7, full_bar(stage));
            tma_load_2d(sX, &a.tmA, kb * 64, 0, full_bar(stage));
            tma_load_2d(sF + F4_SF, &a.tmSA, kb * 256, 0, full_bar(stage));
            issued |= 1u << stage;
            par = (par & ~(1u << stage)) | (ph << stage);
            if (++stage == STAGES) {
                stage = 0;
                ph ^= 1;
            }
        }
        // let every copy in flight land before the CTA retires, whoever gave up
        for (int s = 0; s < STAGES; ++s)
            if (issued & (1u << s)) mbar_wait_warp(full_bar(s), (par >> s) & 1, nullptr, a.status, lim + 10000000ull);
    } else if (warp == 5) {
        // ------------------------------------------------ MMA issuer
        int stage = 0;
        uint32_t ph = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait_warp(full_bar(stage), ph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t sW = smem_u32(sm + stage * C::STAGE_BYTES), sF = sW + C::W_BYTES + C::X_BYTES;
            const uint64_t wd = sdesc_kmajor_sw128(sW), xd = sdesc_kmajor_sw128(sW + C::W_BYTES);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // 128 columns, a word of scales
                if (4 * kb + 2 * h >= a.ksteps) break;
                const uint32_t sf = tmem + C::SF_COL + 8 * h;
                tmem_cp_scales<1>(sf, sF + 512 * h);
                tmem_cp_scales<1>(sf + 4, sF + F4_SF + 512 * h);
#pragma unroll
                for (int j = 0; j < 2; ++j) {  // 64 columns: 32 bytes on in each row
                    const int k = 2 * h + j;
                    if (4 * kb + k < a.ksteps) umma_few(tmem, wd + 2 * k, xd + 2 * k, idesc_mxf4(128, NT, j), sf, sf + 4, kb > kb0 || k);
                }
            }
            umma_commit(empty_bar(stage));
            if (++stage == STAGES) {
                stage = 0;
                ph ^= 1;
            }
        }
        umma_commit(done_bar);  // every MMA issued above has completed once this fires
        mbar_wait_warp(done_bar, 0, nullptr, a.status, lim + 10000000ull);
    }
    __syncthreads();  // every copy has landed and every MMA is done: the stages are free
    tc_fence_after();
    if (warp < 4) {
#pragma unroll
        for (int c = 0; c < NT; c += 16) {
            uint32_t u[16];
            CM_TMEM_LD_X16(tmem + ((uint32_t)(warp * 32) << 16) + c, u);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) s_sum[(c + i) * 128 + warp * 32 + lane] = __uint_as_float(u[i]);
        }
    }
    tc_fence_before();
    cluster_sync();  // every CTA's sums are in its shared memory
    tc_fence_after();
    if (warp < 4) {
        // Row rank + split j is warp j % 4's, four columns a lane; every CTA's part of it is asked for before the first is added.
        const int n = n0 + 4 * lane;
        float4 bias = make_float4(0.f, 0.f, 0.f, 0.f);
        if (a.bias) {
            float b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                b[i] = n + i >= a.N  ? 0.f
                       : a.bias_bf16 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(a.bias) + n + i))
                                     : __ldcg(static_cast<const float*>(a.bias) + n + i);
            bias = make_float4(b[0], b[1], b[2], b[3]);
        }
        const int piece = KIND == FP8_OUT_BF16 ? 8 : 16;
        const bool vec = (reinterpret_cast<uintptr_t>(a.out) & (piece - 1)) == 0 && a.ldo % 4 == 0;
        uint32_t part[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) part[r] = map_to_rank(smem_u32(s_sum + 4 * lane), r < split ? r : 0);
        constexpr int R = NT == 16 ? 1 : 2;  // rows of a warp at a time
        for (int m0 = rank + split * warp; m0 < (int)a.M; m0 += 4 * R * split) {
            float4 p[R][8];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int m = min(m0 + 4 * i * split, (int)a.M - 1);
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < split) p[i][r] = ld_cluster_f32x4(part[r] + m * 512);
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int m = m0 + 4 * i * split;
                if (m >= (int)a.M) break;
                float4 v = p[i][0];
#pragma unroll
                for (int r = 1; r < 8; ++r)
                    if (r < split) v = make_float4(v.x + p[i][r].x, v.y + p[i][r].y, v.z + p[i][r].z, v.w + p[i][r].w);
                finish<KIND>(a, v, bias, m, n, vec, lane);
            }
        }
    }
    cluster_sync();  // nobody reads this CTA's shared memory any more
    if (warp == 5) tmem_dealloc(tmem, C::TMEM_COLS);
}

template <int NT, int KIND>
cudaError_t launch_kind(const Fp4GemmArgs<1>& a, int split, cudaStream_t s) {
    using C = FewCfg<NT>;
    const cudaError_t e = smem_attr_once((const void*)fp4_few_kernel<NT, KIND>, C::SMEM);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.N + 127) / 128 * split));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)split;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, fp4_few_kernel<NT, KIND>, a, split);
}
template <int NT>
cudaError_t launch_nt(const Fp4GemmArgs<1>& a, int split, cudaStream_t s) {
    return a.out_kind == FP4_OUT_FP4    ? launch_kind<NT, FP4_OUT_FP4>(a, split, s)
           : a.out_kind == FP8_OUT_BF16 ? launch_kind<NT, FP8_OUT_BF16>(a, split, s)
                                        : launch_kind<NT, FP8_OUT_F32>(a, split, s);
}

}  // namespace

int fp4_few_rows(int64_t M) { return M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128; }

// CTAs that share a tile's K: as many as leave each an SM and two stages; where the stages a CTA asks for at once are then
// less than its part, two CTAs an SM. 4 x 4,096 x 4,096: four CTAs of four stages 3.8 us, eight of two 4.2, two 4.4; 16 x
// 1,024 x 4,096: eight 3.3, four 3.6; 3 x 8,192 x 8,192: four CTAs, two an SM, 8.5, two 9.0; 32 x 2,048 x 2,048: four of two
// stages 3.2, eight of one 4.8.
static int few_split(int N, int nkb, int num_sms) {
    const int tiles = (N + 127) / 128, stages = FewCfg<16>::STAGES;
    int split = num_sms / tiles;
    if (split < 1 || nkb > split * stages) split = 2 * num_sms / tiles;
    split = split > 8 ? 8 : split;
    split = split > nkb / 2 ? nkb / 2 : split;
    return split < 1 ? 1 : split;
}

// Whether the kernel is the better one: of the 0.17 us that a stage of K takes a tile of 64 columns and 128 rows, the
// cluster saves all but its split's part; joining its sums takes 0.35 us, and 0.025 a row. Us, this kernel and that one:
// 1 x 1,024 x 4,096 3.1, 4.8; 16 x 4,096 x 4,096 3.8, 4.8; 64 x 1,024 x 4,096 4.1, 4.9; 100 x 512 x 8,192 5.7, 7.6; otherwise
// 1 x 768 x 768 2.9, 2.3; 16 x 8,192 x 2,048 4.0, 3.7; 64 x 2,048 x 2,048 4.1, 3.5; 100 x 4,096 x 4,096 6.3, 5.6.
bool fp4_few_pays(int64_t M, int N, int nkb, int num_sms) {
    const int64_t split = few_split(N, nkb, num_sms);
    // with two CTAs an SM the weights are what takes time: 32 x 8,192 x 8,192 9.5 us against 9.6, 64 x 8,192 x 8,192 10.4 against 9.8
    if (M > ((N + 127) / 128 * split > num_sms ? 32 : FP4_FEW_MAX)) return false;
    return 7 * nkb * (split - 1) > (M + 14) * split;
}

cudaError_t launch_fp4_few(const Fp4GemmArgs<1>& a, int num_sms, cudaStream_t s) {
    const int split = few_split(a.N, a.nkb, num_sms);
    const int nt = fp4_few_rows(a.M);
    return nt == 16   ? launch_nt<16>(a, split, s)
           : nt == 32 ? launch_nt<32>(a, split, s)
           : nt == 64 ? launch_nt<64>(a, split, s)
                      : launch_nt<128>(a, split, s);
}

}  // namespace cm
