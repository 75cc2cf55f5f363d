// Products of matrices in 4-bit blocks on the 5th-generation tensor cores (tcgen05, sm_103a):
//
//   C[m, n] = epilogue( sum_b 2^(sa[m, b] + sw[n, b] - 254) sum_{k in block b} qa[m, k] qw[n, k] )
//
// kind::mxf4 with block scales multiplies 64 columns an MMA and takes one power-of-two scale per row and 32 of them from
// tensor memory: two bytes of the word that holds a row's four scales of 128 columns. The scales of 128 rows x 128
// columns lie in global memory as tcgen05.cp wants them in shared memory, so that they come with the tiles they belong
// to, by the same producer and on the same barrier, and no warp handles them.
//
// One persistent, warp-specialised kernel per N tile width:
//   epilogue     16 warps, 8 for 64 columns: warp w reads TMEM lane quarter w % 4 (its 32 rows), 32 columns at a time;
//   1 warp       TMEM allocation, tcgen05.cp of the scales, tcgen05.mma and commits (the whole warp in step, one
//                elected lane issues);
//   1 warp       TMA producer: 128 rows of A and BN of W, 128 bytes each (256 columns), 128-byte swizzle, and their scales.
// Grouped products walk (group, row tile, column tile) from the device-resident offsets. Every wait is bounded; a CTA that
// gives up records CLEARMOE_ETIMEOUT, lets its copies and MMAs in flight finish, frees its tensor memory and returns.
#include <cstdint>
#include <cstring>

#include "common.cuh"
#include "fp4.cuh"
#include "fp4_gemm.cuh"
#include "internal.h"

namespace cm {

namespace {

constexpr int F4_BM = 128;

template <int BN_>
struct F4Cfg {
    static constexpr int BN = BN_;
    static constexpr int NUM_EPI = BN >= 128 ? 16 : 8, SPAN = NUM_EPI / 4;  // warps per lane quarter
    static constexpr int WARP_MMA = NUM_EPI, WARP_TMA = NUM_EPI + 1;
    static constexpr int THREADS = 32 * (NUM_EPI + 2);
    static constexpr int A_BYTES = F4_BM * 128, B_BYTES = BN * 128;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + 2 * F4_SF;  // q of A and W, then their scales
    static constexpr int STAGES = 200 * 1024 / STAGE_BYTES < 8 ? 200 * 1024 / STAGE_BYTES : 8;
    static constexpr int NBARS = 2 * STAGES + 4 + 1;
    static constexpr int SF_COL = 2 * BN;  // scale columns: two slots of A's four and W's four
    static constexpr int TMEM_COLS = SF_COL + 16 <= 256 ? 256 : 512;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + NUM_EPI * 32 * 4 + NBARS * 8 + 16 + 8 * (CM_MAX_E + 1);
    static_assert(STAGE_BYTES % 1024 == 0);
};

__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
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
// KIND: FP8_OUT_F32, FP8_OUT_BF16 or FP4_OUT_FP4.
template <int BN_, int KIND, int NE>
__global__ void __launch_bounds__(F4Cfg<BN_>::THREADS, 1) fp4_gemm_kernel(const __grid_constant__ Fp4GemmArgs<NE> a) {
    using C = F4Cfg<BN_>;
    constexpr int BN = C::BN;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    float* s_bias = reinterpret_cast<float*>(sm + C::STAGES * C::STAGE_BYTES);  // [epilogue warp][32]
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_bias + C::NUM_EPI * 32);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NBARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    int* s_prefix = reinterpret_cast<int*>(tmem_slot + 4);  // [E + 1]
    int* s_off = s_prefix + CM_MAX_E + 1;                   // [E + 1]

    const int warp = warp_uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto tfull_bar = [&](int i) { return bar0 + 8u * (2 * C::STAGES + i); };
    auto tempty_bar = [&](int i) { return bar0 + 8u * (2 * C::STAGES + 2 + i); };
    const uint32_t drain_bar = bar0 + 8u * (2 * C::STAGES + 4);
    const uint64_t lim = (uint64_t)a.wait_limit_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull_bar(i), 1);
            mbar_init(tempty_bar(i), C::NUM_EPI);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == C::WARP_TMA && lane == 0) f4_prefetch_maps(a);
    if (warp == C::WARP_MMA) tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr bool GROUPED = Fp4GemmArgs<NE>::GROUPED;
    auto begin = [&]() {
        pdl_wait();  // everything below may read the previous kernel's results
        pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    };
    if constexpr (GROUPED) {
        begin();
        if (warp == 0) f4_groups(a, F4_BM, s_off, s_prefix, lane);
        __syncthreads();
    }
    const uint32_t tmem = warp_uniform(*tmem_slot);
    F4Walk<GROUPED> t(blockIdx.x, gridDim.x, a, F4_BM, BN, s_off, s_prefix);
    if constexpr (!GROUPED) begin();
    const int nkb = a.nkb;

    if (warp == C::WARP_TMA) {
        // ------------------------------------------------ TMA producer
        int stage = 0;
        uint32_t ph = 0, issued = 0, par = 0;  // bit s: stage s has had a load; parity of its last
        bool ok = true;
        for (; warp_uniform((int)t.live()) && ok; t.next()) {
            const int e = warp_uniform(t.e), n0 = warp_uniform(t.n0), m0 = warp_uniform(t.m0);
            for (int kb = 0; kb < nkb; ++kb) {
                if (!mbar_wait_warp(empty_bar(stage), ph ^ 1, abort_flag, a.status, lim)) {
                    ok = false;
                    break;
                }
                const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES), sB = sA + C::A_BYTES, sF = sB + C::B_BYTES;
                mbar_arrive_expect_tx_warp(full_bar(stage), a.box_rows * 128 + C::B_BYTES + 2 * F4_SF);
                // coordinates in the maps' elements: 16-bit ones of four columns, 32-bit ones of four scales
                tma_load_2d(sA, &a.tmA, kb * 64, m0, full_bar(stage));
                tma_load_2d(sB, &a.tmB[e], kb * 64, n0, full_bar(stage));
                tma_load_2d(sF, &a.tmSA, kb * 256, m0 >> 7, full_bar(stage));
                tma_load_2d(sF + F4_SF, &a.tmSB[e], kb * 256, n0 >> 7, full_bar(stage));
                issued |= 1u << stage;
                par = (par & ~(1u << stage)) | (ph << stage);
                if (++stage == C::STAGES) {
                    stage = 0;
                    ph ^= 1;
                }
            }
        }
        // let every copy in flight land before the CTA retires, whoever gave up
        for (int s = 0; s < C::STAGES; ++s)
            if (issued & (1u << s)) mbar_wait_warp(full_bar(s), (par >> s) & 1, nullptr, a.status, lim + 10000000ull);
    } else if (warp == C::WARP_MMA) {
        // ------------------------------------------------ MMA issuer
        int stage = 0, acc = 0;
        uint32_t ph = 0, aph = 0;
        bool ok = true;
        for (; warp_uniform((int)t.live()) && ok; t.next()) {
            if (!mbar_wait_warp(tempty_bar(acc), aph ^ 1, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + acc * BN;
            const int at = warp_uniform(t.n0 >> 5 & 3);  // W's first column of scales in its tile of 128 rows
            for (int kb = 0; kb < nkb; ++kb) {
                if (!mbar_wait_warp(full_bar(stage), ph, abort_flag, a.status, lim)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES), sF = sA + C::A_BYTES + C::B_BYTES;
                const uint64_t ad = sdesc_kmajor_sw128(sA), bd = sdesc_kmajor_sw128(sA + C::A_BYTES);
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // 128 columns, a word of scales
                    if (4 * kb + 2 * h >= a.ksteps) break;
                    const uint32_t sf = tmem + C::SF_COL + 8 * h;
                    tmem_cp_scales<1>(sf, sF + 512 * h);
                    tmem_cp_scales<1>(sf + 4, sF + F4_SF + 512 * h);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {  // 64 columns: 32 bytes on in each row
                        const int k = 2 * h + j;
                        if (4 * kb + k < a.ksteps) umma_mxf4(d, ad + 2 * k, bd + 2 * k, idesc_mxf4(F4_BM, BN, j), sf, sf + 4 + at, (kb | k) != 0);
                    }
                }
                umma_commit(empty_bar(stage));
                if (++stage == C::STAGES) {
                    stage = 0;
                    ph ^= 1;
                }
            }
            if (!ok) break;
            umma_commit(tfull_bar(acc));
            if (++acc == 2) {
                acc = 0;
                aph ^= 1;
            }
        }
        umma_commit(drain_bar);  // every MMA issued above has completed once this fires
        mbar_wait_warp(drain_bar, 0, nullptr, a.status, lim + 10000000ull);
    } else {
        // ------------------------------------------------ epilogue
        // warp w takes 32-column chunks w / 4, w / 4 + SPAN, .. of the tile
        constexpr int SPAN = C::SPAN, ROUNDS = (BN / 32 + SPAN - 1) / SPAN;
        static_assert(ROUNDS * SPAN * 32 == BN);
        const int quarter = warp & 3, cg = warp >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float* bias_line = s_bias + warp * 32;
        const bool has_bias = a.bias != nullptr;
        const bool wide = f8_wide(a);
        int acc = 0;
        uint32_t aph = 0;
        for (; t.live(); t.next()) {
            const int orow = f4_out_row(a, t.m0 + quarter * 32 + lane, t.lo, t.hi);
            float b[ROUNDS];
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int n = t.n0 + (SPAN * r + cg) * 32 + lane;
                b[r] = 0.f;
                if (has_bias && n < a.N)
                    b[r] = a.bias_bf16 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(a.bias) + n))
                                       : __ldcg(static_cast<const float*>(a.bias) + n);
            }
            if (!mbar_wait_warp(tfull_bar(acc), aph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + lanes + acc * BN;
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int nc = t.n0 + (SPAN * r + cg) * 32;
                float v[32];
                __syncwarp();  // the bias line is read, rows without a store have caught up
                uint32_t u[32];
                CM_TMEM_LD_X32(d + (SPAN * r + cg) * 32, u);
                if (has_bias) bias_line[lane] = b[r];
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
                if (r + 1 == ROUNDS) tc_fence_before();
                __syncwarp();
                if (r + 1 == ROUNDS && lane == 0) mbar_arrive(tempty_bar(acc));  // the accumulator is read
                f8_act<32, KIND == FP8_OUT_F32 ? GELU_F32 : GELU_BF16>(v, bias_line, has_bias, a.act);
                f4_store32<KIND>(a, v, orow, nc, wide, lane);
            }
            if (++acc == 2) {
                acc = 0;
                aph ^= 1;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == C::WARP_MMA) tmem_dealloc(tmem, C::TMEM_COLS);
}

template <int BN, int KIND, int NE>
cudaError_t launch_bn(const Fp4GemmArgs<NE>& a, int num_sms, cudaStream_t s) {
    using C = F4Cfg<BN>;
    static_assert(C::SMEM <= 227 * 1024);
    const cudaError_t e = smem_attr_once((const void*)fp4_gemm_kernel<BN, KIND, NE>, C::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t m_tiles = (a.M + F4_BM - 1) / F4_BM + a.E - 1;
    const int64_t tiles = m_tiles * ((a.N + BN - 1) / BN);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles < num_sms ? tiles : num_sms));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fp4_gemm_kernel<BN, KIND, NE>, a);
}

template <int BN, int NE>
cudaError_t launch_kind(const Fp4GemmArgs<NE>& a, int num_sms, cudaStream_t s) {
    if constexpr (NE == 1) {
        if (a.out_kind == FP4_OUT_FP4) return launch_bn<BN, FP4_OUT_FP4>(a, num_sms, s);
    }
    return a.out_kind == FP8_OUT_BF16 ? launch_bn<BN, FP8_OUT_BF16>(a, num_sms, s) : launch_bn<BN, FP8_OUT_F32>(a, num_sms, s);
}

// Stages of K up to which bf16 rows leave by bulk copies: 8,192 x 4,096 x 1,024 22.9 us by the lanes' stores, 18.8 so. Longer
// K wants the shared memory for one stage more: 16,384 x 4,096 x 4,096 76 us against 81.
constexpr int BULK_NKB = 8;

// The kernel that tests have fixed for their thread's calls (width << 1 | pair), or 0.
thread_local int g_forced = 0;
constexpr int64_t WAIT_LIMIT_NS = 1000000000LL;
thread_local int64_t g_wait = WAIT_LIMIT_NS;  // of their waits

constexpr int FEW_WIDTH = 16;  // stands for the kernel for few rows
struct Pick {
    int bn, pair;
};
// Cycles (at 1.9 GHz) a product takes on a kernel: its start; rounds of tiles, each of which multiplies its stages or, where
// that is longer, runs the epilogue of the tile before it; and a part of the last epilogue. A round of halves of tiles
// (256 columns on pairs) counts 0.6. A stage's cycles grow from what the MMAs and their scales take to what the path from L2
// allows with every SM at work. Fitted to 99 products of 8 to 16,384 rows; what the rule chooses is 0.5 % slower than the
// best kernel in the mean, 7 % at the most. In us, (64, 0), (128, 0), (128, 1), (256, 1) at M x N x K: 197 x 1,536 x 384 with
// bias and GELU 3.0, 3.9, 3.9, 5.4; 788 x 768 x 2,048 3.7, 4.5, 4.6, 6.1; 1,970 x 2,304 x 768 5.5, 5.1, 5.5, 5.8; 6,000 x
// 384 x 1,536 5.2, 4.7, 5.5, 6.3; 2,048 x 4,096 x 4,096 24.4, 18.7, 16.5, 15.2; 4,096 x 4,096 x 4,096 45.3, 30.3, 25.9, 23.3.
// (Tiles of 192 columns on pairs were nowhere the best by more than 1 %.)
struct Fp4Kernel {
    Pick pick;
    int start, low, block, between;  // low, block: a stage's cycles on an idle GPU and with every SM at work
    int gelu;                        // bias and GELU, of a tile
    double last;                     // the part of the last epilogue that nothing runs beside
    int epilogue[4];                 // of a tile by the kind of its stores: bf16 and fp32 in whole 32-byte pieces, rows of any pitch, 4-bit
};
double cost(const Fp4Kernel& k, int64_t M, int N, int nkb, int store, bool gelu, int groups, int num_sms) {
    const int rows = k.pick.pair ? 256 : 128, units = k.pick.pair ? num_sms / 2 : num_sms;
    if (units < 1) return 1e30;
    const int64_t tiles = ((M + rows - 1) / rows + groups - 1) * (((int64_t)N + k.pick.bn - 1) / k.pick.bn);
    const int64_t walkers = tiles < units ? tiles : units, rest = tiles % walkers;
    const double last = !rest ? 0.0 : k.pick.bn == 256 && 2 * rest <= walkers ? 0.6 : 1.0;  // of halves of tiles
    const double rounds = (double)(tiles / walkers) + last, busy = (double)walkers / units;
    const double main = nkb * (k.low + (k.block - k.low) * busy * busy), beside = k.epilogue[store] + (gelu ? k.gelu : 0);
    const double next = main + k.between > beside ? main + k.between : beside;
    return k.start + main + (rounds - 1) * next + k.last * beside;
}
template <int NE>
Pick pick(const Fp4GemmArgs<NE>& g, int num_sms) {
    static const Fp4Kernel all[] = {{{64, 0}, 3550, 326, 390, 321, 1140, 0.57, {1270, 2490, 2710, 1240}},
                                    {{128, 0}, 3090, 380, 546, 0, 1200, 0.96, {2440, 4040, 4560, 1930}},
                                    {{128, 1}, 5160, 273, 454, 387, 1160, 0.82, {1620, 3650, 4240, 1340}},
                                    {{256, 1}, 4920, 509, 747, 598, 2360, 0.90, {3030, 6870, 8690, 3050}}};
    if (NE == 1 && fp4_few_pays(g.M, g.N, g.nkb, num_sms)) return {FEW_WIDTH, 0};
    const int store = g.out_kind == FP4_OUT_FP4 ? 3 : !f8_wide(g) ? 2 : g.out_kind == FP8_OUT_F32 ? 1 : 0;
    Pick best = all[0].pick;
    double least = 1e30;
    for (const Fp4Kernel& k : all) {
        const double c = cost(k, g.M, g.N, g.nkb, store, g.act == CLEARMOE_ACT_GELU, g.E, num_sms);
        if (c < least) {
            least = c;
            best = k.pick;
        }
    }
    return best;
}

// Operands, epilogue and output of a product; fills g's epilogue fields.
template <int NE>
int check_gemm(const clearmoe_fp4* A, const clearmoe_fp4* W, int E, const clearmoe_fp8_epilogue* epi, Fp4GemmArgs<NE>& g) {
    std::memset(&g, 0, sizeof(g));
    int rc = check_fp4(A);
    if (rc) return rc;
    for (int e = 0; e < E; ++e) {
        if ((rc = check_fp4(W + e))) return rc;
        if (W[e].cols != A->cols || W[e].rows != W[0].rows || W[e].rows > (int64_t)1 << 24) return CLEARMOE_EINVAL;
    }
    g.act = CLEARMOE_ACT_NONE;
    g.wait_limit_ns = g_wait;
    if (epi) {
        if (epi->act != CLEARMOE_ACT_NONE && epi->act != CLEARMOE_ACT_RELU && epi->act != CLEARMOE_ACT_GELU)
            return CLEARMOE_EINVAL;
        if (epi->bias) {
            if (epi->bias_dtype != CLEARMOE_F32 && epi->bias_dtype != CLEARMOE_BF16) return CLEARMOE_EINVAL;
            if (reinterpret_cast<uintptr_t>(epi->bias) & (epi->bias_dtype == CLEARMOE_BF16 ? 1 : 3)) return CLEARMOE_EINVAL;
        }
        if (reinterpret_cast<uintptr_t>(epi->status) & 3) return CLEARMOE_EINVAL;
        g.bias = epi->bias;
        g.bias_bf16 = epi->bias_dtype == CLEARMOE_BF16;
        g.act = epi->act;
        g.status = epi->status;
    }
    return CLEARMOE_OK;
}

template <int NE>
int set_out(Fp4GemmArgs<NE>& g, void* out, int32_t dtype, int64_t ldo, int64_t N) {
    if (!out || (dtype != CLEARMOE_F32 && dtype != CLEARMOE_BF16) || ldo < N || ldo > (int64_t)1 << 30) return CLEARMOE_EINVAL;
    if (reinterpret_cast<uintptr_t>(out) & (dtype == CLEARMOE_BF16 ? 1 : 3)) return CLEARMOE_EINVAL;
    g.out = out;
    g.out_kind = dtype == CLEARMOE_BF16 ? FP8_OUT_BF16 : FP8_OUT_F32;
    g.ldo = ldo;
    return CLEARMOE_OK;
}

template <int NE>
int run(Fp4GemmArgs<NE>& g, const clearmoe_fp4* A, const clearmoe_fp4* W, int E, void* stream) {
    const int sms = current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    g.M = A->rows;
    g.N = (int)W[0].rows;
    g.ksteps = (int)((A->cols + 63) / 64);
    g.nkb = (g.ksteps + 3) / 4;
    g.E = E;
    const int64_t tiles = fp4_tiles(A->cols);
    Pick k = pick(g, sms);
    if (g_forced) k = {g_forced >> 1, g_forced & 1};
    const bool few = NE == 1 && k.bn == FEW_WIDTH && g.M <= FP4_FEW_MAX;
    if (k.bn == FEW_WIDTH) k.bn = few ? 128 : 64;
    const int wt = k.pair ? (k.bn + 127) / 128 : 1;  // scale tiles of a tile's columns
    const int64_t cols16 = fp4_ldq(A->cols) / 2;
    // Fewer rows than a tile: a box of those alone (the copy engine takes longer over a row past the end).
    g.box_rows = few ? fp4_few_rows(g.M) : !k.pair && g.M < F4_BM ? (int)(g.M + 7) / 8 * 8 : F4_BM;
    if (encode_tmap_bf16(&g.tmA, A->q, A->rows, cols16, g.box_rows)) return CLEARMOE_ECUDA;
    if (encode_tmap_fp4_scales(&g.tmSA, A->scale, (A->rows + 127) / 128, tiles, 1)) return CLEARMOE_ECUDA;
    // bf16 rows in order, in whole 16-byte pieces, leave by bulk copies where the epilogue is what takes time
    const int64_t pitch = g.ldo * 2;
    if (NE == 1 && k.pair && g.nkb <= BULK_NKB && g.out_kind == FP8_OUT_BF16 && pitch % 16 == 0 && (reinterpret_cast<uintptr_t>(g.out) & 15) == 0) {
        if (encode_tmap_out_bytes(&g.tmOut, g.out, g.M, (int64_t)g.N * 2, pitch)) return CLEARMOE_ECUDA;
        g.tma_out = 1;
    }
    for (int e = 0; e < E; ++e) {
        if (encode_tmap_bf16(&g.tmB[e], W[e].q, W[e].rows, cols16, k.pair ? k.bn / 2 : k.bn)) return CLEARMOE_ECUDA;
        if (k.pair && k.bn == 256 && encode_tmap_bf16(&g.tmH[e], W[e].q, W[e].rows, cols16, k.bn / 4)) return CLEARMOE_ECUDA;
        if (encode_tmap_fp4_scales(&g.tmSB[e], W[e].scale, (W[e].rows + 127) / 128, tiles, wt)) return CLEARMOE_ECUDA;
    }
    cudaError_t e;
    if constexpr (NE == 1) {
        e = few ? launch_fp4_few(g, sms, s) : k.pair ? launch_fp4_gemm2(g, k.bn, sms, s) : k.bn == 128 ? launch_kind<128>(g, sms, s) : launch_kind<64>(g, sms, s);
    } else {
        e = k.pair ? launch_fp4_gemm2(g, k.bn, sms, s) : k.bn == 128 ? launch_kind<128>(g, sms, s) : launch_kind<64>(g, sms, s);
    }
    if (e == cudaSuccess) return CLEARMOE_OK;
    (void)cudaGetLastError();
    return CLEARMOE_ECUDA;
}

}  // namespace

}  // namespace cm

extern "C" {

int clearmoe_fp4_gemm(const clearmoe_fp4* A, const clearmoe_fp4* W, const clearmoe_fp8_epilogue* epi, void* out,
                      int32_t out_dtype, int64_t ldo, void* stream) {
    cm::Fp4GemmArgs<1> g;
    int rc = cm::check_gemm(A, W, 1, epi, g);
    if (rc || (rc = cm::set_out(g, out, out_dtype, ldo, W->rows))) return rc;
    return cm::run(g, A, W, 1, stream);
}

int clearmoe_fp4_gemm_fp4(const clearmoe_fp4* A, const clearmoe_fp4* W, const clearmoe_fp8_epilogue* epi,
                          const clearmoe_fp4* out, void* stream) {
    cm::Fp4GemmArgs<1> g;
    int rc = cm::check_gemm(A, W, 1, epi, g);
    if (rc || (rc = cm::check_fp4(out))) return rc;
    if (out->rows != A->rows || out->cols != W->rows) return CLEARMOE_EINVAL;
    g.out = out->q;
    g.out_kind = cm::FP4_OUT_FP4;
    g.ldo = cm::fp4_ldq(out->cols);
    g.out_scale = out->scale;
    g.ldos = cm::fp4_tiles(out->cols);
    return cm::run(g, A, W, 1, stream);
}

int clearmoe_fp4_grouped_gemm(const clearmoe_fp4* A, const clearmoe_fp4* W, int32_t E, const int32_t* offsets,
                              const int32_t* perm, const clearmoe_fp8_epilogue* epi, void* out, int32_t out_dtype,
                              int64_t ldo, void* stream) {
    if (E < 1 || E > CM_MAX_E || !W || !offsets || (reinterpret_cast<uintptr_t>(offsets) & 3) ||
        (reinterpret_cast<uintptr_t>(perm) & 3))
        return CLEARMOE_EINVAL;
    cm::Fp4GemmArgs<CM_MAX_E> g;
    int rc = cm::check_gemm(A, W, E, epi, g);
    if (rc || (rc = cm::set_out(g, out, out_dtype, ldo, W->rows))) return rc;
    g.offsets = offsets;
    g.rows = perm;
    return cm::run(g, A, W, E, stream);
}

int clearmoe_debug_fp4_kernel(int32_t width, int32_t pair) {
    if (width == 0 && pair == 0) {
        cm::g_forced = 0;
        return CLEARMOE_OK;
    }
    const bool known = pair == 1 ? width == 256 || width == 128 : pair == 0 && (width == 128 || width == 64 || width == cm::FEW_WIDTH);
    if (!known) return CLEARMOE_EINVAL;
    cm::g_forced = width << 1 | pair;
    return CLEARMOE_OK;
}

int clearmoe_debug_fp4_wait(int64_t wait_limit_ns) {
    if (wait_limit_ns < 0 || wait_limit_ns > cm::WAIT_LIMIT_NS) return CLEARMOE_EINVAL;
    cm::g_wait = wait_limit_ns ? wait_limit_ns : cm::WAIT_LIMIT_NS;
    return CLEARMOE_OK;
}

}  // extern "C"
