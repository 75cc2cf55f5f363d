// Products of matrices in 8-bit blocks on the 5th-generation tensor cores (tcgen05, sm_103a):
//
//   C[m, n] = epilogue( sum_b 2^(sa[m, b] + sw[n / 128, b] - 254) sum_{k in block b} qa[m, k] qw[n, k] )
//
// kind::mxf8f6f4 with block scales takes one power-of-two scale per row and 32 values of K from tensor memory,
// one byte each, and multiplies in the scale before the fp32 accumulation. A block of 128 is four such
// 32-blocks with the same byte: the MMA of each K = 32 step names the same byte again. A 32-bit column of scale
// memory holds four bytes of a row, so four consecutive blocks (512 of K) make one column for 32 rows, and the
// rows of scales in global memory are padded to whole words, which are moved as they lie.
//
// One persistent, warp-specialised kernel per N tile width:
//   epilogue     8 warps, 16 for tiles of 128 columns or more: warp w reads TMEM lane quarter w % 4 (its 32 rows) and
//                32 columns at a time;
//   2 warps      scales: load the words of the tile's rows and of W's blocks and lay them out in shared memory;
//   1 warp       TMEM allocation, tcgen05.cp of the scales, tcgen05.mma and commits (the whole warp in step, one
//                elected lane issues);
//   1 warp       TMA producer of the q tiles: 128 rows of A and BN of W, 128 bytes each, 128-byte swizzle.
// Rings: q stages in shared memory (full: TMA bytes, empty: commit), scale slots (full: the scale
// warp's arrival, empty: commit), two accumulators. Grouped products walk (group, row tile, column
// tile) from the device-resident offsets; a row tile never crosses its group's end.
// Every wait is bounded; a CTA that gives up records CLEARMOE_ETIMEOUT, lets its copies and MMAs in flight
// finish, frees its tensor memory and returns.
#include <cstdint>
#include <cstring>

#include "common.cuh"
#include "fp8.cuh"
#include "fp8_gemm.cuh"
#include "internal.h"

namespace cm {

namespace {

constexpr int F8_BM = 128;
constexpr int F8_BK = 128;

template <int BN_>
struct F8Cfg {
    static constexpr int BN = BN_;
    static constexpr int NUM_EPI = BN >= 128 ? 16 : 8, SPAN = NUM_EPI / 4;  // warps per lane quarter
    static constexpr int WARP_SCALE = NUM_EPI, WARP_MMA = NUM_EPI + 2, WARP_TMA = NUM_EPI + 3;
    static constexpr int THREADS = 32 * (NUM_EPI + 4);
    static constexpr int A_BYTES = F8_BM * F8_BK, B_BYTES = BN * F8_BK;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STAGES = (200 * 1024 / STAGE_BYTES) < 8 ? (200 * 1024 / STAGE_BYTES) : 8;
    static constexpr int NBARS = 2 * STAGES + 2 * F8_SLOTS + 4 + 1 + 4;
    static constexpr int SF_COL = 2 * BN;                  // first scale column
    static constexpr int SF_COLS = f8_slot_cols(BN), SF_BYTES = f8_slot_bytes(BN);
    static constexpr int TMEM_USED = 2 * BN + 2 * SF_COLS;
    static constexpr int TMEM_COLS = TMEM_USED <= 128 ? 128 : TMEM_USED <= 256 ? 256 : 512;
    static_assert(TMEM_USED <= 512);
    // scales, bias of a chunk per epilogue warp, largest magnitudes of a row's halves, group prefixes
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + F8_SLOTS * SF_BYTES + NUM_EPI * 32 * 4 + 2 * NUM_EPI * 32 * 4 + NBARS * 8 + 16 +
                                8 * (CM_MAX_E + 1);
};

__device__ __forceinline__ void umma_mxf8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
                                          uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
// KIND: Fp8Out.
template <int BN_, int KIND>
__global__ void __launch_bounds__(F8Cfg<BN_>::THREADS, 1) fp8_gemm_kernel(const __grid_constant__ Fp8GemmArgs a) {
    using C = F8Cfg<BN_>;
    constexpr int BN = C::BN;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char* s_sf = sm + C::STAGES * C::STAGE_BYTES;                       // [slot]
    float* s_bias = reinterpret_cast<float*>(s_sf + F8_SLOTS * C::SF_BYTES);     // [epilogue warp][32]
    float* s_amax = s_bias + C::NUM_EPI * 32;                                    // [2][epilogue warp][32]
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_amax + 2 * C::NUM_EPI * 32);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NBARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    int* s_prefix = reinterpret_cast<int*>(tmem_slot + 4);  // [E + 1]
    int* s_off = s_prefix + CM_MAX_E + 1;                    // [E + 1]

    const int warp = warp_uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto sfull_bar = [&](int s) { return bar0 + 8u * (2 * C::STAGES + s); };
    auto sempty_bar = [&](int s) { return bar0 + 8u * (2 * C::STAGES + F8_SLOTS + s); };
    auto tfull_bar = [&](int i) { return bar0 + 8u * (2 * C::STAGES + 2 * F8_SLOTS + i); };
    auto tempty_bar = [&](int i) { return bar0 + 8u * (2 * C::STAGES + 2 * F8_SLOTS + 2 + i); };
    const uint32_t drain_bar = bar0 + 8u * (2 * C::STAGES + 2 * F8_SLOTS + 4);
    auto pair_bar = [&](int q) { return bar0 + 8u * (2 * C::STAGES + 2 * F8_SLOTS + 5 + q); };
    const uint64_t lim = (uint64_t)a.wait_limit_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int s = 0; s < F8_SLOTS; ++s) {
            mbar_init(sfull_bar(s), 1);
            mbar_init(sempty_bar(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull_bar(i), 1);
            mbar_init(tempty_bar(i), C::NUM_EPI);
        }
        mbar_init(drain_bar, 1);
        for (int q = 0; q < 4; ++q) mbar_init(pair_bar(q), C::SPAN);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == C::WARP_MMA) tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();  // everything below may read the previous kernel's results
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    if (threadIdx.x == 0) {
        f8_groups(a, F8_BM, s_off, s_prefix);
    }
    __syncthreads();
    const uint32_t tmem = warp_uniform(*tmem_slot);
    F8Walk t(blockIdx.x, gridDim.x, a.N, F8_BM, BN, a.E, s_off, s_prefix);
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
                const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES);
                mbar_arrive_expect_tx_warp(full_bar(stage), a.box_rows * F8_BK + C::B_BYTES);
                // coordinates in the maps' 16-bit elements: two bytes each
                tma_load_2d(sA, &a.tmA, kb * (F8_BK / 2), m0, full_bar(stage));
                tma_load_2d(sA + C::A_BYTES, &a.tmB[e], kb * (F8_BK / 2), n0, full_bar(stage));
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
        int stage = 0, slot = 0, acc = 0;
        uint32_t ph = 0, sph = 0, aph = 0;
        bool ok = true;
        for (; warp_uniform((int)t.live()) && ok; t.next()) {
            if (!mbar_wait_warp(tempty_bar(acc), aph ^ 1, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + acc * BN;
            for (int kb = 0; kb < nkb; ++kb) {
                const int byte = kb & 3;
                const uint32_t sf = tmem + C::SF_COL + (slot & 1) * C::SF_COLS;
                if (byte == 0) {
                    if (!mbar_wait_warp(sfull_bar(slot), sph, abort_flag, a.status, lim)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll
                    for (int h = 0; h < C::SF_COLS / 4; ++h)
                        tmem_cp_scales<1>(sf + 4 * h, smem_u32(s_sf) + slot * C::SF_BYTES + 512 * h);
                }
                if (!mbar_wait_warp(full_bar(stage), ph, abort_flag, a.status, lim)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES);
                const uint64_t ad = sdesc_kmajor_sw128(sA), bd = sdesc_kmajor_sw128(sA + C::A_BYTES);
                const uint32_t id = idesc_mxf8(F8_BM, BN, byte);
#pragma unroll
                for (int k = 0; k < 4; ++k)  // 32 of K: 32 bytes on in each row
                    umma_mxf8(d, ad + 2 * k, bd + 2 * k, id, sf, sf + 4, (kb | k) != 0);
                umma_commit(empty_bar(stage));
                if (++stage == C::STAGES) {
                    stage = 0;
                    ph ^= 1;
                }
                if (byte == 3 || kb + 1 == nkb) {
                    umma_commit(sempty_bar(slot));
                    if (++slot == F8_SLOTS) {
                        slot = 0;
                        sph ^= 1;
                    }
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
    } else if (warp >= C::WARP_SCALE) {
        // ------------------------------------------------ scales
        f8_scale_warp<BN>(a, warp - C::WARP_SCALE, t, 0, lane,
                          [&](const F8Scales<BN>& w, int slot, uint32_t ph) {
                              if (!mbar_wait_warp(sempty_bar(slot), ph ^ 1, abort_flag, a.status, lim)) return false;
                              w.store(s_sf + slot * C::SF_BYTES, lane);
                              fence_proxy_async_smem();
                              __syncwarp();
                              if (lane == 0) mbar_arrive(sfull_bar(slot));
                              return true;
                          });
    } else {
        // ------------------------------------------------ epilogue
        // warp w takes 32-column chunks w / 4, w / 4 + SPAN, .. of the tile (a 32-wide tile's only chunk: warps 0-3)
        constexpr int SPAN = C::SPAN, ROUNDS = (BN / 32 + SPAN - 1) / SPAN;
        const int quarter = warp & 3, cg = warp >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float* bias_line = s_bias + warp * 32;
        const bool has_bias = a.bias != nullptr;
        const bool wide = f8_wide(a);
        int acc = 0;
        uint32_t aph = 0, pph = 0;
        for (; t.live(); t.next()) {
            const int orow = f8_out_row(a, t.m0 + quarter * 32 + lane, t.hi);
            float b[ROUNDS];
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const int n = t.n0 + (SPAN * r + cg) * 32 + lane;
                b[r] = 0.f;
                if (has_bias && n < a.N)
                    b[r] = a.bias_bf16 ? bf16_to_f32(__ldg(static_cast<const uint16_t*>(a.bias) + n))
                                       : __ldg(static_cast<const float*>(a.bias) + n);
            }
            if (!mbar_wait_warp(tfull_bar(acc), aph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + lanes + acc * BN;
            float v[ROUNDS][32];
            float mx = 0.f;
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r) {
                const bool mine = (SPAN * r + cg) * 32 < BN;
                const int nc = t.n0 + (SPAN * r + cg) * 32;
                __syncwarp();  // the bias line is read, rows without a store have caught up
                if (mine) {
                    uint32_t u[32];
                    CM_TMEM_LD_X32(d + (SPAN * r + cg) * 32, u);
                    if (has_bias) bias_line[lane] = b[r];
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[r][i] = __uint_as_float(u[i]);
                }
                if (r + 1 == ROUNDS) {  // the accumulator is read: the next tile's MMAs may start
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty_bar(acc));
                }
                __syncwarp();
                if (!mine) continue;
                f8_act<32, KIND == FP8_OUT_F32>(v[r], bias_line, has_bias, a.act);
                if constexpr (KIND == FP8_OUT_FP8) {
                    if (nc + 32 > a.N) {  // the last block's padding is zero
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (nc + i >= a.N) v[r][i] = 0.f;
                    }
                    mx = max_abs(mx, f8_max_abs32(v[r]));
                } else {
                    f8_store32<KIND>(a, v[r], orow, nc, wide, lane);
                }
            }
            if constexpr (KIND == FP8_OUT_FP8) {
                // The tile's 128 columns are one block: each of the quarter's four warps holds 32 of a row, and they exchange
                // the row's largest magnitudes. Double-buffered by tile: a warp's reads of one tile's values precede its
                // arrival for the next tile, and that the other warps' writes two tiles on.
                static_assert(BN == 128 && ROUNDS == 1);
                float* ex = s_amax + acc * C::NUM_EPI * 32;
                ex[warp * 32 + lane] = mx;
                __syncwarp();
                if (lane == 0) mbar_arrive(pair_bar(quarter));
                if (!mbar_wait_warp(pair_bar(quarter), pph, abort_flag, a.status, lim)) break;
                pph ^= 1;
                const float* e = ex + quarter * 32 + lane;
                const uint32_t s = fp8_scale_byte(abs_bits(max_abs3(max_abs(e[0], e[4 * 32]), e[8 * 32], e[12 * 32])));
                if (orow >= 0) {
                    uint32_t o[8];
                    fp8_pack32(o, v[0], fp8_inverse_scale(s));
                    st_global_32(static_cast<uint8_t*>(a.out) + (int64_t)orow * a.ldo + t.n0 + cg * 32, o);
                    if (cg == 0) a.out_scale[(int64_t)orow * a.ldos + t.n0 / 128] = (uint8_t)s;
                }
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

template <int BN, int KIND>
cudaError_t launch_bn(const Fp8GemmArgs& a, int num_sms, cudaStream_t s) {
    using C = F8Cfg<BN>;
    const cudaError_t e = smem_attr_once((const void*)fp8_gemm_kernel<BN, KIND>, C::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t m_tiles = (a.M + F8_BM - 1) / F8_BM + (a.offsets ? a.E - 1 : 0);
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
    return cudaLaunchKernelEx(&cfg, fp8_gemm_kernel<BN, KIND>, a);
}

template <int BN>
cudaError_t launch_kind(const Fp8GemmArgs& a, int num_sms, cudaStream_t s) {
    return a.out_kind == FP8_OUT_F32 ? launch_bn<BN, FP8_OUT_F32>(a, num_sms, s) : launch_bn<BN, FP8_OUT_BF16>(a, num_sms, s);
}

}  // namespace

// Cycles (at 1.9 GHz) a product takes on a kernel: its start, then rounds of tiles, each of which multiplies and loads its
// k-blocks or, where that is longer, runs the epilogue of the tile before it, then the last epilogue. A k-block's cycles
// grow from what the MMAs take (2 a column, 285 at the least) to what the path from L2 allows with every SM at work.
// Fitted to measurements (us, the best two of seven kernels and this rule's choice, at M x N x K): 197 x 3,072 x 768
// 3.9 (64 wide, one SM) and 4.5 (128), 3.9; 1,000 x 384 x 1,536 4.8 (32) and 4.8 (64), 4.7; 4,000 x 1,024 x 1,024 7.2
// (128) and 8.3 (128, pair), 7.1; 9,973 x 384 x 1,536 9.2 (128) and 9.9 (128, pair), 9.1; 25,216 x 768 x 3,072 38.1
// (256, pair) and 44.5 (192, pair), 38.2; 16,384 x 4,096 x 4,096 144 (256, pair) and 158 (192, pair), 143, all in runs
// of a few milliseconds (at the power limit, after some more of them, 155 to 166). The quantising epilogue's cost is that
// with bias and GELU; without them 50,432 x 3,072 x 768 takes 100 us in the 128-wide tiles that it chooses, 79 in 256.
struct Fp8Kernel {
    Fp8Pick pick;
    int block;     // cycles of a k-block with every SM at work
    int epilogue[4];  // of a tile beside the next tile's MMAs, by Fp8Store
    int quantize;     // 8-bit outputs (0: none)
};
// How outputs are stored: bf16 or fp32 rows in whole 32-byte pieces, or of any pitch. Cycles measured at 2,922 x 3,456 (3,453)
// x 60, where the stores are all there is; us of the best kernel and of the one that a single figure had chosen: bf16 7.4 / 10.5,
// fp32 11.4 / 14.7, any pitch 13.8 / 18.5 and 14.6 / 18.3.
enum Fp8Store { FP8_STORE_BF16 = 0, FP8_STORE_F32 = 1, FP8_STORE_ODD = 2 };  // ODD: added to the type's
static double fp8_cost(const Fp8Kernel& k, int64_t M, int N, int nkb, int out_kind, bool wide, int groups, int num_sms) {
    const bool pair = k.pick.pair, q = out_kind == FP8_OUT_FP8;
    const int bn = k.pick.bn, rows = pair ? 256 : 128, units = pair ? num_sms / 2 : num_sms;
    if (units < 1 || (q && !k.quantize)) return 1e30;
    const int64_t tiles = ((M + rows - 1) / rows + groups - 1) * (((int64_t)N + bn - 1) / bn);
    const double rounds = (double)((tiles + units - 1) / units), busy = tiles < units ? (double)tiles / units : 1.0;
    const double low = 2 * bn > 285 ? 2 * bn : 285, main = nkb * (low + (k.block - low) * busy * busy);
    const int store = (out_kind == FP8_OUT_BF16 ? FP8_STORE_BF16 : FP8_STORE_F32) + (wide ? 0 : FP8_STORE_ODD);
    const double beside = q ? k.quantize : k.epilogue[store];
    const double between = bn == 256 ? 1500 : 0;  // 256: accumulators that overlap
    const double next = main + between > beside ? main + between : beside;
    return (pair ? 8800 : 4600) + main + (rounds - 1) * next + (q ? beside : 15.0 * bn);
}

Fp8Pick fp8_pick(int64_t M, int N, int nkb, int out_kind, bool wide, int groups, int num_sms) {
    static const Fp8Kernel all[] = {
        {{256, 1}, 540, {3160, 7200, 8450, 9150}, 5950}, {{192, 1}, 550, {2000, 5050, 7200, 8250}, 0},
        {{128, 1}, 487, {1450, 3300, 4250, 4720}, 3000}, {{192, 0}, 588, {3040, 6960, 9060, 9800}, 0},
        {{128, 0}, 445, {2180, 3960, 4800, 5260}, 4200}, {{64, 0}, 350, {1370, 2320, 2690, 2790}, 0},
        {{32, 0}, 285, {920, 1400, 1840, 1840}, 0}};
    Fp8Pick best = all[4].pick;
    double least = 1e30;
    for (const Fp8Kernel& k : all) {
        const double c = fp8_cost(k, M, N, nkb, out_kind, wide, groups, num_sms);
        if (c < least) {
            least = c;
            best = k.pick;
        }
    }
    return best;
}

cudaError_t launch_fp8_gemm(const Fp8GemmArgs& a, const Fp8Pick& k, int num_sms, cudaStream_t s) {
    if (k.pair) return launch_fp8_gemm2(a, k.bn, num_sms, s);
    if (a.out_kind == FP8_OUT_FP8) return launch_bn<128, FP8_OUT_FP8>(a, num_sms, s);
    switch (k.bn) {
        case 192: return launch_kind<192>(a, num_sms, s);
        case 128: return launch_kind<128>(a, num_sms, s);
        case 64: return launch_kind<64>(a, num_sms, s);
        default: return launch_kind<32>(a, num_sms, s);
    }
}

// The kernel that tests have fixed for their thread's calls (width << 1 | pair), or 0; FP8_FORCE_FEW: the one for few rows.
constexpr int FP8_FORCE_FEW = 16 << 1;
static thread_local int g_forced = 0;

int run_fp8_gemm(Fp8GemmArgs& g, const clearmoe_fp8* A, const clearmoe_fp8* W, int E, int num_sms, cudaStream_t s) {
    g.M = A->rows;
    g.N = (int)W[0].rows;
    g.nkb = (int)((A->cols + 127) / 128);
    g.E = E;
    g.lds = fp8_lds(A->cols);
    g.sa = A->scale;
    const int forced = g_forced;
    // Few rows, while the SMs take all CTAs of 16 columns at once: us against the best tcgen05 tile, 1 x 4,096 x 4,096 4.6 / 7.4,
    // 12 x 4,096 x 4,096 6.3 / 7.5, 12 x 768 x 3,072 3.6 / 5.9; more CTAs than that: 12 x 8,192 x 1,024 5.2 / 4.1, 8 x 8,192 x
    // 8,192 18.2 / 14.8.
    const bool few_fits = !g.offsets && g.out_kind != FP8_OUT_FP8 && g.M <= FP8_FEW_MAX && (g.M + 1) * g.nkb <= FP8_FEW_SCALES;
    if (few_fits && (forced == FP8_FORCE_FEW || (forced == 0 && (g.N + 15) / 16 <= 2 * num_sms))) {
        g.x = A->q;
        g.w = W->q;
        g.sb[0] = W->scale;
        if (launch_fp8_few(g, s) == cudaSuccess) return CLEARMOE_OK;
        (void)cudaGetLastError();
        return CLEARMOE_ECUDA;
    }
    Fp8Pick k = fp8_pick(g.M, g.N, g.nkb, g.out_kind, f8_wide(g), E, num_sms);
    if (forced && forced != FP8_FORCE_FEW) {
        const Fp8Pick f = {forced >> 1, forced & 1};
        if (g.out_kind != FP8_OUT_FP8 || f.bn % 128 == 0) k = f;
    }
    // rows of bytes as rows of half as many 16-bit elements: boxes of 64 of them are 128 bytes
    const int64_t cols16 = fp8_ldq(A->cols) / 2;
    // One SM, fewer rows than a tile: a box of those alone. The copy engine takes longer over a row past the end, which it
    // fills with zeros, than over one that it reads (24 x 4,096 x 4,096, 64 wide: 10.9 us, 7.7 so); what the others' sums are
    // made of does not matter.
    g.box_rows = !k.pair && g.M < F8_BM ? (int)(g.M + 7) / 8 * 8 : F8_BM;
    if (encode_tmap_bf16(&g.tmA, A->q, A->rows, cols16, g.box_rows)) return CLEARMOE_ECUDA;
    if (g.out_kind == FP8_OUT_FP8 && k.pair && encode_tmap_bytes(&g.tmOut, g.out, g.M, g.ldo, 32)) return CLEARMOE_ECUDA;
    for (int e = 0; e < E; ++e) {
        g.sb[e] = W[e].scale;
        if (encode_tmap_bf16(&g.tmB[e], W[e].q, W[e].rows, cols16, k.pair ? k.bn / 2 : k.bn)) return CLEARMOE_ECUDA;
    }
    if (launch_fp8_gemm(g, k, num_sms, s) == cudaSuccess) return CLEARMOE_OK;
    (void)cudaGetLastError();
    return CLEARMOE_ECUDA;
}

}  // namespace cm

namespace {

// Operands, epilogue and output of a product; fills g's epilogue fields.
int check_gemm(const clearmoe_fp8* A, const clearmoe_fp8* W, int E, const clearmoe_fp8_epilogue* epi, cm::Fp8GemmArgs& g) {
    std::memset(&g, 0, sizeof(g));
    int rc = cm::check_fp8(A);
    if (rc) return rc;
    for (int e = 0; e < E; ++e) {
        if ((rc = cm::check_fp8(W + e))) return rc;
        if (W[e].cols != A->cols || W[e].rows != W[0].rows || W[e].rows > (int64_t)1 << 24) return CLEARMOE_EINVAL;
    }
    g.act = CLEARMOE_ACT_NONE;
    g.wait_limit_ns = 1000000000LL;
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

int set_out(cm::Fp8GemmArgs& g, void* out, int32_t dtype, int64_t ldo, int64_t N) {
    if (!out || (dtype != CLEARMOE_F32 && dtype != CLEARMOE_BF16) || ldo < N || ldo > (int64_t)1 << 30) return CLEARMOE_EINVAL;
    if (reinterpret_cast<uintptr_t>(out) & (dtype == CLEARMOE_BF16 ? 1 : 3)) return CLEARMOE_EINVAL;
    g.out = out;
    g.out_kind = dtype == CLEARMOE_BF16 ? cm::FP8_OUT_BF16 : cm::FP8_OUT_F32;
    g.ldo = ldo;
    return CLEARMOE_OK;
}

int run(cm::Fp8GemmArgs& g, const clearmoe_fp8* A, const clearmoe_fp8* W, int E, void* stream) {
    const int sms = cm::current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    return cm::run_fp8_gemm(g, A, W, E, sms, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

int clearmoe_fp8_gemm(const clearmoe_fp8* A, const clearmoe_fp8* W, const clearmoe_fp8_epilogue* epi, void* out,
                      int32_t out_dtype, int64_t ldo, void* stream) {
    cm::Fp8GemmArgs g;
    int rc = check_gemm(A, W, 1, epi, g);
    if (rc || (rc = set_out(g, out, out_dtype, ldo, W->rows))) return rc;
    return run(g, A, W, 1, stream);
}

int clearmoe_fp8_gemm_fp8(const clearmoe_fp8* A, const clearmoe_fp8* W, const clearmoe_fp8_epilogue* epi,
                          const clearmoe_fp8* out, void* stream) {
    cm::Fp8GemmArgs g;
    int rc = check_gemm(A, W, 1, epi, g);
    if (rc || (rc = cm::check_fp8(out))) return rc;
    if (out->rows != A->rows || out->cols != W->rows) return CLEARMOE_EINVAL;
    g.out = out->q;
    g.out_kind = cm::FP8_OUT_FP8;
    g.ldo = cm::fp8_ldq(out->cols);
    g.out_scale = out->scale;
    g.ldos = cm::fp8_lds(out->cols);
    return run(g, A, W, 1, stream);
}

int clearmoe_fp8_grouped_gemm(const clearmoe_fp8* A, const clearmoe_fp8* W, int32_t E, const int32_t* offsets,
                              const int32_t* perm, const clearmoe_fp8_epilogue* epi, void* out, int32_t out_dtype,
                              int64_t ldo, void* stream) {
    if (E < 1 || E > CM_MAX_E || !W || !offsets || (reinterpret_cast<uintptr_t>(offsets) & 3) ||
        (reinterpret_cast<uintptr_t>(perm) & 3))
        return CLEARMOE_EINVAL;
    cm::Fp8GemmArgs g;
    int rc = check_gemm(A, W, E, epi, g);
    if (rc || (rc = set_out(g, out, out_dtype, ldo, W->rows))) return rc;
    g.offsets = offsets;
    g.rows = perm;
    return run(g, A, W, E, stream);
}

int clearmoe_debug_fp8_kernel(int32_t width, int32_t pair) {
    if (width == 0 && pair == 0) {
        cm::g_forced = 0;
        return CLEARMOE_OK;
    }
    const bool known = pair == 1 ? width == 256 || width == 192 || width == 128
                                 : pair == 0 && (width == 192 || width == 128 || width == 64 || width == 32 || width == 16);
    if (!known) return CLEARMOE_EINVAL;
    cm::g_forced = width << 1 | pair;
    return CLEARMOE_OK;
}

}  // extern "C"
