// Products of matrices in 4-bit blocks on pairs of SMs (tcgen05 cta_group::2, sm_103a): fp4_gemm.cu's arithmetic in
// 256 x BN tiles. CTA r of a pair loads A rows [128 r, +128) and W rows [BN / 2 r, +BN / 2) of the tile, and the scales of
// its own rows of A and of all BN columns; the even CTA's MMAs (M = 256, N = BN, K = 64) read both halves and leave 128
// rows of the accumulator in each CTA's tensor memory.
//
// Tensor memory: two accumulators of 256 columns and the scales do not fit its 512 columns. So the second accumulator
// starts at column 224, 32 columns inside the first: the epilogue reads the shared columns of a tile first and says so
// (ovl_bar), and the next tile's MMAs start then rather than when the whole accumulator is read. Columns 480 .. 503 hold
// the scales of two times 128 of K, in turn.
//
// A last round with tiles for half of the pairs at the most has them in halves of 128 columns, one a pair (9,973 x 1,024 x
// 4,096 in eight groups 21.3 -> 19.9 us, 2,560 x 2,048 x 4,096 15.1 -> 12.4, 10,240 x 1,024 x 4,096 20.4 -> 18.1).
//
// Epilogue: 16 warps (four per lane quarter), each 32 columns at a time (one block of a 4-bit output), two times side by
// side. What bounds it is the path of loads and stores (TMEM, shared and global memory): a store whose lanes write 32 rows
// apart takes it 32 cycles whatever its width, so bf16 rows leave by bulk copies from shared memory and 4-bit rows 32
// bytes at a time.
// Hand-offs and giving up as in fp8_gemm2.cu: TMA bytes of both CTAs on the even CTA's full barriers, commits on both
// CTAs' empty and tfull barriers, the epilogue warps of both on the even CTA's ovl and tempty; every wait is bounded, and
// the even CTA lets copies in flight land before the cluster retires.
#include <cstdint>

#include "common.cuh"
#include "drain.h"
#include "fp4.cuh"
#include "fp4_gemm.cuh"
#include "internal.h"
#include "pair.cuh"

namespace cm {

namespace {

constexpr int P4_BM = 128;  // rows per CTA
constexpr int P4_STAGED = 32 * 64;  // bytes of a warp's 32 rows and columns of bf16

template <int BN_, int KIND>
struct P4Cfg {
    static constexpr int BN = BN_;
    static constexpr int BH = BN / 2;  // W rows per CTA
    static constexpr int NUM_EPI = 16;  // epilogue warps
    static constexpr int WARP_MMA = NUM_EPI, WARP_TMA = NUM_EPI + 1;
    static constexpr int THREADS = 32 * (WARP_TMA + 1);
    static constexpr int A_BYTES = P4_BM * 128, B_BYTES = BH * 128;
    static constexpr int NF = BN / 128;  // scale tiles of a tile's columns
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + (1 + NF) * F4_SF;
    static constexpr int OUT_BYTES = KIND == FP4_OUT_BF16_BULK ? NUM_EPI * P4_STAGED : 0;
    static constexpr int ROOM = 220 * 1024 - OUT_BYTES, STAGES = ROOM / STAGE_BYTES < 8 ? ROOM / STAGE_BYTES : 8;
    static constexpr bool OVL = BN == 256;
    static constexpr bool HALVES = BN == 256;  // of tiles of the last round
    static constexpr int HALF_BYTES = STAGE_BYTES - (HALVES ? B_BYTES / 2 : 0);  // of a stage of theirs
    static constexpr int ACC1 = OVL ? 224 : BN;  // first column of the second accumulator
    static constexpr int SF_COL = ACC1 + BN, SF_COLS = 4 * (1 + NF);
    static_assert(SF_COL + 2 * SF_COLS <= 512);
    // Epilogue warps in GROUPS that take every GROUPS-th tile (two: one accumulator each); a warp has PASSES times CH chunks
    // of 32 columns side by side.
    static constexpr int GROUPS = KIND == FP4_OUT_FP4 ? 2 : 1, TILE_WARPS = NUM_EPI / GROUPS;
    static constexpr int PASSES = GROUPS == 2 ? BN / 128 : 1, CH = GROUPS == 2 ? 2 : BN / 128, WIDTH = 32 * PASSES * CH;
    static constexpr int NBARS = 2 * STAGES + 4 + 3;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + NUM_EPI * CH * 32 * 4 + NBARS * 8 + 16 + 8 * (CM_MAX_E + 1) + 8;
    static_assert(STAGE_BYTES % 1024 == 0);
};

__device__ __forceinline__ void umma2_mxf4(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
                                           uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// 32 rows' 32 columns (a row a lane) to a warp's shared memory as bf16, where the copy engine takes them from: piece j of
// 16 bytes of row i lies at j ^ (i >> 1 & 3). The engine has read what was there before.
__device__ __forceinline__ void stage_bf16(const float (&v)[32], uint32_t staged, int lane) {
    bulk_wait_read();
    __syncwarp();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const float* w = v + 8 * p;
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(staged + lane * 64 + ((p ^ (lane >> 1 & 3)) << 4)),
                     "r"(pack_bf16(w[0], w[1])), "r"(pack_bf16(w[2], w[3])), "r"(pack_bf16(w[4], w[5])), "r"(pack_bf16(w[6], w[7]))
                     : "memory");
    }
    fence_proxy_async_smem();
    __syncwarp();
}

// KIND: FP8_OUT_F32, FP8_OUT_BF16, FP4_OUT_FP4 or FP4_OUT_BF16_BULK.
template <int BN_, int KIND, int NE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P4Cfg<BN_, KIND>::THREADS, 1)
    fp4_gemm2_kernel(const __grid_constant__ Fp4GemmArgs<NE> a) {
    using C = P4Cfg<BN_, KIND>;
    constexpr int BN = C::BN, STAGES = C::STAGES;
    constexpr bool GROUPED = Fp4GemmArgs<NE>::GROUPED;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char* s_out = sm + STAGES * C::STAGE_BYTES;               // [epilogue warp][32 rows][64], bf16 outputs
    float* s_bias = reinterpret_cast<float*>(s_out + C::OUT_BYTES);    // [epilogue warp][CH][32]
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_bias + C::NUM_EPI * C::CH * 32);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NBARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile uint32_t* s_issued = tmem_slot + 2;  // k-blocks this CTA's producer has loaded, once it has stopped
    int* s_prefix = reinterpret_cast<int*>(tmem_slot + 4);  // [E + 1]
    int* s_off = s_prefix + CM_MAX_E + 1;                   // [E + 1]

    const int warp = warp_uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const bool leader = rank == 0;
    const uint32_t bar0 = smem_u32(bars);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (STAGES + s); };
    auto tfull_bar = [&](int i) { return bar0 + 8u * (2 * STAGES + i); };
    auto tempty_bar = [&](int i) { return bar0 + 8u * (2 * STAGES + 2 + i); };
    const uint32_t ovl_bar = bar0 + 8u * (2 * STAGES + 4);
    const uint32_t drain_bar = ovl_bar + 8, stop_bar = ovl_bar + 16;
    const uint64_t lim = (uint64_t)a.wait_limit_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);   // the even CTA's producer arrives; both CTAs' bytes land here
            mbar_init(empty_bar(s), 1);  // one multicast commit per stage
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull_bar(i), 1);
            mbar_init(tempty_bar(i), 2 * C::TILE_WARPS);  // epilogue warps of both CTAs
        }
        mbar_init(ovl_bar, 8);  // the warps whose chunk lies in the shared columns, of both CTAs
        mbar_init(drain_bar, 1);
        mbar_init(stop_bar, 2);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == C::WARP_TMA && lane == 0) f4_prefetch_maps(a);
    if (warp == C::WARP_MMA) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // barriers initialised and tensor memory allocated in both CTAs
    tc_fence_after();
    auto begin = [&]() {
        pdl_wait();  // everything below may read the previous kernel's results
        pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    };
    if constexpr (GROUPED) {
        begin();
        if (warp == 0) f4_groups(a, 2 * P4_BM, s_off, s_prefix, lane);
        __syncthreads();
    }
    const uint32_t tmem = warp_uniform(*tmem_slot);  // all 512 columns: the same base in both CTAs
    const int nkb = a.nkb;
    const int unit = (int)blockIdx.x >> 1;
    F4PairWalk<GROUPED, C::HALVES> t(unit, gridDim.x >> 1, a, 2 * P4_BM, BN, s_off, s_prefix);
    if constexpr (!GROUPED) begin();

    if (warp >= C::NUM_EPI) {
        if (warp == C::WARP_TMA) {
            // ------------------------------------------------ producers (both CTAs)
            const uint32_t full_leader0 = map_to_rank(full_bar(0), 0);
            int stage = 0;
            uint32_t ph = 0, issued = 0;
            bool ok = true;
            for (; warp_uniform((int)t.live()) && ok; t.next(unit)) {
                const int e = warp_uniform(t.e);
                const int m0 = warp_uniform(t.m0 + (int)rank * P4_BM), n0 = warp_uniform(t.n0);
                const bool half = warp_uniform((int)t.half());
                const int w0 = n0 + (int)rank * (half ? C::BH / 2 : C::BH);
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait_warp(empty_bar(stage), ph ^ 1, abort_flag, a.status, lim)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES), sB = sA + C::A_BYTES, sF = sB + C::B_BYTES;
                    const uint32_t fb = full_leader0 + 8u * stage;
                    if (leader) mbar_arrive_expect_tx_warp(full_bar(stage), 2 * (half ? C::HALF_BYTES : C::STAGE_BYTES));
                    // coordinates in the maps' elements: 16-bit ones of four columns, 32-bit ones of four scales
                    tma_load_2d_pair(sA, &a.tmA, kb * 64, m0, fb);
                    tma_load_2d_pair(sB, half ? &a.tmH[e] : &a.tmB[e], kb * 64, w0, fb);
                    tma_load_2d_pair(sF, &a.tmSA, kb * 256, m0 >> 7, fb);
                    tma_load_2d_pair(sF + F4_SF, &a.tmSB[e], kb * 256, n0 >> 7, fb);
                    ++issued;
                    if (++stage == STAGES) {
                        stage = 0;
                        ph ^= 1;
                    }
                }
            }
            *s_issued = issued;
            __syncwarp();
            mbar_arrive_release_cluster_warp(map_to_rank(stop_bar, 0));
        } else if (warp == C::WARP_MMA) {
            // ------------------------------------------------ MMA issuer (even CTA, the whole warp)
            if (leader) {
                int stage = 0, acc = 0;
                uint32_t ph = 0, aph = 0, oph = 1;  // oph: phase of the previous tile's shared columns
                bool ok = true;
                for (; warp_uniform((int)t.live()) && ok; t.next(unit)) {
                    if (!mbar_wait_warp(tempty_bar(acc), aph ^ 1, abort_flag, a.status, lim)) break;
                    if (C::OVL && !mbar_wait_warp(ovl_bar, oph, abort_flag, a.status, lim)) break;
                    oph ^= 1;
                    tc_fence_after();
                    const uint32_t d = tmem + acc * C::ACC1;
                    const int width = warp_uniform(t.half() ? BN / 2 : BN);
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
                            const uint32_t sf = tmem + C::SF_COL + h * C::SF_COLS;
                            tmem_cp_scales<2>(sf, sF + 512 * h);
#pragma unroll
                            for (int i = 0; i < C::NF; ++i) tmem_cp_scales<2>(sf + 4 + 4 * i, sF + F4_SF * (1 + i) + 512 * h);
#pragma unroll
                            for (int j = 0; j < 2; ++j) {  // 64 columns: 32 bytes on in each row
                                const int k = 2 * h + j;
                                if (4 * kb + k < a.ksteps)
                                    umma2_mxf4(d, ad + 2 * k, bd + 2 * k, idesc_mxf4(2 * P4_BM, width, j), sf, sf + 4, (kb | k) != 0);
                            }
                        }
                        umma2_commit_both(empty_bar(stage));
                        if (++stage == STAGES) {
                            stage = 0;
                            ph ^= 1;
                        }
                    }
                    if (!ok) break;
                    umma2_commit_both(tfull_bar(acc));
                    if (++acc == 2) {
                        acc = 0;
                        aph ^= 1;
                    }
                }
                umma2_commit_one(drain_bar);  // every MMA issued above has completed once this fires
                mbar_wait_warp(drain_bar, 0, nullptr, a.status, lim + 10000000ull);
                // An issuer that ran all its tiles has seen every copy of both CTAs land. One that gave up waits, once
                // both producers have stopped, for the last copies issued to each stage; a stage that only one producer
                // reached gets the other's part of its barrier here.
                if (warp_uniform((int)*abort_flag) && mbar_wait_warp(stop_bar, 0, nullptr, a.status, 2 * lim + 10000000ull)) {
                    fence_cluster();
                    int rest;
                    const uint32_t k_half = (uint32_t)(t.whole(a, (int)gridDim.x >> 1, rest) * nkb);
                    const uint32_t at = smem_u32(tmem_slot + 2);
                    const uint32_t n0 = ld_cluster_u32(map_to_rank(at, 0)), n1 = ld_cluster_u32(map_to_rank(at, 1)), n = max(n0, n1);
    #pragma unroll 1
                    for (uint32_t k = n > STAGES ? n - STAGES : 0; k < n; ++k) {
                        const uint32_t s = k % STAGES;
                        const DrainStep st = drain_step(k, n0, n1);
                        const uint32_t bytes = drain_bytes(k, t.halved, k_half, C::STAGE_BYTES, C::HALF_BYTES);
                        // the odd CTA alone reached it: expect its bytes; the even CTA alone: count the odd one's as landed
                        if (st.arrive) mbar_arrive_expect_tx_warp(full_bar(s), bytes);
                        if (st.complete) mbar_complete_tx_warp(full_bar(s), bytes);
                        mbar_wait_warp(full_bar(s), (k / STAGES) & 1, nullptr, a.status, 10000000ull);
                    }
                }
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------ epilogue (both CTAs, own 128 rows)
        const int quarter = warp & 3, cg = warp % C::TILE_WARPS >> 2, group = warp / C::TILE_WARPS;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float* bias_line = s_bias + warp * C::CH * 32;
        const bool has_bias = a.bias != nullptr;
        const bool wide = f8_wide(a);
        unsigned char* staged = s_out + warp * P4_STAGED;
        const uint32_t tempty_leader0 = map_to_rank(tempty_bar(0), 0), ovl_leader = map_to_rank(ovl_bar, 0);
        int acc = group;
        // The warp's first column in pass p: the pass with the columns that the accumulators share first.
        auto column = [&](int p) { return cg * C::WIDTH + (C::OVL && acc == 0 ? C::PASSES - 1 - p : p) * C::CH * 32; };
        // What a tile's epilogue needs beside its sums, loaded a tile ahead: a load waits behind the queued tile loads.
        float bias[C::PASSES][C::CH];
        int row = 0;
        auto prefetch = [&]() {
            if (!t.live()) return;
            row = f4_out_row(a, t.m0 + (int)rank * P4_BM + quarter * 32 + lane, t.lo, t.hi);
            if (has_bias) {
#pragma unroll
                for (int p = 0; p < C::PASSES; ++p)
#pragma unroll
                    for (int r = 0; r < C::CH; ++r) {
                        const int n = t.n0 + column(p) + 32 * r + lane;
                        bias[p][r] = n >= a.N      ? 0.f
                                     : a.bias_bf16 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(a.bias) + n))
                                                   : __ldcg(static_cast<const float*>(a.bias) + n);
                    }
            }
        };
        if (group && t.live()) t.next(unit);
        prefetch();
        uint32_t aph = 0;
        while (t.live()) {
            const int n0 = t.n0, orow = row, row0 = t.m0 + (int)rank * P4_BM + quarter * 32;
            int col[C::PASSES];
            float b[C::PASSES][C::CH];
#pragma unroll
            for (int p = 0; p < C::PASSES; ++p) {
                col[p] = column(p);
#pragma unroll
                for (int r = 0; r < C::CH; ++r) b[p][r] = bias[p][r];
            }
            // A half tile is the walker's last one: nobody waits for its accumulator to be read.
            if (t.half() && cg * C::WIDTH >= BN / 2) break;
            const int now = acc;
            if (C::GROUPS == 1) acc ^= 1;
            t.next(unit);
            if (C::GROUPS == 2 && t.live()) t.next(unit);
            prefetch();
            if (!mbar_wait_warp(tfull_bar(now), aph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + lanes + now * C::ACC1;
#pragma unroll
            for (int p = 0; p < C::PASSES; ++p) {
                // All of a pass's columns at once: the accumulator is free the sooner, and one chunk's arithmetic passes under
                // the other's.
                float v[C::CH][32];
                {
                    uint32_t u[C::CH][32];
#pragma unroll
                    for (int r = 0; r < C::CH; ++r) CM_TMEM_LD_X32(d + col[p] + 32 * r, u[r]);
                    __syncwarp();
                    if (has_bias) {
#pragma unroll
                        for (int r = 0; r < C::CH; ++r) bias_line[32 * r + lane] = b[p][r];
                    }
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < C::CH; ++r)
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[r][i] = __uint_as_float(u[r][i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {  // the columns may be written again
                    if (C::OVL && p == 0 && cg == (now == 0 ? C::TILE_WARPS / 4 - 1 : 0)) mbar_arrive_cluster(ovl_leader);
                    if (p + 1 == C::PASSES) mbar_arrive_cluster(tempty_leader0 + 8u * now);
                }
                const int nc = n0 + col[p];
                uint4 blocks[C::CH];
                uint32_t scales[C::CH];
#pragma unroll
                for (int r = 0; r < C::CH; ++r) {
                    f8_act<32, KIND == FP8_OUT_F32 ? GELU_F32 : GELU_BF16>(v[r], bias_line + 32 * r, has_bias, a.act);
                    if constexpr (KIND == FP4_OUT_FP4) {
                        blocks[r] = f4_block(a, v[r], nc + 32 * r, scales[r]);
                    } else if constexpr (KIND == FP4_OUT_BF16_BULK) {
                        stage_bf16(v[r], smem_u32(staged), lane);
                        if (row0 < a.M && nc + 32 * r < a.N) tma_store_2d(&a.tmOut, smem_u32(staged), (nc + 32 * r) * 2, row0);
                        bulk_commit();
                    } else {
                        f4_store32<KIND>(a, v[r], orow, nc + 32 * r, wide, lane);
                    }
                }
                if constexpr (KIND == FP4_OUT_FP4) f4_store_blocks<C::CH>(a, blocks, scales, orow, nc);
            }
            if (C::GROUPS == 2 || now == 1) aph ^= 1;
        }
        if (KIND == FP4_OUT_BF16_BULK) bulk_wait_all();  // the stores read this CTA's shared memory
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // no copy, commit or remote arrival is left in flight towards either CTA
    tc_fence_after();
    if (warp == C::WARP_MMA)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <int BN, int KIND, int NE>
cudaError_t launch_pair(Fp4GemmArgs<NE>& a, int num_sms, cudaStream_t s) {
    using C = P4Cfg<BN, KIND>;
    static_assert(C::SMEM <= 227 * 1024);
    const cudaError_t e = smem_attr_once((const void*)fp4_gemm2_kernel<BN, KIND, NE>, C::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t m_tiles = (a.M + 2 * P4_BM - 1) / (2 * P4_BM) + a.E - 1;
    const int64_t tiles = m_tiles * ((a.N + BN - 1) / BN), pairs = num_sms / 2, units = tiles < pairs ? tiles : pairs;
    a.whole = (int)(tiles / units);
    a.rest = (int)(tiles % units);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * units));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fp4_gemm2_kernel<BN, KIND, NE>, a);
}

template <int KIND, int NE>
cudaError_t launch_kind2(Fp4GemmArgs<NE>& a, int bn, int num_sms, cudaStream_t s) {
    return bn == 256 ? launch_pair<256, KIND>(a, num_sms, s) : launch_pair<128, KIND>(a, num_sms, s);
}

}  // namespace

template <int NE>
cudaError_t launch_fp4_gemm2(Fp4GemmArgs<NE>& a, int bn, int num_sms, cudaStream_t s) {
    if constexpr (NE == 1) {
        if (a.out_kind == FP4_OUT_FP4) return launch_kind2<FP4_OUT_FP4>(a, bn, num_sms, s);
        if (a.tma_out) return launch_kind2<FP4_OUT_BF16_BULK>(a, bn, num_sms, s);
    }
    return a.out_kind == FP8_OUT_BF16 ? launch_kind2<FP8_OUT_BF16>(a, bn, num_sms, s) : launch_kind2<FP8_OUT_F32>(a, bn, num_sms, s);
}
template cudaError_t launch_fp4_gemm2<1>(Fp4GemmArgs<1>&, int, int, cudaStream_t);
template cudaError_t launch_fp4_gemm2<CM_MAX_E>(Fp4GemmArgs<CM_MAX_E>&, int, int, cudaStream_t);

}  // namespace cm
