// Products of matrices in 8-bit blocks on pairs of SMs (tcgen05 cta_group::2, sm_103a): fp8_gemm.cu's arithmetic
// in 256 x BN tiles. CTA r of a pair loads A rows [128 r, +128) and W rows [BN / 2 r, +BN / 2) of the tile; the even
// CTA's MMAs (M = 256, N = BN, K = 32) read both halves and leave 128 rows of the accumulator in each CTA's tensor
// memory. Scales: each CTA holds those of its own 128 rows of A and of all BN columns.
//
// What bounds it: at 2 x the bf16 rate a k-block of a 256 x 256 tile takes 512 cycles, in which an SM loads 32 KB;
// 128 x 192 tiles on one SM ask for 107 bytes a cycle where the path from L2 gives about 64, and were bound by it.
//
// Tensor memory: two accumulators of 256 columns and the scale slots do not fit its 512 columns. So the second
// accumulator starts at column 224, 32 columns inside the first: the epilogue reads the shared columns of a tile
// first and says so (ovl_bar), and the next tile's MMAs start then rather than when the whole accumulator is read.
// Columns 480 .. 503 hold two scale slots of 512 of K each. The scales go there by tcgen05.cp from shared memory, which
// the MMA warp issues in line with its MMAs: stored by other warps (tcgen05.st, a hand-over per slot) they waited for
// the accumulator traffic and bounded the kernel, 101 us against 93 for 19,456 x 1,792 x 4,096.
//
// Epilogue: 16 warps (four per lane quarter, so that each scheduler has four to hide the latencies of bias, GELU and
// conversions), each 32 columns of a 128-column block at a time. For 8-bit outputs, whose epilogue takes longer than the
// MMAs (a 128 x 256 tile 5,850 cycles, of which the MMAs need 3,072 and the packed arithmetic of bias, GELU and scaling some
// 2,500; tensor pipe 45 % busy, issue 56 %: no unit is full, its steps wait for one another), two groups of eight take every
// other tile, one accumulator each, so that one group's waits pass under the other's arithmetic; a warp has 64 columns of a
// 128-column scale block and exchanges its rows' largest magnitudes with the warp that has the others. 50,432 x 3,072 x 768
// with bias and GELU: 106 us (2,250 TFLOP/s); all 16 warps on every tile, pair after pair of values, 121; eight warps with 128
// columns a lane and no exchange 106, and 113 in 128-wide tiles against 105. Without bias and GELU 79.
// Hand-offs and giving up as in tc_gemm2.cu: TMA bytes of both CTAs on the even CTA's full barriers, commits on
// both CTAs' empty, sempty and tfull barriers, the scale warp and epilogue warps of both on the even CTA's sfull,
// ovl and tempty; every wait is bounded, and the even CTA lets copies in flight land before the cluster retires.
#include <cstdint>

#include "common.cuh"
#include "drain.h"
#include "fp8.cuh"
#include "fp8_gemm.cuh"
#include "internal.h"
#include "pair.cuh"

namespace cm {

namespace {

constexpr int P8_BM = 128;  // rows per CTA
constexpr int P8_BK = 128;

template <int BN_, int KIND>
struct P8Cfg {
    static constexpr int BN = BN_;
    static constexpr int BH = BN / 2;  // W rows per CTA
    static constexpr bool Q = KIND == FP8_OUT_FP8;
    static constexpr int NUM_EPI = 16;  // epilogue warps
    static constexpr int WARP_SCALE = NUM_EPI, WARP_MMA = NUM_EPI + F8_SCALE_WARPS, WARP_TMA = WARP_MMA + 1;
    static constexpr int THREADS = 32 * (WARP_TMA + 1);
    static constexpr int TILE_WARPS = Q ? NUM_EPI / 2 : NUM_EPI;  // that share a tile's 128 rows
    static constexpr int BIAS_LINE = Q ? 64 : 32;                 // floats per epilogue warp
    static constexpr int A_BYTES = P8_BM * P8_BK, B_BYTES = BH * P8_BK;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int OUT_BYTES = Q ? NUM_EPI * F8_STAGED : 0;
    static constexpr int STAGES = (192 * 1024 - OUT_BYTES) / STAGE_BYTES;
    static constexpr bool OVL = BN == 256;
    static constexpr int ACC1 = OVL ? 224 : BN;  // first column of the second accumulator
    static constexpr int SF_COL = ACC1 + BN;
    static constexpr int SF_COLS = f8_slot_cols(BN), SF_BYTES = f8_slot_bytes(BN);
    static_assert(SF_COL + 2 * SF_COLS <= 512);
    static constexpr int CHUNKS = BN / 32;
    static constexpr int ROUNDS = (CHUNKS + 3) / 4;  // of four 32-column chunks, one per warp of a quarter
    static constexpr int NBARS = 2 * STAGES + 2 * F8_SLOTS + 4 + 3 + (Q ? 8 : 0);
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + F8_SLOTS * SF_BYTES + NUM_EPI * BIAS_LINE * 4 +
                                (Q ? NUM_EPI * 64 * 4 : 0) + NBARS * 8 + 16 + 8 * (CM_MAX_E + 1) + 8;
};

__device__ __forceinline__ void umma2_mxf8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa,
                                           uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(
            d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}

// KIND: Fp8Out.
template <int BN_, int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P8Cfg<BN_, KIND>::THREADS, 1)
    fp8_gemm2_kernel(const __grid_constant__ Fp8GemmArgs a) {
    using C = P8Cfg<BN_, KIND>;
    constexpr int BN = C::BN, STAGES = C::STAGES, SLOTS = F8_SLOTS;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char* s_out = sm + STAGES * C::STAGE_BYTES;                   // [epilogue warp][32 rows][64], 8-bit outputs
    unsigned char* s_sf = s_out + C::OUT_BYTES;                            // [slot]
    float* s_bias = reinterpret_cast<float*>(s_sf + SLOTS * C::SF_BYTES);  // [epilogue warp][BIAS_LINE]
    float* s_amax = s_bias + C::NUM_EPI * C::BIAS_LINE;                    // [epilogue warp][2][32], 8-bit outputs
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_amax + (C::Q ? C::NUM_EPI * 64 : 0));
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
    auto sfull_bar = [&](int s) { return bar0 + 8u * (2 * STAGES + s); };
    auto sempty_bar = [&](int s) { return bar0 + 8u * (2 * STAGES + SLOTS + s); };
    auto tfull_bar = [&](int i) { return bar0 + 8u * (2 * STAGES + 2 * SLOTS + i); };
    auto tempty_bar = [&](int i) { return bar0 + 8u * (2 * STAGES + 2 * SLOTS + 2 + i); };
    const uint32_t ovl_bar = bar0 + 8u * (2 * STAGES + 2 * SLOTS + 4);
    const uint32_t drain_bar = ovl_bar + 8, stop_bar = ovl_bar + 16;
    auto pair_bar = [&](int q) { return ovl_bar + 24 + 8u * q; };  // 8-bit outputs: two warps with the same rows
    const uint64_t lim = (uint64_t)a.wait_limit_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);   // the even CTA's producer arrives; both CTAs' bytes land here
            mbar_init(empty_bar(s), 1);  // one multicast commit per stage
        }
        for (int s = 0; s < SLOTS; ++s) {
            mbar_init(sfull_bar(s), 2);  // the scale warps of both CTAs
            mbar_init(sempty_bar(s), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(tfull_bar(i), 1);
            mbar_init(tempty_bar(i), 2 * C::TILE_WARPS);  // epilogue warps of both CTAs
        }
        mbar_init(ovl_bar, 8);  // the warps whose chunk lies in the shared columns, of both CTAs
        mbar_init(drain_bar, 1);
        mbar_init(stop_bar, 2);
        if constexpr (C::Q)
            for (int q = 0; q < 8; ++q) mbar_init(pair_bar(q), 2);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == C::WARP_MMA) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // barriers initialised and tensor memory allocated in both CTAs
    tc_fence_after();
    pdl_wait();  // everything below may read the previous kernel's results
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    if (threadIdx.x == 0) f8_groups(a, 2 * P8_BM, s_off, s_prefix);
    __syncthreads();
    const uint32_t tmem = warp_uniform(*tmem_slot);  // all 512 columns: the same base in both CTAs
    const int nkb = a.nkb;
    F8Walk t(blockIdx.x >> 1, gridDim.x >> 1, a.N, 2 * P8_BM, BN, a.E, s_off, s_prefix);

    if (warp >= C::NUM_EPI) {
        if (warp == C::WARP_TMA) {
            // ------------------------------------------------ producers (both CTAs)
            const uint32_t full_leader0 = map_to_rank(full_bar(0), 0);
            int stage = 0;
            uint32_t ph = 0, issued = 0;
            bool ok = true;
            for (; warp_uniform((int)t.live()) && ok; t.next()) {
                const int e = warp_uniform(t.e);
                const int m0 = warp_uniform(t.m0 + (int)rank * P8_BM), n0 = warp_uniform(t.n0 + (int)rank * C::BH);
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait_warp(empty_bar(stage), ph ^ 1, abort_flag, a.status, lim)) {
                        ok = false;
                        break;
                    }
                    const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES);
                    const uint32_t fb = full_leader0 + 8u * stage;
                    if (leader) mbar_arrive_expect_tx_warp(full_bar(stage), 2 * C::STAGE_BYTES);
                    // coordinates in the maps' 16-bit elements: two bytes each
                    tma_load_2d_pair(sA, &a.tmA, kb * (P8_BK / 2), m0, fb);
                    tma_load_2d_pair(sA + C::A_BYTES, &a.tmB[e], kb * (P8_BK / 2), n0, fb);
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
                int stage = 0, slot = 0, acc = 0;
                uint32_t ph = 0, sph = 0, aph = 0, oph = 1;  // oph: phase of the previous tile's shared columns
                bool ok = true;
                for (; warp_uniform((int)t.live()) && ok; t.next()) {
                    if (!mbar_wait_warp(tempty_bar(acc), aph ^ 1, abort_flag, a.status, lim)) break;
                    if (C::OVL && !mbar_wait_warp(ovl_bar, oph, abort_flag, a.status, lim)) break;
                    oph ^= 1;
                    tc_fence_after();
                    const uint32_t d = tmem + acc * C::ACC1;
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
                                tmem_cp_scales<2>(sf + 4 * h, smem_u32(s_sf) + slot * C::SF_BYTES + 512 * h);
                        }
                        if (!mbar_wait_warp(full_bar(stage), ph, abort_flag, a.status, lim)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint32_t sA = smem_u32(sm + stage * C::STAGE_BYTES);
                        const uint64_t ad = sdesc_kmajor_sw128(sA), bd = sdesc_kmajor_sw128(sA + C::A_BYTES);
                        const uint32_t id = idesc_mxf8(2 * P8_BM, BN, byte);
    #pragma unroll
                        for (int k = 0; k < 4; ++k)  // 32 of K: 32 bytes on in each row
                            umma2_mxf8(d, ad + 2 * k, bd + 2 * k, id, sf, sf + 4, (kb | k) != 0);
                        umma2_commit_both(empty_bar(stage));
                        if (++stage == STAGES) {
                            stage = 0;
                            ph ^= 1;
                        }
                        if (byte == 3 || kb + 1 == nkb) {
                            umma2_commit_both(sempty_bar(slot));
                            if (++slot == SLOTS) {
                                slot = 0;
                                sph ^= 1;
                            }
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
                    const uint32_t at = smem_u32(tmem_slot + 2);
                    const uint32_t n0 = ld_cluster_u32(map_to_rank(at, 0)), n1 = ld_cluster_u32(map_to_rank(at, 1)), n = max(n0, n1);
    #pragma unroll 1
                    for (uint32_t k = n > STAGES ? n - STAGES : 0; k < n; ++k) {
                        const uint32_t s = k % STAGES;
                        const DrainStep st = drain_step(k, n0, n1);
                        // the odd CTA alone reached it: expect its bytes; the even CTA alone: count the odd one's as landed
                        if (st.arrive) mbar_arrive_expect_tx_warp(full_bar(s), C::STAGE_BYTES);
                        if (st.complete) mbar_complete_tx_warp(full_bar(s), C::STAGE_BYTES);
                        mbar_wait_warp(full_bar(s), (k / STAGES) & 1, nullptr, a.status, 10000000ull);
                    }
                }
            }
            __syncwarp();
        } else {
            // ------------------------------------------------ scales (both CTAs)
            const uint32_t sfull_leader0 = map_to_rank(sfull_bar(0), 0);
            f8_scale_warp<BN>(a, warp - C::WARP_SCALE, t, (int)rank * P8_BM, lane,
                              [&](const F8Scales<BN>& w, int slot, uint32_t ph) {
                                  if (!mbar_wait_warp(sempty_bar(slot), ph ^ 1, abort_flag, a.status, lim)) return false;
                                  w.store(s_sf + slot * C::SF_BYTES, lane);
                                  fence_proxy_async_smem();
                                  __syncwarp();
                                  mbar_arrive_release_cluster_warp(sfull_leader0 + 8u * slot);
                                  return true;
                              });
        }
    } else if constexpr (KIND == FP8_OUT_FP8) {
        // ------------------------------------------------ epilogue (both CTAs, own 128 rows): 8-bit outputs
        const int acc = warp >> 3, half = warp >> 2 & 1, quarter = warp & 3;  // every other tile is its group's
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t tempty_leader = map_to_rank(tempty_bar(acc), 0), ovl_leader = map_to_rank(ovl_bar, 0);
        F8Halves out{a, s_bias + warp * C::BIAS_LINE, s_amax + warp * 64, s_amax + (warp ^ 4) * 64, pair_bar(acc * 4 + quarter),
                     s_out + warp * F8_STAGED, lane};
        // first the block in the columns that the accumulators share
        auto column = [&](int r) { return (C::OVL && acc == 0 ? C::ROUNDS - 1 - r : r) * 128 + half * 64; };
        if (acc && t.live()) t.next();
        if (t.live()) out.prefetch(t.n0 + column(0));
        uint32_t ph = 0;
        bool ok = true;
        while (t.live() && ok) {
            const int row0 = t.m0 + (int)rank * P8_BM + quarter * 32, n0 = t.n0;
            t.next();
            if (t.live()) t.next();
            if (!mbar_wait_warp(tfull_bar(acc), ph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            ph ^= 1;
#pragma unroll 1
            for (int r = 0; r < C::ROUNDS && ok; ++r) {
                float v[64];
                {
                    uint32_t u[64];
                    CM_TMEM_LD_X32(tmem + lanes + acc * C::ACC1 + column(r), u);
                    CM_TMEM_LD_X32(tmem + lanes + acc * C::ACC1 + column(r) + 32, (u + 32));
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(u[i]);
                }
                const bool last = r + 1 == C::ROUNDS;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {  // these columns may be written again
                    if (C::OVL && r == 0 && half == 1 - acc) mbar_arrive_cluster(ovl_leader);
                    if (last) mbar_arrive_cluster(tempty_leader);
                }
                ok = out.store(v, row0, n0 + column(r), last ? (t.live() ? t.n0 + column(0) : -1) : n0 + column(r + 1),
                               [&](uint32_t bar, uint32_t p) { return mbar_wait_warp(bar, p, abort_flag, a.status, lim); });
            }
        }
        bulk_wait_all();  // the stores read this CTA's shared memory
    } else {
        // ------------------------------------------------ epilogue (both CTAs, own 128 rows)
        const int quarter = warp & 3, cg = warp >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float* bias_line = s_bias + warp * 32;
        const bool has_bias = a.bias != nullptr;
        const bool wide = f8_wide(a);
        const uint32_t tempty_leader0 = map_to_rank(tempty_bar(0), 0), ovl_leader = map_to_rank(ovl_bar, 0);
        // What a tile's epilogue needs beside its sums, loaded a tile ahead: a load waits behind the queued tile loads.
        float bias[C::ROUNDS];
        int row = 0;
        auto prefetch = [&](int acc) {
            if (!t.live()) return;
            row = f8_out_row(a, t.m0 + (int)rank * P8_BM + quarter * 32 + lane, t.hi);
            if (has_bias) {
#pragma unroll
                for (int r = 0; r < C::ROUNDS; ++r) {
                    const int n = t.n0 + ((C::OVL && acc == 0 ? C::ROUNDS - 1 - r : r) * 4 + cg) * 32 + lane;
                    bias[r] = n >= a.N      ? 0.f
                              : a.bias_bf16 ? bf16_to_f32(__ldg(static_cast<const uint16_t*>(a.bias) + n))
                                            : __ldg(static_cast<const float*>(a.bias) + n);
                }
            }
        };
        prefetch(0);
        int acc = 0;
        uint32_t aph = 0;
        while (t.live()) {
            const int n0 = t.n0, orow = row;
            // The chunk of round r: the one in the columns that the accumulators share first.
            int chunk[C::ROUNDS];
            float b[C::ROUNDS];
#pragma unroll
            for (int r = 0; r < C::ROUNDS; ++r) {
                chunk[r] = (C::OVL && acc == 0 ? C::ROUNDS - 1 - r : r) * 4 + cg;
                b[r] = bias[r];
            }
            t.next();
            prefetch(acc ^ 1);
            if (!mbar_wait_warp(tfull_bar(acc), aph, abort_flag, a.status, lim)) break;
            tc_fence_after();
            const uint32_t d = tmem + lanes + acc * C::ACC1;
            // after the read of round r: its columns may be written again
            auto released = [&](int r) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (C::OVL && r == 0 && cg == (acc == 0 ? 3 : 0)) mbar_arrive_cluster(ovl_leader);
                    if (r + 1 == C::ROUNDS) mbar_arrive_cluster(tempty_leader0 + 8u * acc);
                }
            };
#pragma unroll
            for (int r = 0; r < C::ROUNDS; ++r) {
                const bool mine = chunk[r] < C::CHUNKS;
                float v[32];
                __syncwarp();
                if (mine) {
                    uint32_t u[32];
                    CM_TMEM_LD_X32(d + chunk[r] * 32, u);
                    if (has_bias) bias_line[lane] = b[r];
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
                }
                released(r);
                const int nc = n0 + chunk[r] * 32;
                if (mine) {
                    f8_act<32, KIND == FP8_OUT_F32>(v, bias_line, has_bias, a.act);
                    f8_store32<KIND>(a, v, orow, nc, wide, lane);
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
    cluster_sync();  // no copy, commit or remote arrival is left in flight towards either CTA
    tc_fence_after();
    if (warp == C::WARP_MMA)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

template <int BN, int KIND>
cudaError_t launch_pair(const Fp8GemmArgs& a, int num_sms, cudaStream_t s) {
    using C = P8Cfg<BN, KIND>;
    static_assert(C::SMEM <= 227 * 1024);
    const cudaError_t e = smem_attr_once((const void*)fp8_gemm2_kernel<BN, KIND>, C::SMEM);
    if (e != cudaSuccess) return e;
    const int64_t m_tiles = (a.M + 2 * P8_BM - 1) / (2 * P8_BM) + (a.offsets ? a.E - 1 : 0);
    const int64_t tiles = m_tiles * ((a.N + BN - 1) / BN), pairs = num_sms / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs)));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fp8_gemm2_kernel<BN, KIND>, a);
}

template <int KIND>
cudaError_t launch_kind2(const Fp8GemmArgs& a, int bn, int num_sms, cudaStream_t s) {
    if (bn == 256) return launch_pair<256, KIND>(a, num_sms, s);
    if (bn == 128) return launch_pair<128, KIND>(a, num_sms, s);
    if constexpr (KIND != FP8_OUT_FP8) {
        if (bn == 192) return launch_pair<192, KIND>(a, num_sms, s);
    }
    return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_fp8_gemm2(const Fp8GemmArgs& a, int bn, int num_sms, cudaStream_t s) {
    return a.out_kind == FP8_OUT_FP8    ? launch_kind2<FP8_OUT_FP8>(a, bn, num_sms, s)
           : a.out_kind == FP8_OUT_BF16 ? launch_kind2<FP8_OUT_BF16>(a, bn, num_sms, s)
                                        : launch_kind2<FP8_OUT_F32>(a, bn, num_sms, s);
}

}  // namespace cm
