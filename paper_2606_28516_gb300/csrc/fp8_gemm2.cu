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
// conversions), each 32 columns of a 128-column block at a time. For 8-bit outputs the block is one scale block: its
// four warps exchange the row's largest magnitudes through shared memory.
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

constexpr int P8_NUM_EPI = 16;
constexpr int P8_WARP_SCALE = 16, P8_WARP_MMA = 18, P8_WARP_TMA = 19;
constexpr int P8_THREADS = 32 * 20;
constexpr int P8_BM = 128;  // rows per CTA
constexpr int P8_BK = 128;

template <int BN_, int KIND>
struct P8Cfg {
    static constexpr int BN = BN_;
    static constexpr int BH = BN / 2;  // W rows per CTA
    static constexpr int A_BYTES = P8_BM * P8_BK, B_BYTES = BH * P8_BK;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    // 8-bit outputs: a tile's rows of bytes, staged for whole-line stores
    static constexpr int OUT_BYTES = KIND == FP8_OUT_FP8 ? P8_BM * BN : 0;
    static constexpr int STAGES = (192 * 1024 - OUT_BYTES) / STAGE_BYTES;
    static constexpr bool OVL = BN == 256;
    static constexpr int ACC1 = OVL ? 224 : BN;  // first column of the second accumulator
    static constexpr int SF_COL = ACC1 + BN;
    static constexpr int SF_COLS = f8_slot_cols(BN), SF_BYTES = f8_slot_bytes(BN);
    static_assert(SF_COL + 2 * SF_COLS <= 512);
    static constexpr int CHUNKS = BN / 32;
    static constexpr int ROUNDS = (CHUNKS + 3) / 4;  // of four 32-column chunks, one per warp of a quarter
    static constexpr int NBARS = 2 * STAGES + 2 * F8_SLOTS + 4 + 3 + 4 * ROUNDS + 4;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + OUT_BYTES + F8_SLOTS * SF_BYTES + P8_NUM_EPI * 32 * 4 + 2 * ROUNDS * P8_NUM_EPI * 32 * 4 + NBARS * 8 + 16 +
                                8 * (CM_MAX_E + 1) + 8;
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
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(P8_THREADS, 1)
    fp8_gemm2_kernel(const __grid_constant__ Fp8GemmArgs a) {
    using C = P8Cfg<BN_, KIND>;
    constexpr int BN = C::BN, STAGES = C::STAGES, SLOTS = F8_SLOTS;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sm = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    unsigned char* s_out = sm + STAGES * C::STAGE_BYTES;                      // [block][row][128], 8-bit outputs
    unsigned char* s_sf = s_out + C::OUT_BYTES;                               // [slot]
    float* s_bias = reinterpret_cast<float*>(s_sf + SLOTS * C::SF_BYTES);      // [epilogue warp][32]
    float* s_amax = s_bias + P8_NUM_EPI * 32;                                  // [2][round][epilogue warp][32]
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_amax + 2 * C::ROUNDS * P8_NUM_EPI * 32);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::NBARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile uint32_t* s_issued = tmem_slot + 2;  // k-blocks this CTA's producer has loaded, once it has stopped
    int* s_prefix = reinterpret_cast<int*>(tmem_slot + 4);  // [E + 1]
    int* s_off = s_prefix + CM_MAX_E + 1;                   // [E + 1]

    pdl_launch_dependents();
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
    auto pair_bar = [&](int q) { return ovl_bar + 24 + 8u * q; };
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
            mbar_init(tempty_bar(i), 2 * P8_NUM_EPI);  // epilogue warps of both CTAs
        }
        mbar_init(ovl_bar, 8);  // the warps whose chunk lies in the shared columns, of both CTAs
        mbar_init(drain_bar, 1);
        mbar_init(stop_bar, 2);
        for (int q = 0; q < 4 * C::ROUNDS + 4; ++q) mbar_init(pair_bar(q), 4);
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == P8_WARP_MMA) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // barriers initialised and tensor memory allocated in both CTAs
    tc_fence_after();
    pdl_wait();  // everything below may read the previous kernel's results
    if (threadIdx.x == 0) f8_groups(a, 2 * P8_BM, s_off, s_prefix);
    __syncthreads();
    const uint32_t tmem = warp_uniform(*tmem_slot);  // all 512 columns: the same base in both CTAs
    const int nkb = a.nkb;
    F8Walk t(blockIdx.x >> 1, gridDim.x >> 1, a.N, 2 * P8_BM, BN, a.E, s_off, s_prefix);

    if (warp == P8_WARP_TMA) {
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
    } else if (warp == P8_WARP_MMA) {
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
    } else if (warp >= P8_WARP_SCALE) {
        // ------------------------------------------------ scales (both CTAs)
        const uint32_t sfull_leader0 = map_to_rank(sfull_bar(0), 0);
        f8_scale_warp<BN>(a, warp - P8_WARP_SCALE, t, (int)rank * P8_BM, lane,
                          [&](const F8Scales<BN>& w, int slot, uint32_t ph) {
                              if (!mbar_wait_warp(sempty_bar(slot), ph ^ 1, abort_flag, a.status, lim)) return false;
                              w.store(s_sf + slot * C::SF_BYTES, lane);
                              fence_proxy_async_smem();
                              __syncwarp();
                              mbar_arrive_release_cluster_warp(sfull_leader0 + 8u * slot);
                              return true;
                          });
    } else {
        // ------------------------------------------------ epilogue (both CTAs, own 128 rows)
        const int quarter = warp & 3, cg = warp >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float* bias_line = s_bias + warp * 32;
        const bool has_bias = a.bias != nullptr;
        const int esz = KIND == FP8_OUT_BF16 ? 2 : 4;
        // rows of the output in whole 32-byte pieces
        const bool wide = KIND == FP8_OUT_FP8 || ((reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && (a.ldo * esz & 31) == 0);
        const uint32_t tempty_leader0 = map_to_rank(tempty_bar(0), 0), ovl_leader = map_to_rank(ovl_bar, 0);
        // What a tile's epilogue needs beside its sums, loaded a tile ahead: a load waits behind the queued tile loads.
        float bias[C::ROUNDS];
        int row = 0;
        auto prefetch = [&](int acc) {
            if (!t.live()) return;
            if (KIND != FP8_OUT_FP8) row = f8_out_row(a, t.m0 + (int)rank * P8_BM + quarter * 32 + lane, t.hi);
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
        uint32_t aph = 0, pph = 0;
        float* ex = s_amax;
        bool ok = true;
        while (t.live() && ok) {
            const int m0 = t.m0 + (int)rank * P8_BM, hi = t.hi, n0 = t.n0, orow = row;
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
            if constexpr (KIND == FP8_OUT_FP8) {
                // All of the tile's sums are read before any is worked on and before the next tile's MMAs start: reads
                // beside MMAs wait for them (133 us against 128, 50,432 x 3,072 x 768). Then every round's values are activated and its magnitudes handed
                // over before the first exchange is waited for, so that arithmetic hides the latencies.
                float v[C::ROUNDS][32];
                {
                    uint32_t u[C::ROUNDS][32];
#pragma unroll
                    for (int r = 0; r < C::ROUNDS; ++r) CM_TMEM_LD_X32(d + chunk[r] * 32, u[r]);
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < C::ROUNDS; ++r) {
                        released(r);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[r][i] = __uint_as_float(u[r][i]);
                    }
                }
#pragma unroll
                for (int r = 0; r < C::ROUNDS; ++r) {
                    if (has_bias) bias_line[lane] = b[r];
                    __syncwarp();
                    f8_act<32, false>(v[r], bias_line, has_bias, a.act);
                    const int nc = n0 + chunk[r] * 32;
                    if (nc + 32 > a.N) {  // columns past N are zero, in the last block's padding and where no block is
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (nc + i >= a.N) v[r][i] = 0.f;
                    }
                    ex[(r * P8_NUM_EPI + warp) * 32 + lane] = f8_max_abs32(v[r]);
                    if (r == 0 && cg == 0) bulk_wait_read();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(pair_bar(quarter * C::ROUNDS + r));
                }
#pragma unroll
                for (int r = 0; r < C::ROUNDS; ++r) {
                    if (!mbar_wait_warp(pair_bar(quarter * C::ROUNDS + r), pph, abort_flag, a.status, lim)) {
                        ok = false;
                        break;
                    }
                    const float* e = ex + (r * P8_NUM_EPI + quarter) * 32 + lane;
                    const float mx = max_abs3(max_abs(e[0], e[4 * 32]), e[8 * 32], e[12 * 32]);
                    const uint32_t s = fp8_scale_byte(abs_bits(mx));
                    const int nc = n0 + chunk[r] * 32, trow = quarter * 32 + lane;
                    uint32_t o[8];
                    fp8_pack32(o, v[r], fp8_inverse_scale(s));
                    // the row's 16-byte pieces 2 cg and 2 cg + 1, piece j at j ^ (row & 7)
                    unsigned char* at = s_out + ((chunk[r] >> 2) * P8_BM + trow) * 128;
                    *reinterpret_cast<uint4*>(at + (((2 * cg) ^ (trow & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<uint4*>(at + (((2 * cg + 1) ^ (trow & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
                    if (cg == 0 && m0 + trow < hi && nc < a.ldo) a.out_scale[(int64_t)(m0 + trow) * a.ldos + nc / 128] = (uint8_t)s;
                }
                if (!ok) break;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(pair_bar(4 * C::ROUNDS + quarter));
                // The quarter's rows as boxes of 32 rows x 128 bytes, by its first warp, which lets them be read before it
                // arrives for the next tile's exchange, and so before any warp writes there again. (Copied out by the
                // warps, whole lines or 32 bytes a lane, the stores cost 0.75 us a tile: 130 us
                // against 114, 50,432 x 3,072 x 768.)
                if (cg == 0) {
                    if (!mbar_wait_warp(pair_bar(4 * C::ROUNDS + quarter), pph, abort_flag, a.status, lim)) break;
#pragma unroll
                    for (int blk = 0; blk < C::ROUNDS; ++blk)
                        if (n0 + blk * 128 < a.ldo)
                            tma_store_2d(&a.tmOut, smem_u32(s_out + (blk * P8_BM + quarter * 32) * 128), (n0 + blk * 128) / 2,
                                         m0 + quarter * 32);
                    bulk_commit();
                }
                // the exchange of the next tile uses the other half: a warp's reads of this one precede its arrivals for
                // the next, and those the other warps' writes two tiles on
                pph ^= 1;
                ex = s_amax + pph * (C::ROUNDS * P8_NUM_EPI * 32);
            } else {
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
            }
            if (++acc == 2) {
                acc = 0;
                aph ^= 1;
            }
        }
    }
    if (KIND == FP8_OUT_FP8 && warp < 4) bulk_wait_all();  // the stores read this CTA's shared memory
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // no copy, commit or remote arrival is left in flight towards either CTA
    tc_fence_after();
    if (warp == P8_WARP_MMA)
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
    cfg.blockDim = dim3(P8_THREADS);
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
