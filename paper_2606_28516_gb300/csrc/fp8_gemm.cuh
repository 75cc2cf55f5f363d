// Pieces shared by the kernels of products in 8-bit blocks: descriptors, tiles, epilogue arithmetic.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "pair.cuh"

namespace cm {

// Instruction descriptor of kind::mxf8f6f4: e4m3 A and W, both K-major, UE8M0 scales; `byte` selects the byte of
// each scale word.
__device__ __forceinline__ uint32_t idesc_mxf8(int M, int N, int byte) {
    return ((uint32_t)byte << 4) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 4) << 24) |
           ((uint32_t)byte << 29);
}
// 32 rows of 16 bytes at smem (contiguous: core matrices of 8 rows, 128 bytes apart, no swizzle) to four columns of
// tensor memory, lanes 0 .. 31 and again in each other quarter; CG 2: in both CTAs of a pair, each from its own. In
// order with the MMAs issued by the same lane.
template <int CG>
__device__ __forceinline__ void tmem_cp_scales(uint32_t tmem, uint32_t smem) {
    const uint64_t desc = (uint64_t)((smem & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
            "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem),
            "l"(desc)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
            "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem),
            "l"(desc)
            : "memory");
}
#define CM_TMEM_LD_X32(taddr, r)                                                                                        \
    asm volatile(                                                                                                       \
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19," \
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                                                      \
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),   \
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),        \
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),       \
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])                     \
        : "r"(taddr))


// Row boundaries of the groups and the row tiles before each, in shared memory: off[E + 1], prefix[E + 1]. Held to
// ascend within the rows: after a routing that gave up they may be an earlier call's.
__device__ __forceinline__ void f8_groups(const Fp8GemmArgs& a, int bm, int* off, int* prefix) {
    int acc = 0;
    for (int e = 0; e <= a.E; ++e) {
        const int v = a.offsets ? __ldcg(a.offsets + e) : (e == 0 ? 0 : (int)a.M);
        off[e] = min(max(v, acc), (int)a.M);
        acc = off[e];
    }
    acc = 0;
    for (int e = 0; e < a.E; ++e) {
        prefix[e] = acc;
        acc += (off[e + 1] - off[e] + bm - 1) / bm;
    }
    prefix[a.E] = acc;
}
// A CTA's (or pair's) walk over the tiles first, first + step, ...: row tile by row tile, columns fastest. m0: the tile's
// first row, of the group's rows up to hi. Advanced by additions (a division and a search per tile and warp were an
// eighth of the epilogue's instructions).
struct F8Walk {
    int mt, nt;  // row and column tile
    int e, m0, hi, n0;
    int n_tiles, bm, bn, E, step_mt, step_nt;
    const int* off;
    const int* prefix;
    __device__ __forceinline__ F8Walk(int first, int step, int N, int bm_, int bn_, int E_, const int* off_, const int* prefix_)
        : e(0), n_tiles((N + bn_ - 1) / bn_), bm(bm_), bn(bn_), E(E_), off(off_), prefix(prefix_) {
        mt = first / n_tiles;
        nt = first - mt * n_tiles;
        step_mt = step / n_tiles;
        step_nt = step - step_mt * n_tiles;
        place();
    }
    __device__ __forceinline__ bool live() const { return mt < prefix[E]; }
    __device__ __forceinline__ void next() {
        mt += step_mt;
        nt += step_nt;
        if (nt >= n_tiles) {
            nt -= n_tiles;
            ++mt;
        }
        place();
    }
    __device__ __forceinline__ void place() {
        while (e + 1 < E && prefix[e + 1] <= mt) ++e;
        m0 = off[e] + (mt - prefix[e]) * bm;
        hi = off[e + 1];
        n0 = nt * bn;
    }
};

// The output row of row m of A (-1: none). An index outside the output, of a routing that gave up, is no row.
template <class Args>
__device__ __forceinline__ int f8_out_row(const Args& a, int m, int hi) {
    if (m >= hi) return -1;
    if (!a.rows) return m;
    const int r = __ldcg(a.rows + m);
    return (uint32_t)r < (uint32_t)a.M ? r : -1;
}

// The scale words of one 512-column chunk as a lane of the scale warp holds them: rows 32 j + lane of the CTA's 128
// rows of A, and those of W's blocks (columns n0 + 32 j of the tile lie in one block of 128 rows). Tensor memory
// holds the word of row 32 j + l in lane l (of every quarter) and column j, which is what tcgen05.cp makes of 32
// rows of 16 bytes in shared memory.
constexpr int f8_slot_bytes(int bn) { return 512 * (1 + (bn + 127) / 128); }
constexpr int f8_slot_cols(int bn) { return 4 * (1 + (bn + 127) / 128); }
template <int BN>
struct F8Scales {
    static constexpr int NW = BN % 128 == 0 ? BN / 128 : BN >= 64 ? BN / 64 : 1;  // different words of W at most
    static constexpr int SPAN = BN / NW;                                          // columns of each
    uint32_t a[4], w[NW];
    __device__ __forceinline__ void load(const Fp8GemmArgs& g, const F8Walk& t, int m0, int chunk, int lane) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // rows past the group's end: any row's scales will do
            const int r = min(m0 + 32 * j + lane, t.hi - 1);
            a[j] = __ldcg(reinterpret_cast<const uint32_t*>(g.sa + (int64_t)r * g.lds) + chunk);
        }
        const uint8_t* sb = g.sb[t.e];
#pragma unroll
        for (int j = 0; j < NW; ++j)
            w[j] = __ldcg(reinterpret_cast<const uint32_t*>(sb + (int64_t)(min(t.n0 + SPAN * j, g.N - 1) / 128) * g.lds) + chunk);
    }
    // to a slot in shared memory (f8_slot_bytes): 16 bytes a lane for A, and for each 128 columns of the tile
    __device__ __forceinline__ void store(unsigned char* slot, int lane) const {
        *reinterpret_cast<uint4*>(slot + lane * 16) = make_uint4(a[0], a[1], a[2], a[3]);
#pragma unroll
        for (int h = 0; h < (BN + 127) / 128; ++h) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = 128 * h + 32 * j < BN ? w[(128 * h + 32 * j) / SPAN] : 0u;
            *reinterpret_cast<uint4*>(slot + 512 * (1 + h) + lane * 16) = make_uint4(b[0], b[1], b[2], b[3]);
        }
    }
};

constexpr int F8_SLOTS = 4;  // scale slots in shared memory, each 512 of K; two of them at a time in tensor memory
constexpr int F8_SCALE_WARPS = 2;
constexpr int F8_AHEAD = 2;

// The work of scale warp `which` of F8_SCALE_WARPS: the words of every F8_SCALE_WARPS-th 512-column chunk of the CTA's
// tiles, in order, each handed to put(words, slot, phase), false when it gave up. Two warps, because a chunk takes a
// warp over a microsecond from the free slot to the arrival (loads that wait behind the queued tile loads, the fence
// between the proxies): one warp 93 us, four 83, two
// 83 for 19,456 x 1,792 x 4,096 in 256 x 256 tiles.
// F8_AHEAD chunks' loads are in flight; a set of registers is loaded again as soon as its words are stored (a set
// moved to another would wait for its loads).
template <int BN, class Put>
__device__ __forceinline__ void f8_scale_warp(const Fp8GemmArgs& a, int which, F8Walk t, int row0, int lane, Put put) {
    const int nsb = (a.nkb + 3) / 4;
    F8Scales<BN> w[F8_AHEAD];
    int c = which;  // the next chunk to load: its place in tile t
    auto load_next = [&](F8Scales<BN>& x) {
        while (c >= nsb && t.live()) {
            c -= nsb;
            t.next();
        }
        if (!t.live()) return false;
        x.load(a, t, t.m0 + row0, c, lane);
        c += F8_SCALE_WARPS;
        return true;
    };
    bool full[F8_AHEAD];
#pragma unroll
    for (int i = 0; i < F8_AHEAD; ++i) full[i] = load_next(w[i]);
    for (uint32_t at = which;;) {  // chunk number, as far as slots and phases go
#pragma unroll
        for (int i = 0; i < F8_AHEAD; ++i) {
            if (!full[i] || !put(w[i], (int)(at % F8_SLOTS), at / F8_SLOTS & 1)) return;
            full[i] = load_next(w[i]);
            at += F8_SCALE_WARPS;
        }
    }
}

__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// v[i] of lane r becomes v[r] of lane i: a 32 x 32 transposition across the warp.
__device__ __forceinline__ void f8_transpose(float (&v)[32], int lane) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (i & o) continue;
            const float send = up ? v[i] : v[i + o];
            const float got = __shfl_xor_sync(0xFFFFFFFFu, send, o);
            if (up)
                v[i] = got;
            else
                v[i + o] = got;
        }
    }
}

// Rows of an fp32 or bf16 output in whole 32-byte pieces.
template <class Args>
__host__ __device__ __forceinline__ bool f8_wide(const Args& a) {
    return (reinterpret_cast<uintptr_t>(a.out) & 31) == 0 && (a.ldo * (a.out_kind == FP8_OUT_BF16 ? 2 : 4) & 31) == 0;
}

// 32 rows' 32 columns [nc, nc + 32) (one row a lane: its output row, or -1) to out, fp32 or bf16. Rows in whole 32-byte
// pieces (wide) are stored as each lane has them; others transposed first, so that a store's lanes write consecutive
// columns of one row (an element a lane, rows apart, took 9.8 us for 1,001 x 777 x 1,131 where this takes 5.7; with each
// row's number shuffled from its lane, 2,922 x 3,453 x 60 to bf16 took 18.5 us where this takes 13.8).
template <int KIND, class Args>
__device__ __forceinline__ void f8_store32(const Args& a, float (&v)[32], int row, int nc, bool wide, int lane) {
    if (wide && nc + 32 <= a.N) {
        if (row < 0) return;
        if constexpr (KIND == FP8_OUT_BF16) {
            uint16_t* o = static_cast<uint16_t*>(a.out) + (int64_t)row * a.ldo + nc;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[16 * p + 2 * i], v[16 * p + 2 * i + 1]);
                st_global_32(o + 16 * p, w);
            }
        } else {
            float* o = static_cast<float*>(a.out) + (int64_t)row * a.ldo + nc;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * p + i]);
                st_global_32(o + 8 * p, w);
            }
        }
        return;
    }
    __syncwarp();
    f8_transpose(v, lane);
    const bool mine = nc + lane < a.N;
    auto put = [&](int64_t at, float f) {
        if constexpr (KIND == FP8_OUT_BF16)
            static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(f);
        else
            static_cast<float*>(a.out)[at] = f;
    };
    if (!a.rows) {  // consecutive rows from lane 0's on: without their shuffles a store waits for nothing
        const int rows = __popc(__ballot_sync(0xFFFFFFFFu, row >= 0)), n = mine ? rows : 0;
        using T = std::conditional_t<KIND == FP8_OUT_BF16, uint16_t, float>;
        T* o = static_cast<T*>(a.out) + (int64_t)__shfl_sync(0xFFFFFFFFu, row, 0) * a.ldo + nc + lane;
#pragma unroll
        for (int r = 0; r < 32; ++r, o += a.ldo) {
            if (r < n) {
                if constexpr (KIND == FP8_OUT_BF16)
                    *o = f32_to_bf16(v[r]);
                else
                    *o = v[r];
            }
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 32; ++r) {
        const int64_t orow = __shfl_sync(0xFFFFFFFFu, row, r);
        if (orow >= 0 && mine) put(orow * a.ldo + nc + lane, v[r]);
    }
}

// gelu_pair_bf16 for P pairs at once, step by step, so that a step's latency passes under the other pairs' (50,432 x 3,072 x
// 768 with 8-bit outputs, on pairs of SMs: one pair after another 122 us, two at a time 109, four 106, eight 106), and with
// max(u, 0) taken directly, two operations a pair less: -inf gives 0, GELU's limit, instead of NaN.
template <int P>
__device__ __forceinline__ void gelu_pairs_fp8(float* u) {
    float2 v[P], q[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
        v[i] = make_float2(fmaxf(-fabsf(u[2 * i]), GeluE::HOLD), fmaxf(-fabsf(u[2 * i + 1]), GeluE::HOLD));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(make_float2(GeluE::C6, GeluE::C6), v[i], make_float2(GeluE::C5, GeluE::C5));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(GeluE::C4, GeluE::C4));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(GeluE::C3, GeluE::C3));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(GeluE::C2, GeluE::C2));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(GeluE::C1, GeluE::C1));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(-1.f, -1.f));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = make_float2(ex2_approx(q[i].x), ex2_approx(q[i].y));
#pragma unroll
    for (int i = 0; i < P; ++i) {
        float2 r;  // NaN stays NaN
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r.x) : "f"(u[2 * i]));
        asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r.y) : "f"(u[2 * i + 1]));
        r = __ffma2_rn(v[i], q[i], r);
        u[2 * i] = r.x, u[2 * i + 1] = r.y;
    }
}

// gelu_pair_bf16 for P pairs at once in the same way, of products in 4-bit blocks whichever kernel they take: NaN for -inf as
// for NaN, by max(u, 0) = u - min(u, 0), which is exact. It costs an operation a value (8,192 x 4,096 x 1,024 to 4-bit blocks
// 22.5 us with -inf to 0, 23.6 so; 25.6 with the difference packed, whose register pairs spilled; 29.1 with gelu_pair_f32).
template <int P>
__device__ __forceinline__ void gelu_pairs_bf16(float* u) {
    float2 v[P], q[P];
#pragma unroll
    for (int i = 0; i < P; ++i)
        v[i] = make_float2(fmaxf(-fabsf(u[2 * i]), GeluE::HOLD), fmaxf(-fabsf(u[2 * i + 1]), GeluE::HOLD));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(make_float2(GeluE::C6, GeluE::C6), v[i], make_float2(GeluE::C5, GeluE::C5));
    constexpr float C[5] = {GeluE::C4, GeluE::C3, GeluE::C2, GeluE::C1, -1.f};
#pragma unroll
    for (int k = 0; k < 5; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) q[i] = __ffma2_rn(q[i], v[i], make_float2(C[k], C[k]));
#pragma unroll
    for (int i = 0; i < P; ++i) q[i] = make_float2(ex2_approx(q[i].x), ex2_approx(q[i].y));
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const float2 relu = make_float2(u[2 * i] - fminf(u[2 * i], 0.f), u[2 * i + 1] - fminf(u[2 * i + 1], 0.f));
        const float2 r = __ffma2_rn(v[i], q[i], relu);
        u[2 * i] = r.x, u[2 * i + 1] = r.y;
    }
}

enum F8Gelu { GELU_8BIT = 0, GELU_F32 = 1, GELU_BF16 = 2 };  // by gelu_pairs_fp8, gelu_pair_f32, gelu_pairs_bf16
// CW accumulator columns + bias, activation; bias from the warp's shared-memory line.
template <int CW, int GELU>
__device__ __forceinline__ void f8_act(float (&v)[CW], const float* s_bias, bool has_bias, int act) {
    if (has_bias) {
#pragma unroll
        for (int i = 0; i < CW; i += 4) {
            const float4 b = *reinterpret_cast<const float4*>(s_bias + i);
            const float2 lo = __fadd2_rn(make_float2(v[i], v[i + 1]), make_float2(b.x, b.y));
            const float2 hi = __fadd2_rn(make_float2(v[i + 2], v[i + 3]), make_float2(b.z, b.w));
            v[i] = lo.x, v[i + 1] = lo.y, v[i + 2] = hi.x, v[i + 3] = hi.y;
        }
    }
    if (act == CLEARMOE_ACT_GELU) {
        if constexpr (GELU == GELU_F32) {
#pragma unroll
            for (int i = 0; i < CW; i += 2) {
                const float2 g = gelu_pair_f32(make_float2(v[i], v[i + 1]));
                v[i] = g.x, v[i + 1] = g.y;
            }
        } else if constexpr (GELU == GELU_BF16) {
#pragma unroll
            for (int i = 0; i < CW; i += 8) gelu_pairs_bf16<4>(v + i);
        } else {
#pragma unroll
            for (int i = 0; i < CW; i += 8) gelu_pairs_fp8<4>(v + i);
        }
    } else if (act == CLEARMOE_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < CW; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];  // NaN stays NaN
    }
}
__device__ __forceinline__ float f8_max_abs32(const float (&v)[32]) {
    float m[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
        m[0] = max_abs3(m[0], v[i], v[i + 1]);
        m[1] = max_abs3(m[1], v[i + 2], v[i + 3]);
    }
    return max_abs(m[0], m[1]);
}

// 8-bit outputs of an epilogue warp: a row a lane and 64 columns, half of a scale block, at a time. The warp with the same
// rows' other half is its mate; they exchange the rows' largest magnitudes through shared memory, in two buffers by block:
// a warp's read of one precedes its arrival for the next block, and that the mate's write two blocks on.
constexpr int F8_STAGED = 32 * 64;  // bytes of a warp's staged half block
struct F8Halves {
    const Fp8GemmArgs& a;
    float* line;            // [64] of the warp: the bias of its columns
    float* amax;            // [2][32] of the warp; its mate's
    const float* mate;
    uint32_t bar;           // both warps arrive
    unsigned char* staged;  // [32][64] of the warp
    int lane;
    uint32_t ph = 0;
    uint32_t b[2];  // as loaded, bf16 or fp32: converted here, it would be waited for here
    // The bias of columns [n, n + 64), a block ahead: a load waits behind the queued tile loads.
    __device__ __forceinline__ void prefetch(int n) {
        if (!a.bias) return;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = n + 32 * i + lane;
            b[i] = 0;
            if (c < a.N) {
                b[i] = a.bias_bf16 ? __ldcg(static_cast<const uint16_t*>(a.bias) + c) : __ldcg(static_cast<const uint32_t*>(a.bias) + c);
            }
        }
    }
    // The sums of rows row0 .. row0 + 31 and columns [n, n + 64) to bytes and scales; next: the columns of the block after
    // this one, or -1. The bytes leave by a bulk copy of 32 rows of 64 bytes, from shared memory where piece j of 16 bytes
    // of row i lies at j ^ (i >> 1 & 3). False when the mate gave up.
    template <class Wait>
    __device__ __forceinline__ bool store(float (&v)[64], int row0, int n, int next, Wait wait) {
        if (a.bias) {
#pragma unroll
            for (int i = 0; i < 2; ++i) line[32 * i + lane] = __uint_as_float(a.bias_bf16 ? b[i] << 16 : b[i]);
            __syncwarp();
        }
        if (next >= 0) prefetch(next);
        f8_act<64, GELU_8BIT>(v, line, a.bias != nullptr, a.act);
        if (n + 64 > a.N) {  // columns past N are zero, in the last block's padding and where no block is
#pragma unroll
            for (int i = 0; i < 64; ++i)
                if (n + i >= a.N) v[i] = 0.f;
        }
        float m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 64; i += 8)
#pragma unroll
            for (int j = 0; j < 4; ++j) m[j] = max_abs3(m[j], v[i + 2 * j], v[i + 2 * j + 1]);
        const float mine = max_abs3(max_abs(m[0], m[1]), m[2], m[3]);
        amax[ph * 32 + lane] = mine;
        bulk_wait_read();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
        if (!wait(bar, ph)) return false;
        const uint32_t s = fp8_scale_byte(abs_bits(max_abs(mine, mate[ph * 32 + lane])));
        ph ^= 1;
        const float inv = fp8_inverse_scale(s);
        const float2 k = make_float2(inv, inv);
        const uint32_t at = smem_u32(staged) + lane * 64;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float* w = v + 16 * p + 4 * i;
                const float2 x = __fmul2_rn(make_float2(w[0], w[1]), k), y = __fmul2_rn(make_float2(w[2], w[3]), k);
                o[i] = fp8_pack4(x.x, x.y, y.x, y.y);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + ((p ^ (lane >> 1 & 3)) << 4)), "r"(o[0]), "r"(o[1]),
                         "r"(o[2]), "r"(o[3])
                         : "memory");
        }
        if ((n & 64) == 0 && row0 + lane < a.M && n < a.ldo)
            a.out_scale[(int64_t)(row0 + lane) * a.ldos + n / 128] = (uint8_t)s;
        fence_proxy_async_smem();
        __syncwarp();
        if (n < a.ldo && row0 < a.M) tma_store_2d(&a.tmOut, smem_u32(staged), n, row0);
        bulk_commit();
        return true;
    }
};

}  // namespace cm
