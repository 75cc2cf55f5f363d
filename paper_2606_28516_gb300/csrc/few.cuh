// The product of a 16-row tile of weights with a few rows of activations, shared by the few-token layer and the
// 8-bit product of few rows.
//
// The warps of a CTA split K. Weights go from global memory straight to the registers they are multiplied from:
// the order of K within a sum is free as long as both operands agree, so lane (g, c) = (lane / 4, lane % 4) takes
// 16 consecutive bytes of weight rows g and g + 8 and the same columns of activation row g, and feeds them to
// m16n8 warp-level MMAs as their fragments. A lane issues the loads of a round (DEPTH steps) before the round's
// products; the depth is what fits 128 registers a thread, so that two CTAs of eight warps share an SM.
#pragma once

#include "common.cuh"
#include "fp8.cuh"

namespace cm {

constexpr int FEW_WARPS = 8;
constexpr int FEW_THREADS = FEW_WARPS * 32;

// Kernel variants by element types: FEWV_W8A8 has 8-bit weights and activations, FEWV_W8A16 8-bit weights and bf16
// activations.
enum FewVar { FEWV_F32 = 0, FEWV_BF16 = 1, FEWV_W8A16 = 2, FEWV_W8A8 = 3 };

template <int V, int NT>
struct FewT {
    static constexpr int LANE = V == FEWV_F32 ? 4 : V == FEWV_BF16 ? 8 : 16;  // weight columns per lane and step
    static constexpr int STEP = 4 * LANE;                                     // and of a warp's step
    static constexpr int WSZ = V == FEWV_F32 ? 4 : V == FEWV_BF16 ? 2 : 1;
    static constexpr int XSZ = V == FEWV_F32 ? 4 : V == FEWV_W8A8 ? 1 : 2;
    static constexpr int XV = LANE * XSZ / 16;  // 16-byte loads of activations per step and token tile
    static constexpr int REGS = 8 + 4 * XV * NT;
    static constexpr int DEPTH = REGS >= 72 ? 1 : REGS >= 40 ? 2 : REGS >= 24 ? 3 : REGS >= 16 ? 5 : 6;
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// v rounded to TF32 (to nearest, ties away from zero) and the remainder, rounded likewise
__device__ __forceinline__ void few_split(uint32_t v, uint32_t& h, uint32_t& l) {
    h = (v + 0x1000u) & 0xFFFFE000u;
    l = __float_as_uint(__uint_as_float(v) - __uint_as_float(h)) + 0x1000u;
}
// Two e4m3 values as a pair of bf16, exactly
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t v) {
    const float2 f = fp8_unpack2(v & 0xFFFFu);
    return pack_bf16(f.x, f.y);
}

__device__ __forceinline__ uint4 few_ld_weight(const void* p) { return __ldg(static_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 few_ld_token(const void* p) { return __ldcg(static_cast<const uint4*>(p)); }

// A 16-row tile of a weight matrix as a lane sees it: its two rows, K columns in use.
struct FewTile {
    const char* w0;
    const char* w1;
    const uint8_t* s;  // 8-bit blocks: scale bytes of the tile's rows
    int K;
};
template <int V>
__device__ __forceinline__ FewTile few_tile(const void* w, const uint8_t* s, int64_t pitch, int64_t lds, int r0, int rows,
                                            int K, int lane) {
    constexpr int WSZ = FewT<V, 1>::WSZ;
    const int g = lane >> 2;
    FewTile t;
    t.w0 = static_cast<const char*>(w) + (int64_t)min(r0 + g, rows - 1) * pitch * WSZ;
    t.w1 = static_cast<const char*>(w) + (int64_t)min(r0 + g + 8, rows - 1) * pitch * WSZ;
    t.s = s ? s + (int64_t)(r0 / 128) * lds : nullptr;
    t.K = K;
    return t;
}

// The weights of one round of a warp: steps i0 .. i0 + DEPTH - 1 of its own, step i being step warp + 8 i of K.
template <int V, int NT>
struct FewRound {
    uint4 a[FewT<V, NT>::DEPTH], b[FewT<V, NT>::DEPTH];
    uint32_t s[FewT<V, NT>::DEPTH];
};
template <int V, int NT>
__device__ __forceinline__ void few_load(FewRound<V, NT>& r, const FewTile& t, int i0, int warp, int lane) {
    using F = FewT<V, NT>;
#pragma unroll
    for (int d = 0; d < F::DEPTH; ++d) {
        const int k = (warp + FEW_WARPS * (i0 + d)) * F::STEP + (lane & 3) * F::LANE;
        r.a[d] = r.b[d] = make_uint4(0, 0, 0, 0);
        r.s[d] = 0;
        if (k < t.K) {  // K is a multiple of a lane's columns
            r.a[d] = few_ld_weight(t.w0 + (int64_t)k * F::WSZ);
            r.b[d] = few_ld_weight(t.w1 + (int64_t)k * F::WSZ);
            if (V >= FEWV_W8A16) r.s[d] = __ldg(t.s + k / 128);
        }
    }
}

// acc[j] += the warp's share of the tile times activation rows 8 j .. 8 j + 7 (tok[j]: the lane's row 8 j + g).
// first: the first round's weights, loaded by the caller. xs[j] (FEWV_W8A8): the scale bytes of the lane's two
// accumulator columns' rows. sums (LN): += W 1.
// Sums: a step's products are added from zero and then to acc in fp32, so that the tensor cores' truncating
// accumulation runs over one step (fp32) or one scale block's part (8 bits) only; bf16 outputs, whose own rounding
// is 2^-9, accumulate in place.
template <int V, int NT, bool LN>
__device__ __forceinline__ void few_product(float (&acc)[NT][4], float (&sums)[4], const FewTile& t,
                                            FewRound<V, NT>& first, const char* const (&tok)[NT],
                                            const uint8_t* const (&xs)[NT][2], int warp, int lane) {
    using F = FewT<V, NT>;
    const int steps = (t.K + F::STEP - 1) / F::STEP;
    for (int i0 = 0; warp + FEW_WARPS * i0 < steps; i0 += F::DEPTH) {
        if (i0) few_load<V, NT>(first, t, i0, warp, lane);
        uint4 x[F::DEPTH][NT][F::XV];
#pragma unroll
        for (int d = 0; d < F::DEPTH; ++d) {
            const int k = (warp + FEW_WARPS * (i0 + d)) * F::STEP + (lane & 3) * F::LANE;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < F::XV; ++q) {
                    x[d][j][q] = make_uint4(0, 0, 0, 0);
                    if (k < t.K) x[d][j][q] = few_ld_token(tok[j] + (int64_t)k * F::XSZ + 16 * q);
                }
        }
#pragma unroll
        for (int d = 0; d < F::DEPTH; ++d) {
            const uint4 a = first.a[d], b = first.b[d];
            const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
            if constexpr (V == FEWV_F32) {
                uint32_t ah[4], al[4], bh[4], bl[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    few_split(wa[i], ah[i], al[i]);
                    few_split(wb[i], bh[i], bl[i]);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint32_t xv[4] = {x[d][j][0].x, x[d][j][0].y, x[d][j][0].z, x[d][j][0].w};
                    uint32_t xh[4], xl[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) few_split(xv[i], xh[i], xl[i]);
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 4; h += 2) {  // the small products first
                        mma_tf32(part, al[h], bl[h], al[h + 1], bl[h + 1], xh[h], xh[h + 1]);
                        mma_tf32(part, ah[h], bh[h], ah[h + 1], bh[h + 1], xl[h], xl[h + 1]);
                    }
#pragma unroll
                    for (int h = 0; h < 4; h += 2)
                        mma_tf32(part, ah[h], bh[h], ah[h + 1], bh[h + 1], xh[h], xh[h + 1]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][i] += part[i];
                }
                if (LN) {
                    const uint32_t one = __float_as_uint(1.f);
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 4; h += 2) mma_tf32(part, al[h], bl[h], al[h + 1], bl[h + 1], one, one);
#pragma unroll
                    for (int h = 0; h < 4; h += 2) mma_tf32(part, ah[h], bh[h], ah[h + 1], bh[h + 1], one, one);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[i] += part[i];
                }
            } else if constexpr (V == FEWV_W8A8) {
                const int blk = (warp + FEW_WARPS * (i0 + d)) * F::STEP / 128;
                const float sw = fp8_scale(first.s[d]);
                const bool in = blk * 128 < t.K;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 v = x[d][j][0];
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                    mma_e4m3(part, wa[0], wb[0], wa[1], wb[1], v.x, v.y);
                    mma_e4m3(part, wa[2], wb[2], wa[3], wb[3], v.z, v.w);
                    if (in) {
                        const float s0 = fp8_scale(__ldcg(xs[j][0] + blk)), s1 = fp8_scale(__ldcg(xs[j][1] + blk));
                        acc[j][0] = fmaf(part[0] * sw, s0, acc[j][0]);
                        acc[j][1] = fmaf(part[1] * sw, s1, acc[j][1]);
                        acc[j][2] = fmaf(part[2] * sw, s0, acc[j][2]);
                        acc[j][3] = fmaf(part[3] * sw, s1, acc[j][3]);
                    }
                }
            } else {
                constexpr int NS = F::LANE / 4;  // MMAs of 16 columns per step: four of the lane's columns each
                uint32_t f[NS][4];
#pragma unroll
                for (int h = 0; h < NS; ++h) {
                    if (V == FEWV_BF16) {
                        f[h][0] = wa[(2 * h) & 3], f[h][1] = wb[(2 * h) & 3];
                        f[h][2] = wa[(2 * h + 1) & 3], f[h][3] = wb[(2 * h + 1) & 3];
                    } else {
                        f[h][0] = fp8x2_to_bf16x2(wa[h & 3]), f[h][1] = fp8x2_to_bf16x2(wb[h & 3]);
                        f[h][2] = fp8x2_to_bf16x2(wa[h & 3] >> 16), f[h][3] = fp8x2_to_bf16x2(wb[h & 3] >> 16);
                    }
                }
                const float sw = V == FEWV_W8A16 ? fp8_scale(first.s[d]) : 1.f;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    uint32_t xv[2 * NS];
#pragma unroll
                    for (int q = 0; q < F::XV; ++q)
                        xv[4 * q] = x[d][j][q].x, xv[4 * q + 1] = x[d][j][q].y, xv[4 * q + 2] = x[d][j][q].z, xv[4 * q + 3] = x[d][j][q].w;
                    if (V == FEWV_W8A16) {
                        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int h = 0; h < NS; ++h)
                            mma_bf16(part, f[h][0], f[h][1], f[h][2], f[h][3], xv[2 * h], xv[2 * h + 1]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(part[i], sw, acc[j][i]);
                    } else {
#pragma unroll
                        for (int h = 0; h < NS; ++h)
                            mma_bf16(acc[j], f[h][0], f[h][1], f[h][2], f[h][3], xv[2 * h], xv[2 * h + 1]);
                    }
                }
                if (LN) {
                    const uint32_t one = 0x3F803F80u;  // a pair of bf16 ones
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < NS; ++h) mma_bf16(part, f[h][0], f[h][1], f[h][2], f[h][3], one, one);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[i] = fmaf(part[i], sw, sums[i]);
                }
            }
        }
    }
}

// The warps' partial sums to shared memory, [warp][8 NT columns][16 rows].
template <int NT>
__device__ __forceinline__ void few_stage(float* red, const float (&acc)[NT][4], int warp, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        float* p = red + ((warp * NT + j) * 8 + 2 * c) * 16;
        p[g] = acc[j][0];
        p[16 + g] = acc[j][1];
        p[g + 8] = acc[j][2];
        p[16 + g + 8] = acc[j][3];
    }
}
// Their sum over the warps, in warp order.
template <int NT>
__device__ __forceinline__ float few_sum(const float* red, int col, int row) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < FEW_WARPS; ++w) s += red[(w * NT * 8 + col) * 16 + row];
    return s;
}
constexpr int few_smem(int nt) { return FEW_WARPS * nt * 128 * 4; }

}  // namespace cm
