// The product of a 16-row tile of weights with a few rows of activations, shared by the few-token layer and the
// 8-bit product of few rows.
//
// What bounds it is reading the weights once, so every byte is asked for early. The warps of a CTA split K, step by
// step. Weights go from global memory straight to the registers they are multiplied from: the order of K within a sum
// is free as long as both operands agree, so lane (g, c) = (lane / 4, lane % 4) takes 16 consecutive bytes of weight
// rows g and g + 8 and the same columns of activation row g, and feeds them to m16n8 warp-level MMAs as their
// fragments. A register is loaded again for a step further on as soon as it has been multiplied, so that a lane always
// has several steps' loads in flight, as many as fit beside the sums. The partial sums of the warps are added in warp
// order through shared memory.
// (Queues in shared memory filled by cp.async, with more bytes in flight and no registers held, were slower: two warps a
// scheduler do not hide the copies' and reads' own instructions, and large blocks keep the next kernel from starting
// early. One token, d = 768, 8-bit weights: 9.7 us against 5.4, both with z in one part, 5.9 in two; 64 tokens, bf16: 24.4
// against 18.2.)
#pragma once

#include "common.cuh"
#include "fp8.cuh"

namespace cm {

constexpr int FEW_WARPS = 8;
constexpr int FEW_THREADS = FEW_WARPS * 32;  // of kernels with two or three CTAs an SM

// Kernel variants by element types: FEWV_W8A8 has 8-bit weights and activations, FEWV_W8A16 8-bit weights and bf16
// activations.
enum FewVar { FEWV_F32 = 0, FEWV_BF16 = 1, FEWV_W8A16 = 2, FEWV_W8A8 = 3 };

// NT token tiles of 8 columns; CTAS of the kernel's CTAs share an SM: two where there are few, three where there are
// more than the SMs take at once, so that one's start and end hide behind the others' loads; one of twice the warps where
// the CTAs with work leave an SM to each.
template <int V, int NT, int CTAS>
struct FewT {
    static constexpr int WARPS = CTAS == 1 ? 2 * FEW_WARPS : FEW_WARPS, THREADS = 32 * WARPS;
    static constexpr int LANE = V == FEWV_F32 ? 4 : V == FEWV_BF16 ? 8 : 16;  // weight columns per lane and step
    static constexpr int STEP = 4 * LANE;                                     // and of a warp's step
    static constexpr int WSZ = V == FEWV_F32 ? 4 : V == FEWV_BF16 ? 2 : 1;
    static constexpr int XSZ = V == FEWV_F32 ? 4 : V == FEWV_W8A8 ? 1 : 2;
    static constexpr int XV = LANE * XSZ / 16;  // 16-byte loads of activations per step and token tile
    // Steps of weights and of activations in flight, 8 and 4 XV NT registers each
    static constexpr int XR = XV * NT;
    static constexpr int DW = CTAS <= 2 ? (XR == 1 ? 8 : XR == 2 ? 6 : XR == 4 ? 4 : 2) : (XR <= 2 ? 4 : 2);
    static constexpr int DX = CTAS <= 2 ? (XR == 1 ? 4 : XR == 2 ? 3 : XR == 4 ? 2 : 1) : (XR <= 2 ? 2 : 1);
    static_assert(DW % DX == 0);
    static constexpr int SMEM = WARPS * NT * 128 * 4;  // the partial sums
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// v rounded to TF32 (to nearest, ties away from zero) and the exact remainder, which the tensor cores cut to TF32: of at
// most 13 bits, so that three of its last at 2^-24 of v are lost. Not rounded by integer arithmetic as v is: a NaN of
// arithmetic has all its bits set, which makes h a zero, and only the remainder then is the NaN that the sum has to be. Of
// an infinity, and past TF32's largest value (3.4e38), the remainder is a NaN or an infinity against h's, and the sum NaN.
__device__ __forceinline__ void few_split(uint32_t v, uint32_t& h, uint32_t& l) {
    h = (v + 0x1000u) & 0xFFFFE000u;
    l = __float_as_uint(__uint_as_float(v) - __uint_as_float(h));
}
// Two e4m3 values as a pair of fp16, exactly
__device__ __forceinline__ uint32_t fp8x2_to_f16x2(uint32_t v) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)v));
    return h;
}
// Two e4m3 values as a pair of bf16, exactly
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t v) {
    const float2 f = fp8_unpack2(v & 0xFFFFu);
    return pack_bf16(f.x, f.y);
}

// A 16-row tile of weights and its activation rows as a lane sees them. Step i of a warp is columns
// [STEP (warp + WARPS i), + STEP) of K; the lane's bytes of it start at w0 + i * (stride), w1 and tok[j] likewise.
template <int V, int NT, int CTAS>
struct FewTile {
    using F = FewT<V, NT, CTAS>;
    const char* w0;
    const char* w1;
    const char* tok[NT];
    int steps, in;  // the warp's steps, and how many of them lie inside K for this lane (K is a multiple of LANE)
    uint4 a[F::DW], b[F::DW], x[F::DX][NT][F::XV];
    float3 norm[NT];  // fp32 with the LayerNorm: of the lane's activation rows, as FewRow::stats gives them
    __device__ __forceinline__ int column() const {
        return ((int)threadIdx.x >> 5) * F::STEP + (threadIdx.x & 3) * F::LANE;
    }
    __device__ __forceinline__ void set_weights(const void* base, int64_t pitch_bytes, int r0, int n_rows, int K) {
        const int g = (threadIdx.x >> 2) & 7, k = column(), warp = threadIdx.x >> 5, all = (K + F::STEP - 1) / F::STEP;
        w0 = static_cast<const char*>(base) + (int64_t)min(r0 + g, n_rows - 1) * pitch_bytes + (int64_t)k * F::WSZ;
        w1 = static_cast<const char*>(base) + (int64_t)min(r0 + g + 8, n_rows - 1) * pitch_bytes + (int64_t)k * F::WSZ;
        steps = all > warp ? (all - warp + F::WARPS - 1) / F::WARPS : 0;
        in = K > k ? (K - k + F::WARPS * F::STEP - 1) / (F::WARPS * F::STEP) : 0;
    }
    __device__ __forceinline__ void set_row(int j, const void* row) {
        tok[j] = static_cast<const char*>(row) + (int64_t)column() * F::XSZ;
    }
    __device__ __forceinline__ void load_w(int d, int i) {
        a[d] = b[d] = make_uint4(0, 0, 0, 0);
        if (i < in) {
            a[d] = __ldg(reinterpret_cast<const uint4*>(w0 + (int64_t)i * (F::WARPS * F::STEP * F::WSZ)));
            b[d] = __ldg(reinterpret_cast<const uint4*>(w1 + (int64_t)i * (F::WARPS * F::STEP * F::WSZ)));
        }
    }
    __device__ __forceinline__ void load_x(int d, int i) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < F::XV; ++q) {
                x[d][j][q] = make_uint4(0, 0, 0, 0);
                if (i < in)
                    x[d][j][q] = __ldcg(reinterpret_cast<const uint4*>(tok[j] + (int64_t)i * (F::WARPS * F::STEP * F::XSZ)) + q);
            }
    }
    // The first steps' loads: the weights' before the activations may be read.
    __device__ __forceinline__ void start_w() {
#pragma unroll
        for (int d = 0; d < F::DW; ++d) load_w(d, d);
    }
    __device__ __forceinline__ void start_x() {
#pragma unroll
        for (int d = 0; d < F::DX; ++d) load_x(d, d);
    }
};

// acc[j] += the warp's share of the tile (weights and activations started) times its activation rows. sw (8-bit weights): the scale bytes of the
// tile's rows; sx (FEWV_W8A8): those of the activation rows, ldx bytes apart, rows past the last as the last; both in
// shared memory (255 among them: the sums of its row or column mean nothing). LN: sums += W 1, or (fp32)
// the activation rows are normalised on the way.
// A step's products are added from zero and then to acc in fp32, so that the tensor cores' truncating accumulation
// runs over one step (fp32) or one scale block's part (8 bits) only; bf16 outputs, whose own rounding is 2^-9,
// accumulate in place.
template <int V, int NT, int CTAS, bool LN>
__device__ __forceinline__ void few_product(float (&acc)[NT][4], float (&sums)[4], FewTile<V, NT, CTAS>& t, const uint8_t* sw,
                                            const uint8_t* sx, int ldx, int rows) {
    using F = FewT<V, NT, CTAS>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i0 = 0; i0 < t.steps; i0 += F::DW) {
#pragma unroll
        for (int d = 0; d < F::DW; ++d) {
            const int i = i0 + d, xd = d % F::DX;
            if (i >= t.steps) break;
            const uint32_t wa[4] = {t.a[d].x, t.a[d].y, t.a[d].z, t.a[d].w}, wb[4] = {t.b[d].x, t.b[d].y, t.b[d].z, t.b[d].w};
            const int blk = (warp + F::WARPS * i) * F::STEP / 128;  // of 8-bit weights: a step lies in one block
            if constexpr (V == FEWV_F32) {
                uint32_t ah[4], al[4], bh[4], bl[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    few_split(wa[h], ah[h], al[h]);
                    few_split(wb[h], bh[h], bl[h]);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 v = t.x[xd][j][0];
                    const uint32_t xv[4] = {v.x, v.y, v.z, v.w};
                    uint32_t xh[4], xl[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        // past K a lane's zeros become numbers, against weights that are zero
                        const uint32_t y = LN ? __float_as_uint((__uint_as_float(xv[h]) - t.norm[j].x - t.norm[j].y) * t.norm[j].z) : xv[h];
                        few_split(y, xh[h], xl[h]);
                    }
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 4; h += 2) {  // the small products first
                        mma_tf32(part, al[h], bl[h], al[h + 1], bl[h + 1], xh[h], xh[h + 1]);
                        mma_tf32(part, ah[h], bh[h], ah[h + 1], bh[h + 1], xl[h], xl[h + 1]);
                    }
#pragma unroll
                    for (int h = 0; h < 4; h += 2) mma_tf32(part, ah[h], bh[h], ah[h + 1], bh[h + 1], xh[h], xh[h + 1]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[j][c] += part[c];
                }
            } else if constexpr (V == FEWV_W8A8) {
                // both operands widened to fp16, exactly (the warp-level e4m3 MMA is no faster)
                const uint32_t s = sw[blk];
                uint32_t f[4][4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    f[h][0] = fp8x2_to_f16x2(wa[h]), f[h][1] = fp8x2_to_f16x2(wb[h]);
                    f[h][2] = fp8x2_to_f16x2(wa[h] >> 16), f[h][3] = fp8x2_to_f16x2(wb[h] >> 16);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const uint4 v = t.x[xd][j][0];
                    const uint32_t xv[4] = {v.x, v.y, v.z, v.w};
                    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        mma_f16(part, f[h][0], f[h][1], f[h][2], f[h][3], fp8x2_to_f16x2(xv[h]), fp8x2_to_f16x2(xv[h] >> 16));
                    const int r = 8 * j + 2 * (lane & 3);
                    const float2 s0 = fp8_scale_pair(s, sx[min(r, rows - 1) * ldx + blk]), s1 = fp8_scale_pair(s, sx[min(r + 1, rows - 1) * ldx + blk]);
                    acc[j][0] = fmaf(part[0] * s0.x, s0.y, acc[j][0]);
                    acc[j][1] = fmaf(part[1] * s1.x, s1.y, acc[j][1]);
                    acc[j][2] = fmaf(part[2] * s0.x, s0.y, acc[j][2]);
                    acc[j][3] = fmaf(part[3] * s1.x, s1.y, acc[j][3]);
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
                const float s = V == FEWV_W8A16 ? fp8_scale(sw[blk]) : 1.f;
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    uint32_t xv[2 * NS];
#pragma unroll
                    for (int q = 0; q < F::XV; ++q) {
                        const uint4 v = t.x[xd][j][q];
                        xv[4 * q] = v.x, xv[4 * q + 1] = v.y, xv[4 * q + 2] = v.z, xv[4 * q + 3] = v.w;
                    }
                    if (V == FEWV_W8A16) {
                        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int h = 0; h < NS; ++h)
                            mma_bf16(part, f[h][0], f[h][1], f[h][2], f[h][3], xv[2 * h], xv[2 * h + 1]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[j][c] = fmaf(part[c], s, acc[j][c]);
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
                    for (int c = 0; c < 4; ++c) sums[c] = fmaf(part[c], s, sums[c]);
                }
            }
            t.load_w(d, i + F::DW);
            t.load_x(xd, i + F::DX);
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
// The same where each pair of columns is one token's two parts: their sums, [warp][4 NT tokens][16 rows].
template <int NT>
__device__ __forceinline__ void few_stage_pairs(float* red, const float (&acc)[NT][4], int warp, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        float* p = red + ((warp * NT + j) * 4 + c) * 16;
        p[g] = acc[j][0] + acc[j][1];
        p[g + 8] = acc[j][2] + acc[j][3];
    }
}
// The sum over the warps of column col of COLS, in warp order.
template <int COLS, int WARPS = FEW_WARPS>
__device__ __forceinline__ float few_sum(const float* red, int col, int row) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += red[(w * COLS + col) * 16 + row];
    return s;
}

}  // namespace cm
