// 4-bit blocks: value = e2m1(q) 2^(s - 127), one scale byte s per 32 columns of a row, in tiles of 128 rows x 128
// columns. Device helpers shared by the quantiser, the GEMMs' epilogue, the few-row kernel and the norm, and the
// launchers.
#pragma once

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace cm {

// Bytes from one row of q to the next: whole K steps of the MMAs (64 columns).
__host__ __device__ __forceinline__ int64_t fp4_ldq(int64_t cols) { return (cols + 63) / 64 * 32; }
// Tiles of scales side by side; a tile has 512 bytes.
__host__ __device__ __forceinline__ int64_t fp4_tiles(int64_t cols) { return (cols + 127) / 128; }
// The four scale bytes of row `row` in tile column `tile` (of `tiles`), from the start of the scales.
__host__ __device__ __forceinline__ int64_t fp4_scale_word(int64_t row, int64_t tile, int64_t tiles) {
    return ((row >> 7) * tiles + tile) * 512 + (row & 31) * 16 + (row >> 5 & 3) * 4;
}

// Scale byte of a block whose largest |value| has the fp32 bits `amax` (largest as an unsigned integer, so that
// NaN > inf > every finite value): the least s with amax <= 6 2^(s - 127). 6 = 1.5 2^2, so s is amax's biased exponent
// less 2, one more when its significand is above 1.5; held at 0 below, 255 (the scale format's NaN) for a block with an
// infinity or a NaN. At most 253 otherwise; its inverse is fp8_inverse_scale's.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax) {
    if (amax >= 0x7F800000u) return 255u;
    const int s = (int)(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x400000u ? 1 : 0);
    return s < 0 ? 0u : (uint32_t)s;
}
// Eight values to e2m1, to nearest even, the first in the lowest four bits. (NaN has no code.)
__device__ __forceinline__ uint32_t fp4_pack8(float a, float b, float c, float d, float e, float f, float g, float h) {
    uint32_t v;
    asm("{\n\t.reg .b8 p, q, r, s;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 p, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 q, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 r, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 s, %8, %7;\n\t"
        "mov.b32 %0, {p, q, r, s};\n\t}"
        : "=r"(v)
        : "f"(a), "f"(b), "f"(c), "f"(d), "f"(e), "f"(f), "f"(g), "f"(h));
    return v;
}
// Eight values times k (a power of two), to e2m1.
__device__ __forceinline__ uint32_t fp4_pack8_scaled(const float* v, float2 k) {
    const float2 a = __fmul2_rn(make_float2(v[0], v[1]), k), b = __fmul2_rn(make_float2(v[2], v[3]), k);
    const float2 c = __fmul2_rn(make_float2(v[4], v[5]), k), d = __fmul2_rn(make_float2(v[6], v[7]), k);
    return fp4_pack8(a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y);
}
// The values of eight codes, the first in the lowest four bits, exactly (by way of fp16).
__device__ __forceinline__ void fp4_unpack8(uint32_t w, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 p, q, r, s;\n\t"
        "mov.b32 {p, q, r, s}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, p;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, q;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, r;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, s;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}"
            : "=f"(v[2 * i]), "=f"(v[2 * i + 1])
            : "r"(h[i]));
}

// ---- launchers ----
struct Quant4Args {
    const void* x;
    int64_t ld;  // elements
    int64_t rows, K;
    int64_t src_rows;       // x's rows: a row gathered from outside them is NaN
    const int32_t* gather;  // source row of row i (nullable)
    uint8_t* q;
    uint8_t* scale;
    int64_t ldq;
    int tiles;  // scale tiles side by side
};
cudaError_t launch_fp4_quantize(const Quant4Args& a, int dtype, int num_sms, cudaStream_t s);

constexpr int FP4_OUT_FP4 = 3;  // of out_kind, beside FP8_OUT_F32 and FP8_OUT_BF16
constexpr int FP4_OUT_BF16_BULK = 4;  // a kernel's: bf16 by bulk copies
// A product of NE matrices of weights: one, or CM_MAX_E of a grouped product (a launch copies its arguments: 0.2 us of host
// time for those of sixteen).
template <int NE>
struct Fp4GemmArgs {
    static constexpr bool GROUPED = NE > 1;
    CUtensorMap tmA, tmSA;          // bytes of q as half as many 16-bit elements, boxes of 128 bytes; scale tiles, boxes of two side by side
    CUtensorMap tmB[NE], tmSB[NE];  // the same of W
    CUtensorMap tmH[NE];            // W's q in boxes of half as many rows, for halves of tiles
    CUtensorMap tmOut;              // FP4_OUT_BF16_BULK
    int64_t M;
    int N;
    int nkb;       // stages of 256 columns
    int ksteps;    // MMAs of 64 columns
    int box_rows;  // rows of tmA's boxes
    int E;         // groups
    int whole, rest;  // of a product of one matrix on pairs: rounds of tiles that every pair has one of, tiles after them
    const int32_t* offsets;  // [E + 1]; a grouped product's
    const int32_t* rows;     // output row of row i (nullable); a grouped product's
    const void* bias;        // [N], fp32 or bf16 (nullable)
    int bias_bf16;
    int act;       // clearmoe_act
    int out_kind;  // FP8_OUT_F32, FP8_OUT_BF16 or FP4_OUT_FP4
    int tma_out;   // bf16 outputs on pairs leave by tmOut
    void* out;
    int64_t ldo;         // elements; 4-bit outputs: bytes between rows of q
    uint8_t* out_scale;  // FP4_OUT_FP4
    int64_t ldos;        // scale tiles side by side
    int32_t* status;
    int64_t wait_limit_ns;
};
template <int NE>
cudaError_t launch_fp4_gemm2(Fp4GemmArgs<NE>& a, int bn, int num_sms, cudaStream_t s);
// A product of at most FP4_FEW_MAX rows in one group: tmA in boxes of fp4_few_rows(M) rows, tmB of 128.
constexpr int FP4_FEW_MAX = 128;
int fp4_few_rows(int64_t M);
bool fp4_few_pays(int64_t M, int N, int nkb, int num_sms);
cudaError_t launch_fp4_few(const Fp4GemmArgs<1>& a, int num_sms, cudaStream_t s);
int check_fp4(const clearmoe_fp4* m);
// Scale tiles [tile_rows x tile_cols] of 512 bytes as a tensor map, boxes of two tiles side by side x box_rows.
int encode_tmap_fp4_scales(CUtensorMap* map, const void* base, int64_t tile_rows, int64_t tile_cols, int box_rows);
// Bytes [rows x bytes], rows `pitch` apart (a multiple of 16), as a tensor map for stores, boxes of 64 bytes x 32 rows with
// 64-byte swizzle.
int encode_tmap_out_bytes(CUtensorMap* map, const void* base, int64_t rows, int64_t bytes, int64_t pitch);

}  // namespace cm
