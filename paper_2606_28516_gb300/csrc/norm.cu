// A residual's addition and the root-mean-square norm of the sum, s = x + r, y = s w / sqrt(mean(s^2) + eps), with s stored
// and y in fp32 or bf16, 8-bit blocks or 4-bit blocks: one pass, a row in registers between its statistics and its output.
// Bound by HBM: x and r are read, s and y written, once each.
//
// A warp takes 512 columns of a row at a time, 16 a lane; a row is 1 to 16 warps' and each has up to four such pieces.
// Aligned rows: a lane has 16 consecutive columns, so that eight lanes have a block of 128 and two a block of 32, and
// scales take three shuffles or one. Other rows: a lane has columns 32 apart, so that loads and stores are of consecutive
// elements, and a block's scale takes five shuffles.
#include <cmath>
#include <cstdint>

#include "common.cuh"
#include "fp4.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace cm {

namespace {

enum NormOut { NORM_OUT_DTYPE = 0, NORM_OUT_FP8 = 1, NORM_OUT_FP4 = 2 };

struct NormArgs {
    const void* x;
    const void* r;  // nullable
    void* sum;      // nullable
    const void* w;  // nullable
    int64_t ldx, ldr, lds, rows;
    int cols;
    int w_bf16;
    float eps;
    void* out;      // or q
    int out_bf16;
    int64_t ldo;    // elements, or bytes between rows of q
    uint8_t* scale;
    int64_t ld_scale;  // 8 bits: bytes between rows of scales; 4 bits: scale tiles side by side
    int out_vec;       // aligned rows of out; of the weights
    int w_vec;
};

template <typename T>
__device__ __forceinline__ float load1(const void* p, int64_t at) {
    return sizeof(T) == 2 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(p) + at)) : __ldcg(static_cast<const float*>(p) + at);
}
__device__ __forceinline__ void unpack8(const uint4& u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
}
// Eight elements from an aligned place on.
template <typename T>
__device__ __forceinline__ void load8(const void* p, int64_t at, float* v) {
    if (sizeof(T) == 2) {
        unpack8(__ldcg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at)), v);
    } else {
        const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        const float4 a = __ldcg(f), b = __ldcg(f + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}
__device__ __forceinline__ uint4 pack8(const float* v) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(void* p, bool bf16, int64_t at, const float* v) {
    if (bf16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = pack8(v);
    } else {
        float4* f = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
        f[0] = make_float4(v[0], v[1], v[2], v[3]);
        f[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}
__device__ __forceinline__ void store1(void* p, bool bf16, int64_t at, float v) {
    if (bf16)
        static_cast<uint16_t*>(p)[at] = f32_to_bf16(v);
    else
        static_cast<float*>(p)[at] = v;
}
__device__ __forceinline__ float weight1(const NormArgs& a, int k) {
    return a.w_bf16 ? bf16_to_f32(__ldg(static_cast<const uint16_t*>(a.w) + k)) : __ldg(static_cast<const float*>(a.w) + k);
}

// CH pieces of 512 columns a warp; wpr warps a row (blockDim / 32 a multiple of it).
template <typename T, int OUT, bool VEC, int CH>
__global__ void __launch_bounds__(512) rms_norm_kernel(const NormArgs a, const int wpr) {
    __shared__ float s_part[16];
    constexpr bool BF16 = sizeof(T) == 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % wpr;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / 32 / wpr) + warp / wpr;
    const bool live = row < a.rows;
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    // column of element i of piece c
    auto column = [&](int c, int i) { return (c * wpr + part) * 512 + (VEC ? lane * 16 + i : i * 32 + lane); };
    float v[CH][16];
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if constexpr (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = column(c, 8 * h);
                float* o = v[c] + 8 * h;
                if (live && k < a.cols) {
                    load8<T>(a.x, row * a.ldx + k, o);
                    if (a.r) {
                        float r[8];
                        load8<T>(a.r, row * a.ldr + k, r);
#pragma unroll
                        for (int i = 0; i < 8; ++i) o[i] += r[i];
                    }
                    if constexpr (BF16) unpack8(pack8(o), o);  // the sum as it is stored
                    if (a.sum) store8(a.sum, BF16, row * a.lds + k, o);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = 0.f;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = column(c, i);
                float s = 0.f;
                if (live && k < a.cols) {
                    s = load1<T>(a.x, row * a.ldx + k);
                    if (a.r) s += load1<T>(a.r, row * a.ldr + k);
                    if constexpr (BF16) s = bf16_to_f32(f32_to_bf16(s));
                    if (a.sum) store1(a.sum, BF16, row * a.lds + k, s);
                }
                v[c][i] = s;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sq = fmaf(v[c][i], v[c][i], sq);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
    if (wpr > 1) {
        if (lane == 0) s_part[warp] = sq;
        __syncthreads();
        sq = 0.f;
        for (int i = warp - part; i < warp - part + wpr; ++i) sq += s_part[i];
    }
    const float rstd = 1.f / sqrtf(sq / (float)a.cols + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = v[c][i] * rstd;
        if (a.w) {
            if (VEC && a.w_vec) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = column(c, 8 * h);
                    if (k >= a.cols) continue;
                    float w[8];
                    if (a.w_bf16)
                        load8<uint16_t>(a.w, k, w);
                    else
                        load8<float>(a.w, k, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[8 * h + i] *= w[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = column(c, i);
                    if (k < a.cols) y[i] *= weight1(a, k);
                }
            }
        }
        // rows past the last and columns past cols: nothing, or zeros in a block's padding (0 times an infinite rstd: NaN)
        if (!(VEC && OUT == NORM_OUT_DTYPE)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (column(c, i) >= a.cols) y[i] = 0.f;
        }
        if constexpr (OUT == NORM_OUT_DTYPE) {
            if (!live) continue;
            if (VEC && a.out_vec) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = column(c, 8 * h);
                    if (k < a.cols) store8(a.out, a.out_bf16, row * a.ldo + k, y + 8 * h);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = column(c, i);
                    if (k < a.cols) store1(a.out, a.out_bf16, row * a.ldo + k, y[i]);
                }
            }
        } else if constexpr (VEC) {
            const int k = column(c, 0);  // of 16
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) m = max_abs3(m, y[i], y[i + 1]);
#pragma unroll
            for (int o = OUT == NORM_OUT_FP8 ? 4 : 1; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            const uint32_t s = OUT == NORM_OUT_FP8 ? fp8_scale_byte(abs_bits(m)) : fp4_scale_byte(abs_bits(m));
            const float inv = fp8_inverse_scale(s);
            if constexpr (OUT == NORM_OUT_FP8) {
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = fp8_pack4(y[4 * i] * inv, y[4 * i + 1] * inv, y[4 * i + 2] * inv, y[4 * i + 3] * inv);
                if (live && k < a.ldo) {
                    *reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.out) + row * a.ldo + k) = make_uint4(o[0], o[1], o[2], o[3]);
                    if ((lane & 7) == 0) a.scale[row * a.ld_scale + k / 128] = (uint8_t)s;
                }
            } else {
                const uint32_t lo = fp4_pack8_scaled(y, make_float2(inv, inv)), hi = fp4_pack8_scaled(y + 8, make_float2(inv, inv));
                uint32_t w = s << (8 * (lane >> 1 & 3));
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
                if (live && k / 2 < a.ldo) {
                    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.out) + row * a.ldo + k / 2) = make_uint2(lo, hi);
                    if ((lane & 7) == 0) *reinterpret_cast<uint32_t*>(a.scale + fp4_scale_word(row, k >> 7, a.ld_scale)) = w;
                }
            }
        } else {
#pragma unroll
            for (int b = 0; b < 4; ++b) {  // 128 columns: four elements a lane
                const int k = column(c, 4 * b);
                uint32_t m[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) m[i] = abs_bits(y[4 * b + i]);
                if constexpr (OUT == NORM_OUT_FP8) {
                    const uint32_t s = fp8_scale_byte(__reduce_max_sync(0xFFFFFFFFu, max(max(m[0], m[1]), max(m[2], m[3]))));
                    const float inv = fp8_inverse_scale(s);
                    if (live && k - lane < a.cols) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            static_cast<uint8_t*>(a.out)[row * a.ldo + k + 32 * i] = (uint8_t)fp8_pack2(y[4 * b + i] * inv, 0.f);
                        if (lane == 0) a.scale[row * a.ld_scale + (k - lane) / 128] = (uint8_t)s;
                    }
                } else {
                    uint32_t word = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t s = fp4_scale_byte(__reduce_max_sync(0xFFFFFFFFu, m[i]));
                        word |= s << (8 * i);
                        const float f = y[4 * b + i] * fp8_inverse_scale(s), g = __shfl_down_sync(0xFFFFFFFFu, f, 1);
                        const int at = (k + 32 * i) / 2;
                        if (live && (lane & 1) == 0 && at < a.ldo)
                            static_cast<uint8_t*>(a.out)[row * a.ldo + at] = (uint8_t)fp4_pack8(f, g, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f);
                    }
                    if (live && lane == 0 && k < a.cols) *reinterpret_cast<uint32_t*>(a.scale + fp4_scale_word(row, k >> 7, a.ld_scale)) = word;
                }
            }
        }
    }
}

template <typename T, int OUT, bool VEC>
cudaError_t launch_ch(const NormArgs& a, cudaStream_t s) {
    int wpr = 1, ch = 1;
    while (wpr < 16 && wpr * 512 < a.cols) wpr *= 2;
    while (wpr * ch * 512 < a.cols) ch *= 2;
    const int warps = wpr < 8 ? 8 : wpr, rows = warps / wpr;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.rows + rows - 1) / rows));
    cfg.blockDim = dim3(32 * warps);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return ch == 1   ? cudaLaunchKernelEx(&cfg, rms_norm_kernel<T, OUT, VEC, 1>, a, wpr)
           : ch == 2 ? cudaLaunchKernelEx(&cfg, rms_norm_kernel<T, OUT, VEC, 2>, a, wpr)
                     : cudaLaunchKernelEx(&cfg, rms_norm_kernel<T, OUT, VEC, 4>, a, wpr);
}

bool rows_vec(const void* p, int64_t ld, int esz) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * esz % 16 == 0); }
bool off_type(const void* p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) & (dtype == CLEARMOE_BF16 ? 1 : 3); }
bool known(int32_t dtype) { return dtype == CLEARMOE_F32 || dtype == CLEARMOE_BF16; }

int check(const clearmoe_norm* n, NormArgs& a) {
    if (!n || !n->x || !known(n->dtype) || n->rows < 1 || n->rows > (int64_t)1 << 30 || n->cols < 1) return CLEARMOE_EINVAL;
    if (n->cols > CLEARMOE_NORM_MAX) return CLEARMOE_EUNSUPPORTED;
    const int64_t most = (int64_t)1 << 30;
    if (off_type(n->x, n->dtype) || n->ldx < n->cols || n->ldx > most) return CLEARMOE_EINVAL;
    if (n->residual && (off_type(n->residual, n->dtype) || n->ldr < n->cols || n->ldr > most)) return CLEARMOE_EINVAL;
    if (n->sum && (off_type(n->sum, n->dtype) || n->lds < n->cols || n->lds > most)) return CLEARMOE_EINVAL;
    if (n->sum && ((n->sum == n->x && n->lds != n->ldx) || (n->sum == n->residual && n->lds != n->ldr))) return CLEARMOE_EINVAL;
    if (n->weight && (!known(n->weight_dtype) || off_type(n->weight, n->weight_dtype))) return CLEARMOE_EINVAL;
    if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return CLEARMOE_EINVAL;
    a = {};
    a.x = n->x;
    a.r = n->residual;
    a.sum = n->sum;
    a.w = n->weight;
    a.ldx = n->ldx;
    a.ldr = n->ldr;
    a.lds = n->lds;
    a.rows = n->rows;
    a.cols = (int)n->cols;
    a.w_bf16 = n->weight_dtype == CLEARMOE_BF16;
    a.w_vec = rows_vec(n->weight, 0, 1);
    a.eps = n->eps;
    return CLEARMOE_OK;
}

template <int OUT>
int run(const clearmoe_norm* n, const NormArgs& a, void* stream) {
    const int esz = n->dtype == CLEARMOE_BF16 ? 2 : 4;
    const bool vec = n->cols % 8 == 0 && rows_vec(n->x, n->ldx, esz) && rows_vec(n->residual, n->ldr, esz) && rows_vec(n->sum, n->lds, esz);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = esz == 2 ? (vec ? launch_ch<uint16_t, OUT, true>(a, s) : launch_ch<uint16_t, OUT, false>(a, s))
                                   : (vec ? launch_ch<float, OUT, true>(a, s) : launch_ch<float, OUT, false>(a, s));
    if (e == cudaSuccess) return CLEARMOE_OK;
    (void)cudaGetLastError();
    return CLEARMOE_ECUDA;
}

}  // namespace

}  // namespace cm

extern "C" {

int clearmoe_rms_norm(const clearmoe_norm* n, void* out, int32_t out_dtype, int64_t ldo, void* stream) {
    cm::NormArgs a;
    const int rc = cm::check(n, a);
    if (rc) return rc;
    if (!out || !cm::known(out_dtype) || cm::off_type(out, out_dtype) || ldo < n->cols || ldo > (int64_t)1 << 30) return CLEARMOE_EINVAL;
    if (out == n->sum) return CLEARMOE_EINVAL;
    if ((out == n->x && (out_dtype != n->dtype || ldo != n->ldx)) || (out == n->residual && (out_dtype != n->dtype || ldo != n->ldr)))
        return CLEARMOE_EINVAL;
    a.out = out;
    a.out_bf16 = out_dtype == CLEARMOE_BF16;
    a.ldo = ldo;
    a.out_vec = cm::rows_vec(out, ldo, a.out_bf16 ? 2 : 4);
    return cm::run<cm::NORM_OUT_DTYPE>(n, a, stream);
}

int clearmoe_rms_norm_fp8(const clearmoe_norm* n, const clearmoe_fp8* out, void* stream) {
    cm::NormArgs a;
    int rc = cm::check(n, a);
    if (rc || (rc = cm::check_fp8(out))) return rc;
    if (out->rows != n->rows || out->cols != n->cols) return CLEARMOE_EINVAL;
    a.out = out->q;
    a.ldo = cm::fp8_ldq(out->cols);
    a.scale = out->scale;
    a.ld_scale = cm::fp8_lds(out->cols);
    return cm::run<cm::NORM_OUT_FP8>(n, a, stream);
}

int clearmoe_rms_norm_fp4(const clearmoe_norm* n, const clearmoe_fp4* out, void* stream) {
    cm::NormArgs a;
    int rc = cm::check(n, a);
    if (rc || (rc = cm::check_fp4(out))) return rc;
    if (out->rows != n->rows || out->cols != n->cols) return CLEARMOE_EINVAL;
    a.out = out->q;
    a.ldo = cm::fp4_ldq(out->cols);
    a.scale = out->scale;
    a.ld_scale = cm::fp4_tiles(out->cols);
    return cm::run<cm::NORM_OUT_FP4>(n, a, stream);
}

}  // extern "C"
