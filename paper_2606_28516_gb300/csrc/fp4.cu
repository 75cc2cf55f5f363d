// 4-bit blocks with power-of-two scales: quantisation and back. The product is in fp4_gemm.cu.
#include <cstdint>

#include "common.cuh"
#include "fp4.cuh"
#include "internal.h"

namespace cm {

namespace {

// Eight lanes take 128 columns of a row (a word of four scale bytes), 16 consecutive ones a lane, so that a block is two
// lanes'. A warp's four groups of lanes take rows 32 apart, whose words lie side by side, and a CTA's eight warps eight
// consecutive rows of each: 128 consecutive bytes of scales a CTA.
constexpr int Q4_THREADS = 256;
constexpr int Q4_CTAS = 32;  // an SM, at the most

template <typename T, bool VEC>
__device__ __forceinline__ void load16(const T* row, int64_t k, int64_t K, bool live, float (&v)[16]) {
    if (VEC) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = live && k + 8 * h < K;
            if (sizeof(T) == 2) {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (in) u = __ldcg(reinterpret_cast<const uint4*>(row + k) + h);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) v[8 * h + 2 * i] = bf16_lo(w[i]), v[8 * h + 2 * i + 1] = bf16_hi(w[i]);
            } else {
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
                if (in) {
                    a = __ldcg(reinterpret_cast<const float4*>(row + k) + 2 * h);
                    b = __ldcg(reinterpret_cast<const float4*>(row + k) + 2 * h + 1);
                }
                float* o = v + 8 * h;
                o[0] = a.x, o[1] = a.y, o[2] = a.z, o[3] = a.w, o[4] = b.x, o[5] = b.y, o[6] = b.z, o[7] = b.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            v[i] = 0.f;
            if (live && k + i < K)
                v[i] = sizeof(T) == 2 ? bf16_to_f32(__ldg(reinterpret_cast<const uint16_t*>(row) + k + i))
                                      : __ldg(reinterpret_cast<const float*>(row) + k + i);
        }
    }
}

template <typename T, bool VEC, bool GATHER>
__global__ void __launch_bounds__(Q4_THREADS) fp4_quantize_kernel(const Quant4Args a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l8 = lane & 7;
    const int64_t groups = (a.rows + 127) / 128 * 4;  // of 8 rows and those 32, 64 and 96 after them
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    for (int64_t i = blockIdx.x; i < groups * a.tiles; i += gridDim.x) {
        const int64_t group = i / a.tiles;
        const int tile = (int)(i - group * a.tiles);
        const int64_t row = (group >> 2) * 128 + (lane >> 3) * 32 + (group & 3) * 8 + warp;
        const bool live = row < a.rows;
        int64_t src = row;
        bool inside = true;
        if (GATHER && live) {
            src = __ldcg(a.gather + row);
            inside = (uint64_t)src < (uint64_t)a.src_rows;
        }
        const int64_t k = (int64_t)tile * 128 + l8 * 16;
        float v[16];
        load16<T, VEC>(static_cast<const T*>(a.x) + src * a.ld, k, a.K, live && inside, v);
        float m = 0.f;
#pragma unroll
        for (int c = 0; c < 16; c += 2) m = max_abs3(m, v[c], v[c + 1]);
        m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        const uint32_t s = inside ? fp4_scale_byte(abs_bits(m)) : 255u;
        const float inv = fp8_inverse_scale(s);
        const uint32_t lo = fp4_pack8_scaled(v, make_float2(inv, inv)), hi = fp4_pack8_scaled(v + 8, make_float2(inv, inv));
        uint32_t w = s << (8 * (l8 >> 1));  // the word of four blocks
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
        if (live) {
            if ((int64_t)tile * 64 + l8 * 8 < a.ldq)
                *reinterpret_cast<uint2*>(a.q + row * a.ldq + (int64_t)tile * 64 + l8 * 8) = make_uint2(lo, hi);
            if (l8 == 0) *reinterpret_cast<uint32_t*>(a.scale + fp4_scale_word(row, tile, a.tiles)) = w;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
    fp4_dequantize_kernel(const uint8_t* q, const uint8_t* scale, int64_t rows, int64_t K, int64_t ldq, int tiles, T* out, int64_t ld) {
    pdl_wait();
    const int64_t n = rows * K;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / K, k = i - r * K;
        const float v = fp4_value(q[r * ldq + k / 2] >> (k & 1) * 4) * fp8_scale(scale[fp4_scale_word(r, k / 128, tiles) + k / 32 % 4]);
        if (sizeof(T) == 2)
            reinterpret_cast<uint16_t*>(out)[r * ld + k] = f32_to_bf16(v);
        else
            reinterpret_cast<float*>(out)[r * ld + k] = v;
    }
}

template <typename K, typename... A>
cudaError_t launch(K kernel, int64_t grid, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, bool VEC>
cudaError_t launch_rows(const Quant4Args& a, int64_t grid, cudaStream_t s) {
    return a.gather ? launch(fp4_quantize_kernel<T, VEC, true>, grid, s, a) : launch(fp4_quantize_kernel<T, VEC, false>, grid, s, a);
}

}  // namespace

cudaError_t launch_fp4_quantize(const Quant4Args& a, int dtype, int num_sms, cudaStream_t s) {
    const bool bf16 = dtype == CLEARMOE_BF16;
    const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.K % 8 == 0 && (a.ld * (bf16 ? 2 : 4)) % 16 == 0;
    const int64_t one = (a.rows + 127) / 128 * 4 * a.tiles, most = (int64_t)num_sms * Q4_CTAS;
    const int64_t grid = one < most ? one : most;
    if (bf16) return vec ? launch_rows<uint16_t, true>(a, grid, s) : launch_rows<uint16_t, false>(a, grid, s);
    return vec ? launch_rows<float, true>(a, grid, s) : launch_rows<float, false>(a, grid, s);
}

int check_fp4(const clearmoe_fp4* m) {
    if (!m || !m->q || !m->scale || m->rows < 1 || m->cols < 1) return CLEARMOE_EINVAL;
    if (m->rows > (int64_t)1 << 30 || m->cols > (int64_t)1 << 24) return CLEARMOE_EINVAL;
    return ((reinterpret_cast<uintptr_t>(m->q) | reinterpret_cast<uintptr_t>(m->scale)) & 31) == 0 ? CLEARMOE_OK : CLEARMOE_EINVAL;
}

}  // namespace cm

namespace {

int cuda_code(cudaError_t e) {
    if (e == cudaSuccess) return CLEARMOE_OK;
    (void)cudaGetLastError();
    return CLEARMOE_ECUDA;
}

int check_pair(const void* x, int32_t dtype, int64_t ld, const clearmoe_fp4* m) {
    const int rc = cm::check_fp4(m);
    if (rc) return rc;
    if (!x || (dtype != CLEARMOE_F32 && dtype != CLEARMOE_BF16) || ld < m->cols || ld > (int64_t)1 << 30) return CLEARMOE_EINVAL;
    return (reinterpret_cast<uintptr_t>(x) & (dtype == CLEARMOE_BF16 ? 1 : 3)) == 0 ? CLEARMOE_OK : CLEARMOE_EINVAL;
}

}  // namespace

extern "C" {

int clearmoe_fp4_quantize(const void* x, int64_t x_rows, int32_t dtype, int64_t ld, const int32_t* gather,
                          const clearmoe_fp4* out, void* stream) {
    const int rc = check_pair(x, dtype, ld, out);
    if (rc) return rc;
    if (x_rows < 1 || (!gather && x_rows < out->rows) || (reinterpret_cast<uintptr_t>(gather) & 3)) return CLEARMOE_EINVAL;
    const int sms = cm::current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    cm::Quant4Args a = {};
    a.x = x;
    a.ld = ld;
    a.rows = out->rows;
    a.K = out->cols;
    a.src_rows = x_rows;
    a.gather = gather;
    a.q = static_cast<uint8_t*>(out->q);
    a.scale = out->scale;
    a.ldq = cm::fp4_ldq(out->cols);
    a.tiles = (int)cm::fp4_tiles(out->cols);
    return cuda_code(cm::launch_fp4_quantize(a, dtype, sms, static_cast<cudaStream_t>(stream)));
}

int clearmoe_fp4_dequantize(const clearmoe_fp4* in, void* out, int32_t dtype, int64_t ld, void* stream) {
    const int rc = check_pair(out, dtype, ld, in);
    if (rc) return rc;
    const int sms = cm::current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    const int64_t want = (in->rows * in->cols + 255) / 256, grid = want < (int64_t)sms * 8 ? want : (int64_t)sms * 8;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint8_t *q = static_cast<const uint8_t*>(in->q), *scale = in->scale;
    const int64_t ldq = cm::fp4_ldq(in->cols);
    const int tiles = (int)cm::fp4_tiles(in->cols);
    if (dtype == CLEARMOE_BF16)
        return cuda_code(cm::launch(cm::fp4_dequantize_kernel<uint16_t>, grid, s, q, scale, in->rows, in->cols, ldq, tiles,
                                    static_cast<uint16_t*>(out), ld));
    return cuda_code(cm::launch(cm::fp4_dequantize_kernel<float>, grid, s, q, scale, in->rows, in->cols, ldq, tiles,
                                static_cast<float*>(out), ld));
}

}  // extern "C"
