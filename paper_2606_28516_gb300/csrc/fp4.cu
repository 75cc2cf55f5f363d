// 4-bit blocks with power-of-two scales: quantisation and back. The product is in fp4_gemm.cu.
#include <cstdint>

#include "common.cuh"
#include "fp4.cuh"
#include "internal.h"
#include "lane16.cuh"

namespace cm {

namespace {

// Eight lanes take 128 columns of a row (a word of four scale bytes), 16 a lane. A warp's four groups of lanes take rows 32
// apart, whose words lie side by side, and a CTA's eight warps eight consecutive rows of each: 128 consecutive bytes of
// scales a CTA. Bound by HBM: each element is read once and written once as half a byte. Aligned rows come through shared
// memory, each lane's next elements on their way while it converts these: what is on its way to registers lies in L1
// meanwhile, and beside a product, whose shared memory leaves L1 28 KB, that held the loads back (16,384 x 4,096 bf16 and
// its product: 123 us where the two take 105). Other rows: a warp reads 32 consecutive elements at a time, and turns them to
// the same order in shared memory.
constexpr int Q4_THREADS = 256;
constexpr int Q4_CTAS = 8;  // an SM, at the most

// A lane's 16 values (as Lane16's of P columns, eight lanes a row) from column k of row `row` on to codes and scales. live:
// there is such a row; inside: it is one of x's.
template <int P>
__device__ __forceinline__ void quantize16(const Quant4Args& a, float2 (&v)[8], int64_t row, int tile, int l8, bool live, bool inside) {
    uint8_t* q = a.q + row * a.ldq + (int64_t)tile * 64 + l8 * (P / 2);
    const int64_t bytes = a.ldq - (int64_t)tile * 64 - l8 * (P / 2);  // to the row's end
    uint32_t word = 0;
#pragma unroll
    for (int h = 0; h < 16 / P; ++h) {
        float2* f = v + P / 2 * h;
        float m = max_abs3(max_abs(f[0].x, f[0].y), f[1].x, f[1].y);
        if constexpr (P == 8) m = max_abs3(max_abs3(m, f[2].x, f[2].y), f[3].x, f[3].y);
#pragma unroll
        for (int o = 16 / P; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const uint32_t s = inside ? fp4_scale_byte(abs_bits(m)) : 255u;
        const float inv = fp8_inverse_scale(s);
#pragma unroll
        for (int i = 0; i < P / 2; ++i) f[i] = __fmul2_rn(f[i], make_float2(inv, inv));
        word |= s << (P == 8 ? 16 * h + 8 * (l8 >> 2) : 8 * h);
        if (live && 4 * P * h < bytes) {
            if constexpr (P == 8)
                *reinterpret_cast<uint32_t*>(q + 4 * P * h) = fp4_pack8(f[0].x, f[0].y, f[1].x, f[1].y, f[2].x, f[2].y, f[3].x, f[3].y);
            else
                *reinterpret_cast<uint16_t*>(q + 4 * P * h) = (uint16_t)fp4_pack8(f[0].x, f[0].y, f[1].x, f[1].y, 0.f, 0.f, 0.f, 0.f);
        }
    }
    if constexpr (P == 8) word |= __shfl_xor_sync(0xFFFFFFFFu, word, 4);
    if (live && l8 == 0) *reinterpret_cast<uint32_t*>(a.scale + fp4_scale_word(row, tile, a.tiles)) = word;
}

// U: tiles of 128 columns side by side that a lane has at a time, so that more is on its way: 16,384 x 4,096 bf16 26.5 us with
// two, 32.7 with one, 29.9 with four; 9,973 x 4,096 gathered 21.1, 25.6, 21.8. Fewer than four items a CTA are better off
// with one: 197 x 384 1.5 us, two 1.6, four 2.1.
template <typename T, bool VEC, bool GATHER, int U>
__global__ void __launch_bounds__(Q4_THREADS) fp4_quantize_kernel(const Quant4Args a) {
    using Lane = Lane16<T, VEC, 8>;
    __shared__ __align__(16) unsigned char s_mem[VEC ? U * Lane::N * 16 * Q4_THREADS : Q4_THREADS / 32 * 4 * 132 * 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l8 = lane & 7;
    const uint32_t own = smem_u32(s_mem) + 16 * threadIdx.x, pitch = 16 * Q4_THREADS;
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    // items: groups of 8 rows and those 32, 64 and 96 after them, U tiles of each
    const int cols = (a.tiles + U - 1) / U;
    const int64_t groups = (a.rows + 127) / 128 * 4, step_group = gridDim.x / cols;
    const int step_col = (int)(gridDim.x - step_group * cols);
    int64_t group = blockIdx.x / cols, row = 0, src = 0;
    int col = (int)(blockIdx.x - group * cols);
    bool live = false, inside = true;
    auto row_of = [&](int64_t g) { return (g >> 2) * 128 + (lane >> 3) * 32 + (g & 3) * 8 + warp; };
    int index = 0;  // of the next item's row, on its way a turn ahead
    auto ask_index = [&](int64_t g) {
        if (GATHER && row_of(g) < a.rows) index = __ldcg(a.gather + row_of(g));
    };
    auto place = [&]() {
        row = row_of(group);
        live = group < groups && row < a.rows;
        src = GATHER ? index : row;
        inside = !GATHER || (uint64_t)src < (uint64_t)a.src_rows;
        ask_index(group + step_group + (col + step_col >= cols ? 1 : 0));
    };
    // columns from the lane's first one of unit u to the end of its row; none for one that is not there
    auto left = [&](int u) { return live && inside ? (int)(a.K - ((int64_t)col * U + u) * 128 - l8 * Lane::P) : -(1 << 30); };
    auto ask = [&]() {
        if constexpr (VEC) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                Lane::ask(own + u * Lane::N * pitch, pitch, static_cast<const T*>(a.x) + src * a.ld + ((int64_t)col * U + u) * 128 + l8 * Lane::P, left(u));
            cp_async_commit();
        }
    };
    auto next = [&]() {
        group += step_group;
        col += step_col;
        if (col >= cols) col -= cols, ++group;
        place();
    };
    // Other rows: 32 consecutive elements of each of the warp's four rows at a time.
    T e[VEC ? 1 : 4][VEC ? 1 : 4];
    auto load = [&]() {
        if constexpr (!VEC) {
            const T* p = static_cast<const T*>(a.x) + src * a.ld + (int64_t)col * 128;
            const int n = live && inside ? (int)min((int64_t)128, a.K - (int64_t)col * 128) : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const T* pj = reinterpret_cast<const T*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(p), 8 * j)) + lane;
                const int nj = __shfl_sync(0xFFFFFFFFu, n, 8 * j);
#pragma unroll
                for (int c = 0; c < 4; ++c) e[j][c] = lane + 32 * c < nj ? __ldcg(pj + 32 * c) : T(0);
            }
        }
    };
    ask_index(group);
    place();
    ask();
    load();
    while (group < groups) {
        const int64_t r = row;
        const int t = col * U;
        const bool l = live, in = inside;
        if constexpr (VEC) {
            Lane x[U];
            cp_async_wait<0>();
#pragma unroll
            for (int u = 0; u < U; ++u) x[u].take(own + u * Lane::N * pitch, pitch, left(u));
            next();
            ask();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (t + u >= a.tiles) break;
                float2 v[8];
                x[u].values(v);
                quantize16<Lane::P>(a, v, r, t + u, l8, l, in);
            }
        } else {
            float* s = reinterpret_cast<float*>(s_mem) + warp * 4 * 132;  // [row of the warp's four][column]
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if constexpr (sizeof(T) == 2)
                        s[132 * j + 32 * c + lane] = bf16_to_f32(e[j][c]);
                    else
                        s[132 * j + 32 * c + lane] = e[j][c];
                }
            __syncwarp();
            float2 v[8];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const float4 f = *reinterpret_cast<const float4*>(s + 132 * (lane >> 3) + 64 * (h >> 1) + 8 * l8 + 4 * (h & 1));
                v[2 * h] = make_float2(f.x, f.y), v[2 * h + 1] = make_float2(f.z, f.w);
            }
            next();
            load();
            quantize16<8>(a, v, r, t, l8, l, in);
        }
    }
}

// Eight columns a thread (a quarter of a block: four bytes of codes, one scale), blocks of 2,048 columns, every gridDim.y-th
// row. vec: rows of out in whole 16-byte pieces.
template <typename T>
__global__ void __launch_bounds__(256)
    fp4_dequantize_kernel(const uint8_t* q, const uint8_t* scale, int64_t rows, int64_t K, int64_t ldq, int tiles, T* out, int64_t ld, int vec) {
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    const int64_t k = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (k >= K) return;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(q + r * ldq + k / 2);
        const float f = fp8_scale(scale[fp4_scale_word(r, k >> 7, tiles) + (k >> 5 & 3)]);
        float v[8];
        fp4_unpack8(w, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= f;
        T* o = out + r * ld + k;
        if (vec) {
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            } else {
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                *(reinterpret_cast<float4*>(o) + 1) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (k + i >= K) break;
                if constexpr (sizeof(T) == 2)
                    o[i] = f32_to_bf16(v[i]);
                else
                    o[i] = v[i];
            }
        }
    }
}

template <typename K, typename... A>
cudaError_t launch(K kernel, dim3 grid, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, bool VEC, int U>
cudaError_t launch_rows(const Quant4Args& a, int64_t most, cudaStream_t s) {
    const int64_t items = (a.rows + 127) / 128 * 4 * ((a.tiles + U - 1) / U), grid = items < most ? items : most;
    return a.gather ? launch(fp4_quantize_kernel<T, VEC, true, U>, dim3((unsigned)grid), s, a) : launch(fp4_quantize_kernel<T, VEC, false, U>, dim3((unsigned)grid), s, a);
}

}  // namespace

cudaError_t launch_fp4_quantize(const Quant4Args& a, int dtype, int num_sms, cudaStream_t s) {
    const bool bf16 = dtype == CLEARMOE_BF16;
    const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.K % 8 == 0 && (a.ld * (bf16 ? 2 : 4)) % 16 == 0;
    const int64_t most = (int64_t)num_sms * Q4_CTAS;
    const bool two = (a.rows + 127) / 128 * 4 * a.tiles >= 4 * most;
    if (!vec) return bf16 ? launch_rows<uint16_t, false, 1>(a, most, s) : launch_rows<float, false, 1>(a, most, s);
    if (bf16) return two ? launch_rows<uint16_t, true, 2>(a, most, s) : launch_rows<uint16_t, true, 1>(a, most, s);
    return two ? launch_rows<float, true, 2>(a, most, s) : launch_rows<float, true, 1>(a, most, s);
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
    const int64_t wide = (in->cols + 2047) / 2048, most = (int64_t)sms * 32 / wide + 1;
    const dim3 grid((unsigned)wide, (unsigned)(in->rows < most ? in->rows : most));
    const int vec = in->cols % 8 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0 && ld * (dtype == CLEARMOE_BF16 ? 2 : 4) % 16 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint8_t *q = static_cast<const uint8_t*>(in->q), *scale = in->scale;
    const int64_t ldq = cm::fp4_ldq(in->cols);
    const int tiles = (int)cm::fp4_tiles(in->cols);
    if (dtype == CLEARMOE_BF16)
        return cuda_code(cm::launch(cm::fp4_dequantize_kernel<uint16_t>, grid, s, q, scale, in->rows, in->cols, ldq, tiles,
                                    static_cast<uint16_t*>(out), ld, vec));
    return cuda_code(cm::launch(cm::fp4_dequantize_kernel<float>, grid, s, q, scale, in->rows, in->cols, ldq, tiles,
                                static_cast<float*>(out), ld, vec));
}

}  // extern "C"
