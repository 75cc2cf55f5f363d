// A residual's addition and the root-mean-square norm of the sum, s = x + r, y = s w / sqrt(mean(s^2) + eps), with s stored
// and y in fp32 or bf16, 8-bit blocks or 4-bit blocks: one pass, a row in registers between its statistics and its output.
// Bound by HBM: x and r are read, s and y written, once each.
//
// A warp takes 512 columns of a row at a time, 16 a lane; a row is 1 to 16 warps' and each has up to four such pieces.
// Aligned rows: a lane has pieces of 16 bytes, so that 16 (fp32: 32) lanes have a block of 128 columns and four (eight) one
// of 32. Other rows: a lane has columns 32 apart, so that loads and stores are of consecutive elements, and values are
// turned to such pieces in shared memory. CTAs stay and take every gridDim-th group of rows. Aligned rows of one piece a
// warp come through shared memory, each lane's own elements a row ahead, so that loads on their way hold no registers.
#include <cmath>
#include <cstdint>

#include "common.cuh"
#include "fp4.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "lane16.cuh"

namespace cm {

namespace {

enum NormOut { NORM_OUT_F32 = 0, NORM_OUT_BF16 = 1, NORM_OUT_FP8 = 2, NORM_OUT_FP4 = 3 };

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
    int64_t ldo;    // elements, or bytes between rows of q
    uint8_t* scale;
    int64_t ld_scale;  // 8 bits: bytes between rows of scales; 4 bits: scale tiles side by side
    int out_vec;       // aligned rows of out; of the weights
    int w_vec;
};

__device__ __forceinline__ uint4 pack8(const float2* v) {
    return make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
}
// The weights of a lane's 16 columns (as Lane16's) from k on.
template <int P>
__device__ __forceinline__ void weights(const NormArgs& a, int k, float2 (&w)[8]) {
    float f[16];
#pragma unroll
    for (int h = 0; h < 16 / P; ++h) {
        const int n = k + 32 * P * h;
        float* v = f + P * h;
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = 0.f;
        if (!a.w || n >= a.cols) continue;
        if (P > 1 && a.w_vec) {  // whole pieces
            if (!a.w_bf16) {
#pragma unroll
                for (int i = 0; i < P; i += 4) {
                    const float4 q = __ldcg(reinterpret_cast<const float4*>(static_cast<const float*>(a.w) + n + i));
                    v[i] = q.x, v[i + 1] = q.y, v[i + 2] = q.z, v[i + 3] = q.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < P; i += 4) {
                    const uint2 q = __ldcg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.w) + n + i));
                    v[i] = bf16_lo(q.x), v[i + 1] = bf16_hi(q.x), v[i + 2] = bf16_lo(q.y), v[i + 3] = bf16_hi(q.y);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                v[i] = a.w_bf16 ? bf16_to_f32(__ldcg(static_cast<const uint16_t*>(a.w) + n + i)) : __ldcg(static_cast<const float*>(a.w) + n + i);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = make_float2(f[2 * i], f[2 * i + 1]);
}

constexpr int NO_ROW = -(1 << 30);  // `left` where there is no row

// The warps of row `row` of a CTA's (at most four where a row has several warps) meet. 0 is __syncthreads'.
__device__ __forceinline__ void row_sync(int row, int threads) {
    if (row == 0) asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory");
    if (row == 1) asm volatile("bar.sync 2, %0;" ::"r"(threads) : "memory");
    if (row == 2) asm volatile("bar.sync 3, %0;" ::"r"(threads) : "memory");
    if (row == 3) asm volatile("bar.sync 4, %0;" ::"r"(threads) : "memory");
}
// Squares are of values times 2^-8, so that the sum of 2^15 of them is in fp32's range where their mean is; each is off by up to
// 2^-150 at the low end, 2^-134 in the mean. That is nothing beside an eps from here on; with a smaller one a row whose sum of
// squares is past the range, or whose mean and eps are below NORM_LOW, has its statistic taken again (far_rstd), in kernels
// of their own: with that branch in all 4,096 x 16,384 bf16 took 138 us instead of 118, 1,001 x 1,131 fp32 8.3 instead of 6.4.
constexpr float NORM_EPS = 0x1p-108f;
static_assert(CLEARMOE_NORM_MAX <= 1 << 15);
constexpr float NORM_LOW = 0x1p-120f;
// 1 / sqrt(mean(v^2) + eps) of a row whose squares `ss` sums up to infinity or may have lost bits, its values scaled by a power
// of two here and left so: by 2^-8, or by 2^96, after which the smallest one's square is a normal number (they were below
// 2^-52). 0 where the mean itself is past the range, or a value infinite. By all warps of a row: ss is the same in each, a sum
// of the same parts in the same order.
template <int CH>
__device__ __forceinline__ float far_rstd(float2 (&v)[CH][8], float ss, int cols, float eps, float* s_far, int warp, int part, int wpr) {
    const float k = ss == INFINITY ? 0x1p-8f : 0x1p96f;
    float2 sq = make_float2(0.f, 0.f);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c][i] = __fmul2_rn(v[c][i], make_float2(k, k));
            sq = __ffma2_rn(v[c][i], v[c][i], sq);
        }
    float s = sq.x + sq.y;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (wpr > 1) {
        if ((threadIdx.x & 31) == 0) s_far[warp] = s;  // of an earlier row: all have read it, before that barrier of all warps
        row_sync(warp / wpr, 32 * wpr);
        s = 0.f;
        for (int i = warp - part; i < warp - part + wpr; ++i) s += s_far[i];
    }
    const float mean = s / (float)cols;
    return ss == INFINITY && mean * 0x1p16f == INFINITY ? 0.f : 1.f / sqrtf(mean + eps * k * k);
}

// A lane's 16 values (as Lane16's) to row `row`, columns k on, `left` to the row's end.
template <int OUT, int P>
__device__ __forceinline__ void put(const NormArgs& a, int64_t row, int k, int left, float2 (&y)[8], int lane) {
    if constexpr (OUT == NORM_OUT_F32 || OUT == NORM_OUT_BF16) {
        constexpr bool BF16 = OUT == NORM_OUT_BF16;
        uint16_t* b = static_cast<uint16_t*>(a.out) + row * a.ldo + k;
        float* f = static_cast<float*>(a.out) + row * a.ldo + k;
#pragma unroll
        for (int h = 0; h < 16 / P; ++h) {
            const int c = 32 * P * h;
            if (c >= left) continue;
            if (P > 1 && a.out_vec) {
                const float2* v = y + P / 2 * h;
                if constexpr (P == 8 && BF16) {
                    *reinterpret_cast<uint4*>(b + c) = pack8(v);
                } else {
#pragma unroll
                    for (int i = 0; i < P / 2; i += 2) {
                        if constexpr (BF16)
                            *reinterpret_cast<uint2*>(b + c + 2 * i) = make_uint2(pack_bf16(v[i].x, v[i].y), pack_bf16(v[i + 1].x, v[i + 1].y));
                        else
                            *reinterpret_cast<float4*>(f + c + 2 * i) = make_float4(v[i].x, v[i].y, v[i + 1].x, v[i + 1].y);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 p = y[(P * h + i) >> 1];
                    const float v = (P * h + i) & 1 ? p.y : p.x;
                    if constexpr (BF16)
                        b[c + i] = f32_to_bf16(v);
                    else
                        f[c + i] = v;
                }
            }
        }
    } else if constexpr (P > 1) {
        // lanes of rows past the last take part in the shuffles and store nothing
        constexpr bool Q8 = OUT == NORM_OUT_FP8;
        constexpr int L128 = 128 / P, LB = Q8 ? L128 : 32 / P;  // lanes of 128 columns, of a block
        uint8_t* q = static_cast<uint8_t*>(a.out) + row * a.ldo + (Q8 ? k : k / 2);
        uint8_t* scale = a.scale + (Q8 ? row * a.ld_scale + k / 128 : fp4_scale_word(row, k >> 7, a.ld_scale));
        const int pad = (int)a.ldo * (Q8 ? 1 : 2) - a.cols;  // columns of zeros after the last
#pragma unroll
        for (int h = 0; h < 16 / P; ++h) {
            const int c = 32 * P * h;
            float2* f = y + P / 2 * h;
            if (c >= left) {
#pragma unroll
                for (int i = 0; i < P / 2; ++i) f[i] = make_float2(0.f, 0.f);  // (0 times an infinite rstd is NaN)
            }
            float m = max_abs3(max_abs(f[0].x, f[0].y), f[1].x, f[1].y);
            if constexpr (P == 8) m = max_abs3(max_abs3(m, f[2].x, f[2].y), f[3].x, f[3].y);
#pragma unroll
            for (int o = LB / 2; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            const uint32_t s = Q8 ? fp8_scale_byte(abs_bits(m)) : fp4_scale_byte(abs_bits(m));
            const float inv = fp8_inverse_scale(s);
#pragma unroll
            for (int i = 0; i < P / 2; ++i) f[i] = __fmul2_rn(f[i], make_float2(inv, inv));
            const bool stores = c < left + pad && left != NO_ROW;
            if constexpr (Q8) {
                if (stores) {
                    const uint32_t lo = fp8_pack4(f[0].x, f[0].y, f[1].x, f[1].y);
                    if constexpr (P == 8)
                        *reinterpret_cast<uint2*>(q + c) = make_uint2(lo, fp8_pack4(f[2].x, f[2].y, f[3].x, f[3].y));
                    else
                        *reinterpret_cast<uint32_t*>(q + c) = lo;
                    if (lane % L128 == 0) scale[c / 128] = (uint8_t)s;
                }
            } else {
                uint32_t w = s << (8 * (lane / LB & 3));
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, LB);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 2 * LB);
                if (stores) {
                    if constexpr (P == 8)
                        *reinterpret_cast<uint32_t*>(q + c / 2) = fp4_pack8(f[0].x, f[0].y, f[1].x, f[1].y, f[2].x, f[2].y, f[3].x, f[3].y);
                    else
                        *reinterpret_cast<uint16_t*>(q + c / 2) = (uint16_t)fp4_pack8(f[0].x, f[0].y, f[1].x, f[1].y, 0.f, 0.f, 0.f, 0.f);
                    if (lane % L128 == 0) *reinterpret_cast<uint32_t*>(scale + c * 4) = w;
                }
            }
        }
    }
}

// CH pieces of 512 columns a warp; wpr warps a row (blockDim / 32 a multiple of it). FAR: eps below NORM_EPS.
template <typename T, int OUT, bool VEC, int CH, bool FAR>
__global__ void __launch_bounds__(512, CH == 1 ? 2 : 1) rms_norm_kernel(const NormArgs a, const int wpr) {
    constexpr bool AHEAD = VEC && CH == 1;  // elements by cp.async, a row ahead
    constexpr bool TURN = !VEC && (OUT == NORM_OUT_FP8 || OUT == NORM_OUT_FP4);  // values to aligned pieces for their blocks
    __shared__ float s_part[2][16], s_far[16];
    extern __shared__ uint4 s_mem[];  // AHEAD: [x, r][piece][thread]; TURN: [thread][16] values
    using Lane = Lane16<T, VEC, 32>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % wpr, per = (int)(blockDim.x >> 5) / wpr;
    auto first = [&](int c) { return (c * wpr + part) * 512 + lane * Lane::P; };
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    const uint32_t pitch = 16 * blockDim.x, tensor = Lane::N * pitch, own = smem_u32(s_mem) + 16 * threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * per, row0 = (int64_t)blockIdx.x * per + warp / wpr;
    // columns from k to the end of row `row`; none for a row that is not there
    auto left_of = [&](int64_t row, int k) { return row < a.rows ? a.cols - k : NO_ROW; };
    auto ask = [&](int64_t row) {
        if constexpr (AHEAD) {
            const int left = left_of(row, first(0));
            Lane::ask(own, pitch, static_cast<const T*>(a.x) + row * a.ldx + first(0), left);
            if (a.r) Lane::ask(own + tensor, pitch, static_cast<const T*>(a.r) + row * a.ldr + first(0), left);
            cp_async_commit();
        }
    };
    float2 w[8];
    ask(row0);
    if constexpr (CH == 1) weights<Lane::P>(a, first(0), w);
    int turn = 0;
    for (int64_t row = row0; row - warp / wpr < a.rows; row += step, turn ^= 1) {
        float2 v[CH][8], sq = make_float2(0.f, 0.f);
        if constexpr (AHEAD) cp_async_wait<0>();
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int left = left_of(row, first(c));
            Lane x, r;
            if constexpr (AHEAD) {
                x.take(own, pitch, a.cols - first(0));
                if (a.r) r.take(own + tensor, pitch, a.cols - first(0));
            } else {
                x.load(static_cast<const T*>(a.x) + row * a.ldx + first(c), left);
                if (a.r) r.load(static_cast<const T*>(a.r) + row * a.ldr + first(c), left);
            }
            if (a.r) x.add(r);
            ask(row + step);
            if (a.sum) x.store(static_cast<T*>(a.sum) + row * a.lds + first(c), left);
            x.values(v[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 k = FAR ? v[c][i] : __fmul2_rn(v[c][i], make_float2(0x1p-8f, 0x1p-8f));
                sq = __ffma2_rn(k, k, sq);
            }
        }
        float ss = sq.x + sq.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        if (wpr > 1) {  // in two buffers by turn: a warp's reads of one precede its next barrier
            if (lane == 0) s_part[turn][warp] = ss;
            __syncthreads();
            ss = 0.f;
            for (int i = warp - part; i < warp - part + wpr; ++i) ss += s_part[turn][i];
        }
        const float mean = ss / (float)a.cols * (FAR ? 1.f : 0x1p16f) + a.eps;
        float rstd;
        if (FAR && (ss == INFINITY || mean < NORM_LOW))
            rstd = far_rstd<CH>(v, ss, a.cols, a.eps, s_far, warp, part, wpr);
        else
            rstd = 1.f / sqrtf(mean);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (CH > 1) weights<Lane::P>(a, first(c), w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] = __fmul2_rn(v[c][i], make_float2(rstd, rstd));
                if (a.w) v[c][i] = __fmul2_rn(v[c][i], w[i]);
            }
            if constexpr (TURN) {  // element i of lane l is column 32 i + l; lane l then has eight from 8 l and from 256 + 8 l on
                float* t = reinterpret_cast<float*>(s_mem) + warp * 512;
                const int k = first(c) - lane + 8 * lane;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 16; ++i) t[32 * i + lane] = first(c) + 32 * i < a.cols ? (i & 1 ? v[c][i >> 1].y : v[c][i >> 1].x) : 0.f;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 q = *reinterpret_cast<const float4*>(t + 256 * (i >> 1) + 8 * lane + 4 * (i & 1));
                    v[c][2 * i] = make_float2(q.x, q.y), v[c][2 * i + 1] = make_float2(q.z, q.w);
                }
                put<OUT, 8>(a, row, k, left_of(row, k), v[c], lane);
            } else {
                put<OUT, Lane::P>(a, row, first(c), left_of(row, first(c)), v[c], lane);
            }
        }
    }
}

constexpr int NORM_THREADS = 1024;  // an SM

template <typename T, int OUT, bool VEC, int CH, bool FAR>
cudaError_t launch_far(const NormArgs& a, int wpr, int num_sms, cudaStream_t s) {
    const int per = wpr <= 8 ? 8 / wpr : 1, threads = 32 * wpr * per;  // rows at a time
    int ctas = NORM_THREADS / threads;
    cudaLaunchConfig_t cfg = {};
    const bool ahead = VEC && CH == 1, turn = !VEC && (OUT == NORM_OUT_FP8 || OUT == NORM_OUT_FP4);
    if (ahead || turn) {
        cfg.dynamicSmemBytes = threads * (turn ? 64 : (a.r ? 32 : 16) * (int)sizeof(T));
        const cudaError_t e = smem_attr_once((const void*)rms_norm_kernel<T, OUT, VEC, CH, FAR>, 512 * (turn ? 64 : 32 * (int)sizeof(T)));
        if (e != cudaSuccess) return e;
    }
    const int64_t want = (a.rows + per - 1) / per, most = (int64_t)num_sms * (ctas < 1 ? 1 : ctas);
    cfg.gridDim = dim3((unsigned)(want < most ? want : most));
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, rms_norm_kernel<T, OUT, VEC, CH, FAR>, a, wpr);
}
template <typename T, int OUT, bool VEC, int CH>
cudaError_t launch_ch(const NormArgs& a, int wpr, int num_sms, cudaStream_t s) {
    return a.eps < NORM_EPS ? launch_far<T, OUT, VEC, CH, true>(a, wpr, num_sms, s) : launch_far<T, OUT, VEC, CH, false>(a, wpr, num_sms, s);
}
template <typename T, int OUT, bool VEC>
cudaError_t launch_norm(const NormArgs& a, int num_sms, cudaStream_t s) {
    const int pieces = (a.cols + 511) / 512;
    return pieces <= 16 ? launch_ch<T, OUT, VEC, 1>(a, pieces, num_sms, s) : launch_ch<T, OUT, VEC, 4>(a, (pieces + 3) / 4, num_sms, s);
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
    const int sms = current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = esz == 2 ? (vec ? launch_norm<uint16_t, OUT, true>(a, sms, s) : launch_norm<uint16_t, OUT, false>(a, sms, s))
                                   : (vec ? launch_norm<float, OUT, true>(a, sms, s) : launch_norm<float, OUT, false>(a, sms, s));
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
    a.ldo = ldo;
    a.out_vec = cm::rows_vec(out, ldo, out_dtype == CLEARMOE_BF16 ? 2 : 4);
    return out_dtype == CLEARMOE_BF16 ? cm::run<cm::NORM_OUT_BF16>(n, a, stream) : cm::run<cm::NORM_OUT_F32>(n, a, stream);
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
