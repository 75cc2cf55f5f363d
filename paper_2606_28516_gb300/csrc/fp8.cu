// 8-bit blocks with power-of-two scales: quantisation of activations (1 x 128 blocks) and weights (128 x 128
// blocks), and back. The product is in fp8_gemm.cu.
#include <cstdint>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace cm {

namespace {

// Eight consecutive elements of a row from column k on, zeros past K. VEC: the row's start and k are 16-byte
// aligned and K is a multiple of 8, so that eight elements are all inside or all outside.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int64_t k, int64_t K, float (&v)[8]) {
    if (VEC) {
        if (k >= K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            return;
        }
        if (sizeof(T) == 2) {
            const uint4 u = __ldcg(reinterpret_cast<const uint4*>(row + k));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_lo(w[i]);
                v[2 * i + 1] = bf16_hi(w[i]);
            }
        } else {
            const float4 a = __ldcg(reinterpret_cast<const float4*>(row + k));
            const float4 b = __ldcg(reinterpret_cast<const float4*>(row + k) + 1);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f = 0.f;
            if (k + i < K) {
                if (sizeof(T) == 2)
                    f = bf16_to_f32(__ldcg(reinterpret_cast<const uint16_t*>(row) + k + i));
                else
                    f = __ldcg(reinterpret_cast<const float*>(row) + k + i);
            }
            v[i] = f;
        }
    }
}

// Activations. Eight lanes take a block of 128 columns, 16 consecutive ones a lane, so that a lane's conversions
// share one scale and its largest magnitude takes three shuffles to become the block's. Bound by HBM: each element is read
// once and written once as a byte; small blocks and many CTAs keep the loads coming. Measured (16,384 x 4,096 bf16, 202 MB):
// 50 us with a half warp per block, eight columns a lane, a masked redux and integer magnitudes (19 instructions an
// element); 37 us in fp32 with two blocks' loads a lane in flight and 8 CTAs an SM (12 instructions); 30 us (6.7 TB/s) with
// the bf16 words taken two values at a time, a block a lane and 32 CTAs an SM (16: 31 us).
constexpr int Q_THREADS = 256;
constexpr int Q_CTAS = 32;  // an SM, at the most
constexpr int Q_CTA_BLOCKS = Q_THREADS / 8;

// The row of x that row `row` is made from; `inside`: x has it (an index that gather may not have is not followed). A
// kernel of its own for gathered rows (GATHER): in one for both, 8,192 x 4,095 bf16 took 39.4 us instead of 34.
template <bool GATHER>
__device__ __forceinline__ int64_t source_row(const QuantArgs& a, int64_t row, bool live, bool& inside) {
    inside = true;
    if (!GATHER || !live) return row;
    const int64_t src = __ldcg(a.gather + row);
    inside = (uint64_t)src < (uint64_t)a.src_rows;
    return src;
}

// A lane's 16 values of a block to e4m3 at q, the block's scale byte at scale; none: NaN instead.
__device__ __forceinline__ void quantize_block(float (&v)[2][8], int l8, bool write, uint8_t* q, uint8_t* scale, bool none = false) {
    float m = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 8; c += 2) m = max_abs3(m, v[h][c], v[h][c + 1]);
#pragma unroll
    for (int o = 4; o; o >>= 1) m = max_abs(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    const uint32_t s = none ? 255u : fp8_scale_byte(abs_bits(m));
    const float inv = fp8_inverse_scale(s);
    uint32_t o[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float* f = v[h >> 1] + (h & 1) * 4;
        o[h] = fp8_pack4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    }
    if (write) {
        *reinterpret_cast<uint4*>(q) = make_uint4(o[0], o[1], o[2], o[3]);
        if (l8 == 0) *scale = (uint8_t)s;
    }
}

// Aligned bf16 rows as they are loaded, two values a word: 16 of a block a lane, zeros past K.
__device__ __forceinline__ void load16_bf16(const uint16_t* row, int k, int64_t K, bool live, uint4 (&r)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        r[h] = make_uint4(0, 0, 0, 0);
        if (live && k + 8 * h < K) r[h] = __ldcg(reinterpret_cast<const uint4*>(row + k) + h);
    }
}
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t b) {  // each half's; NaN if either is
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// quantize_block on such words: magnitudes and scaling two values an instruction, both exact in bf16 (the scale is a power
// of two; what it takes below bf16's range is far below e4m3's), so that only the conversion takes them one by one.
__device__ __forceinline__ void quantize_block_bf16(const uint4 (&r)[2], int l8, bool write, uint8_t* q, uint8_t* scale, bool none = false) {
    const uint32_t w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
    uint32_t m = max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(w[0], w[1]), max_abs_bf16x2(w[2], w[3])),
                                max_abs_bf16x2(max_abs_bf16x2(w[4], w[5]), max_abs_bf16x2(w[6], w[7])));
#pragma unroll
    for (int o = 4; o; o >>= 1) m = max_abs_bf16x2(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    const uint32_t s = none ? 255u : fp8_scale_byte((max_abs_bf16x2(m, __byte_perm(m, m, 0x1032)) & 0x7FFFu) << 16);
    const uint32_t inv = __byte_perm(__float_as_uint(fp8_inverse_scale(s)), 0, 0x3232);
    uint32_t o[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint32_t a, b;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(w[2 * h]), "r"(inv));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(w[2 * h + 1]), "r"(inv));
        o[h] = fp8_pack4(bf16_lo(a), bf16_hi(a), bf16_lo(b), bf16_hi(b));
    }
    if (write) {
        *reinterpret_cast<uint4*>(q) = make_uint4(o[0], o[1], o[2], o[3]);
        if (l8 == 0) *scale = (uint8_t)s;
    }
}

// Aligned bf16 rows.
template <bool GATHER>
__global__ void __launch_bounds__(Q_THREADS) quantize_bf16_kernel(const QuantArgs a) {
    const int l8 = threadIdx.x & 7;
    const int64_t b0 = (int64_t)blockIdx.x * Q_CTA_BLOCKS + (threadIdx.x >> 3), step = (int64_t)gridDim.x * Q_CTA_BLOCKS;
    int64_t row = b0 / a.kb;
    int kb = (int)(b0 - row * a.kb);
    const int64_t step_row = step / a.kb;
    const int step_kb = (int)(step - step_row * a.kb);
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    while (__any_sync(0xFFFFFFFFu, row < a.rows)) {
        const bool live = row < a.rows;
        bool inside;
        const int64_t src = source_row<GATHER>(a, row, live, inside);
        uint4 r[2];
        load16_bf16(static_cast<const uint16_t*>(a.x) + src * a.ld, kb * 128 + l8 * 16, a.K, live && inside, r);
        quantize_block_bf16(r, l8, live, a.q + row * a.ldq + kb * 128 + l8 * 16, a.scale + row * a.lds + kb, !inside);
        row += step_row;
        kb += step_kb;
        if (kb >= a.kb) kb -= a.kb, ++row;
    }
}

// Other rows: fp32, or not 16-byte aligned (VEC false). Five CTAs an SM: 8,192 x 4,095 bf16 32.2 us, with four 36.4, with six
// 32.1, which then leave the product that follows a later start: 1,001 x 777 x 1,131 fp32 8.8 us for both, 8.7 with four, 9.5
// with six. 16,384 x 4,096 fp32, aligned, 50.6 us (6.6 TB/s).
template <typename T, bool VEC, bool GATHER>
__global__ void __launch_bounds__(Q_THREADS, 5) quantize_rows_kernel(const QuantArgs a) {
    // Unaligned rows go through shared memory, so that a load's lanes read consecutive elements: a block of the warp's four
    // at a time, 16 columns a pitch of 20. (All four at once, 17 KB a CTA, kept the product that follows from starting
    // beside it: 1,001 x 777 x 1,131 fp32 10.3 us for both.)
    __shared__ __align__(16) float s_x[VEC ? 1 : Q_THREADS / 32][VEC ? 1 : 8 * 20];
    const int l8 = threadIdx.x & 7, lane = threadIdx.x & 31;
    const int64_t b0 = (int64_t)blockIdx.x * Q_CTA_BLOCKS + (threadIdx.x >> 3), step = (int64_t)gridDim.x * Q_CTA_BLOCKS;
    int64_t row = b0 / a.kb;
    int kb = (int)(b0 - row * a.kb);
    const int64_t step_row = step / a.kb;
    const int step_kb = (int)(step - step_row * a.kb);
    pdl_wait();
    pdl_launch_dependents();  // after the wait: the next kernel may read weights that one before this has written
    while (__any_sync(0xFFFFFFFFu, row < a.rows)) {
        const bool live = row < a.rows;
        bool inside;
        const int64_t src = source_row<GATHER>(a, row, live, inside);
        const bool reads = live && inside;
        const T* x = static_cast<const T*>(a.x) + src * a.ld;
        float v[2][8];
        if (VEC) {
            load8<T, VEC>(x, (int64_t)kb * 128 + l8 * 16, reads ? a.K : 0, v[0]);
            load8<T, VEC>(x, (int64_t)kb * 128 + l8 * 16 + 8, reads ? a.K : 0, v[1]);
        } else {
            float* sx = s_x[VEC ? 0 : threadIdx.x >> 5];
            float f[16];
#pragma unroll
            for (int b = 0; b < 4; ++b) {  // the warp's four blocks
                const T* p = reinterpret_cast<const T*>(__shfl_sync(0xFFFFFFFFu, reinterpret_cast<unsigned long long>(x), 8 * b));
                const int64_t k = (int64_t)__shfl_sync(0xFFFFFFFFu, reads ? kb : a.kb, 8 * b) * 128 + lane;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    f[4 * b + c] = k + 32 * c >= a.K  ? 0.f
                                   : sizeof(T) == 2 ? bf16_to_f32(__ldcg(reinterpret_cast<const uint16_t*>(p) + k + 32 * c))
                                                    : __ldcg(reinterpret_cast<const float*>(p) + k + 32 * c);
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) sx[(2 * c + (lane >> 4)) * 20 + (lane & 15)] = f[4 * b + c];
                __syncwarp();
                if (lane >> 3 != b) continue;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float4 q = *reinterpret_cast<const float4*>(sx + l8 * 20 + 4 * c);
                    float* o = v[c >> 1] + (c & 1) * 4;
                    o[0] = q.x, o[1] = q.y, o[2] = q.z, o[3] = q.w;
                }
            }
            __syncwarp();
        }
        quantize_block(v, l8, live, a.q + row * a.ldq + kb * 128 + l8 * 16, a.scale + row * a.lds + kb, !inside);
        row += step_row;
        kb += step_kb;
        if (kb >= a.kb) kb -= a.kb, ++row;
    }
}

// The routing's slots and the tokens quantised to them in one launch (a token's row goes to its slot): CTA (c, part)
// takes every SPLIT-th row of routing range c. As route_finalize_kernel it forms the ranges' prefix from their
// histograms and writes counts, offsets and perm.
constexpr int SQ_THREADS = 512;
constexpr int SQ_ROWS = 256;  // rows at a time

template <bool LN>
__global__ void __launch_bounds__(SQ_THREADS, 2) slots_quantize_kernel(const RouteArgs r, const int chunk, const int G, const QuantArgs a) {
    __shared__ int s_before[SQ_THREADS / 32][CM_MAX_E], s_total[SQ_THREADS / 32][CM_MAX_E], s_base[CM_MAX_E];
    __shared__ int s_slot[SQ_ROWS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = r.E, split = gridDim.y;
    const int64_t row0 = (int64_t)blockIdx.x * chunk;
    const int64_t rows = max((int64_t)0, min((int64_t)chunk, r.T - row0));
    const int64_t n_cls = n_class_tokens(r.T, r.cls_stride);
    pdl_wait();  // everything below reads the routing kernel's output
    pdl_launch_dependents();
    int before[CM_MAX_E], total[CM_MAX_E];
#pragma unroll
    for (int e = 0; e < CM_MAX_E; ++e) before[e] = total[e] = 0;
    for (int b = tid; b < G; b += SQ_THREADS) {
        const int4* h = reinterpret_cast<const int4*>(r.cta_counts + (int64_t)b * CM_MAX_E);
#pragma unroll
        for (int q = 0; q < CM_MAX_E / 4; ++q) {
            if (4 * q >= E) break;
            const int4 v = __ldcg(h + q);
            const int c[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                total[4 * q + i] += c[i];
                if (b < (int)blockIdx.x) before[4 * q + i] += c[i];
            }
        }
    }
    if (warp * 32 < G) {
#pragma unroll
        for (int e = 0; e < CM_MAX_E; ++e) {
            if (e >= E) break;
            const int vb = __reduce_add_sync(0xFFFFFFFFu, before[e]), vt = __reduce_add_sync(0xFFFFFFFFu, total[e]);
            if (lane == 0) s_before[warp][e] = vb, s_total[warp][e] = vt;
        }
    }
    __syncthreads();
    if (warp == 0) {
        int b = 0, t = 0;
        if (lane < E)
            for (int w = 0; w * 32 < G && w < SQ_THREADS / 32; ++w) b += s_before[w][lane], t += s_total[w][lane];
        int incl = t;  // over experts
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane < E) {
            s_base[lane] = incl - t + b;
            if (blockIdx.x == 0 && blockIdx.y == 0) {
                r.counts[lane] = t;
                r.offsets[lane] = incl - t;
                if (lane == E - 1) {
                    r.offsets[E] = incl;
                    if (n_cls > 0) r.counts[E] = (int32_t)n_cls, r.offsets[E + 1] = incl + (int32_t)n_cls;
                }
            }
        }
    }
    __syncthreads();
    const int l8 = tid & 7, per = SQ_THREADS / 8;  // blocks at a time
    for (int64_t i0 = blockIdx.y; i0 < rows; i0 += (int64_t)SQ_ROWS * split) {  // rows i0, i0 + split, ..
        const int n = (int)min((int64_t)SQ_ROWS, (rows - i0 + split - 1) / split);
        for (int i = tid; i < n; i += SQ_THREADS) {
            const int64_t tok = row0 + i0 + (int64_t)i * split;
            int64_t slot;
            if (r.cls_stride > 0 && tok % r.cls_stride == 0) {
                slot = r.T - n_cls + tok / r.cls_stride;
            } else {
                const uint32_t w = (uint32_t)__ldcg(r.tinfo + tok);
                const int e = (int)(w & 0xFFu);
                slot = e < E ? (int64_t)s_base[e] + (int)(w >> 8) : -1;  // -1: only a routing that gave up leaves such words
                if ((uint64_t)slot >= (uint64_t)r.T) slot = -1;
            }
            s_slot[i] = (int)slot;
            if (slot >= 0) r.perm[slot] = (int32_t)tok;
        }
        __syncthreads();
        const int blocks = n * a.kb;
        for (int b = tid >> 3; b - (tid >> 3) < blocks; b += per) {
            const int row = (int)((uint32_t)b / (uint32_t)a.kb), kb = b - row * a.kb, k = kb * 128 + l8 * 16;
            const bool live = row < n;
            const int64_t tok = row0 + i0 + (int64_t)row * split;
            const int slot = live ? s_slot[row] : -1;
            uint4 w[2];
            load16_bf16(static_cast<const uint16_t*>(a.x) + tok * a.ld, k, a.K, live, w);
            uint8_t* q = a.q + (int64_t)slot * a.ldq + k;
            uint8_t* scale = a.scale + (int64_t)slot * a.lds + kb;
            if (LN) {
                const float2 st = live ? __ldcg(a.ln_stats + tok) : make_float2(0.f, 0.f);
                const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
                float v[2][8];
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const float f = c & 1 ? bf16_hi(u[c >> 1]) : bf16_lo(u[c >> 1]);
                    v[c >> 3][c & 7] = k + c < a.K ? (f - st.x) * st.y : 0.f;
                }
                quantize_block(v, l8, slot >= 0, q, scale);
            } else {
                quantize_block_bf16(w, l8, slot >= 0, q, scale);
            }
        }
        __syncthreads();
    }
}

// Weights: a block of 256 threads per 128 x 128 block, 8 columns of 8 rows a thread, read twice (the second
// time from L1 / L2). Run once per weight set.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quantize_weight_kernel(const QuantArgs a) {
    __shared__ uint32_t s_max[8];
    pdl_wait();
    const int64_t nb = blockIdx.x / a.kb;
    const int kb = (int)(blockIdx.x - nb * a.kb);
    const int l16 = threadIdx.x & 15, r16 = threadIdx.x >> 4;
    const int64_t k = (int64_t)kb * 128 + l16 * 8;
    uint32_t m = 0;
    for (int r = r16; r < 128; r += 16) {
        const int64_t row = nb * 128 + r;
        if (row >= a.rows) break;
        float v[8];
        load8<T, VEC>(static_cast<const T*>(a.x) + row * a.ld, k, a.K, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
    }
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, s_max[i]);
    const uint32_t s = fp8_scale_byte(m);
    const float inv = fp8_inverse_scale(s);
    for (int r = r16; r < 128; r += 16) {
        const int64_t row = nb * 128 + r;
        if (row >= a.rows) break;
        float v[8];
        load8<T, VEC>(static_cast<const T*>(a.x) + row * a.ld, k, a.K, v);
        uint2 o;
        o.x = fp8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        o.y = fp8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
        *reinterpret_cast<uint2*>(a.q + row * a.ldq + k) = o;
    }
    if (threadIdx.x == 0) a.scale[nb * a.lds + kb] = (uint8_t)s;
}

template <typename T>
__global__ void __launch_bounds__(256)
    dequantize_kernel(const uint8_t* q, const uint8_t* scale, int64_t rows, int64_t K, int64_t ldq, int64_t lds,
                      int block_rows, T* out, int64_t ld) {
    pdl_wait();
    const int64_t n = rows * K;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / K, k = i - r * K;
        const float v = fp8_unpack2(q[r * ldq + k]).x * fp8_scale(scale[r / block_rows * lds + k / 128]);
        if (sizeof(T) == 2)
            reinterpret_cast<uint16_t*>(out)[r * ld + k] = f32_to_bf16(v);
        else
            reinterpret_cast<float*>(out)[r * ld + k] = v;
    }
}

template <typename K, typename... A>
cudaError_t launch(K kernel, dim3 grid, int threads, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

bool vec_ok(const QuantArgs& a, int esz) {
    return (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && a.K % 8 == 0 && (a.ld * esz) % 16 == 0;
}

}  // namespace

template <bool GATHER>
static cudaError_t launch_rows(const QuantArgs& a, bool bf16, int num_sms, cudaStream_t s) {
    const bool vec = vec_ok(a, bf16 ? 2 : 4);
    const int64_t one = (a.rows * a.kb + Q_CTA_BLOCKS - 1) / Q_CTA_BLOCKS, most = (int64_t)num_sms * Q_CTAS;
    const dim3 grid((unsigned)(one < most ? one : most));
    if (vec && bf16) return launch(quantize_bf16_kernel<GATHER>, grid, Q_THREADS, s, a);
    if (bf16) return launch(quantize_rows_kernel<uint16_t, false, GATHER>, grid, Q_THREADS, s, a);
    return vec ? launch(quantize_rows_kernel<float, true, GATHER>, grid, Q_THREADS, s, a)
               : launch(quantize_rows_kernel<float, false, GATHER>, grid, Q_THREADS, s, a);
}
cudaError_t launch_quantize_rows(const QuantArgs& a, int dtype, int num_sms, cudaStream_t s) {
    const bool bf16 = dtype == CLEARMOE_BF16;
    return a.gather ? launch_rows<true>(a, bf16, num_sms, s) : launch_rows<false>(a, bf16, num_sms, s);
}

cudaError_t launch_slots_quantize(const RouteArgs& r, int grid, int chunk, const QuantArgs& a, int num_sms, cudaStream_t s) {
    // as many CTAs as two an SM, while each keeps rows for its threads
    int split = 1;
    while (split < 8 && grid * split * 2 <= 2 * num_sms && chunk >= 2 * split * SQ_THREADS / 8 / a.kb) split *= 2;
    const dim3 g(grid, split);
    return a.ln_stats ? launch(slots_quantize_kernel<true>, g, SQ_THREADS, s, r, chunk, grid, a)
                      : launch(slots_quantize_kernel<false>, g, SQ_THREADS, s, r, chunk, grid, a);
}

cudaError_t launch_quantize_weight(const QuantArgs& a, int dtype, cudaStream_t s) {
    const int esz = dtype == CLEARMOE_BF16 ? 2 : 4;
    const int64_t grid = (a.rows + 127) / 128 * a.kb;
    const bool vec = vec_ok(a, esz);
    if (dtype == CLEARMOE_BF16)
        return vec ? launch(quantize_weight_kernel<uint16_t, true>, dim3((unsigned)grid), 256, s, a)
                   : launch(quantize_weight_kernel<uint16_t, false>, dim3((unsigned)grid), 256, s, a);
    return vec ? launch(quantize_weight_kernel<float, true>, dim3((unsigned)grid), 256, s, a)
               : launch(quantize_weight_kernel<float, false>, dim3((unsigned)grid), 256, s, a);
}

}  // namespace cm

namespace {

using cm::fp8_ldq;
using cm::fp8_lds;

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int cuda_code(cudaError_t e) {
    if (e == cudaSuccess) return CLEARMOE_OK;
    (void)cudaGetLastError();
    return CLEARMOE_ECUDA;
}

int check_pair(const void* x, int32_t dtype, int64_t ld, const clearmoe_fp8* m) {
    const int rc = cm::check_fp8(m);
    if (rc) return rc;
    if (!x || (dtype != CLEARMOE_F32 && dtype != CLEARMOE_BF16) || ld < m->cols) return CLEARMOE_EINVAL;
    if (ld > (int64_t)1 << 30) return CLEARMOE_EINVAL;
    return aligned_to(x, dtype == CLEARMOE_BF16 ? 2 : 4) ? CLEARMOE_OK : CLEARMOE_EINVAL;
}

cm::QuantArgs quant_args(const void* x, int64_t ld, const clearmoe_fp8* m) {
    cm::QuantArgs a = {};
    a.x = x;
    a.ld = ld;
    a.rows = m->rows;
    a.K = m->cols;
    a.kb = (int)((m->cols + 127) / 128);
    a.q = static_cast<uint8_t*>(m->q);
    a.scale = m->scale;
    a.ldq = fp8_ldq(m->cols);
    a.lds = fp8_lds(m->cols);
    return a;
}

}  // namespace

namespace cm {

int check_fp8(const clearmoe_fp8* m) {
    if (!m || !m->q || !m->scale || m->rows < 1 || m->cols < 1) return CLEARMOE_EINVAL;
    if (m->rows > (int64_t)1 << 30 || m->cols > (int64_t)1 << 24) return CLEARMOE_EINVAL;
    return aligned_to(m->q, 32) && aligned_to(m->scale, 4) ? CLEARMOE_OK : CLEARMOE_EINVAL;
}

}  // namespace cm

extern "C" {

int clearmoe_fp8_quantize_rows(const void* x, int32_t dtype, int64_t ld, const int32_t* gather, const clearmoe_fp8* out,
                               void* stream) {
    // gathered rows without a count: 2^31, that is any index but a negative one
    return clearmoe_fp8_quantize_gathered(x, (int64_t)1 << 31, dtype, ld, gather, out, stream);
}

int clearmoe_fp8_quantize_gathered(const void* x, int64_t x_rows, int32_t dtype, int64_t ld, const int32_t* gather,
                                   const clearmoe_fp8* out, void* stream) {
    const int rc = check_pair(x, dtype, ld, out);
    if (rc) return rc;
    if (x_rows < 1 || (!gather && x_rows < out->rows)) return CLEARMOE_EINVAL;
    if (gather && !aligned_to(gather, 4)) return CLEARMOE_EINVAL;
    const int sms = cm::current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    cm::QuantArgs a = quant_args(x, ld, out);
    a.gather = gather;
    a.src_rows = x_rows;
    return cuda_code(cm::launch_quantize_rows(a, dtype, sms, static_cast<cudaStream_t>(stream)));
}

int clearmoe_fp8_quantize_weight(const void* W, int32_t dtype, int64_t ld, const clearmoe_fp8* out, void* stream) {
    const int rc = check_pair(W, dtype, ld, out);
    if (rc) return rc;
    if ((out->rows + 127) / 128 * ((out->cols + 127) / 128) > 0x7FFFFFFF) return CLEARMOE_EUNSUPPORTED;
    return cuda_code(cm::launch_quantize_weight(quant_args(W, ld, out), dtype, static_cast<cudaStream_t>(stream)));
}

int clearmoe_fp8_dequantize(const clearmoe_fp8* in, int32_t block_rows, void* out, int32_t dtype, int64_t ld, void* stream) {
    const int rc = check_pair(out, dtype, ld, in);
    if (rc) return rc;
    if (block_rows != 1 && block_rows != 128) return CLEARMOE_EINVAL;
    const int sms = cm::current_device_sms();
    if (sms <= 0) return CLEARMOE_ECUDA;
    const int64_t want = (in->rows * in->cols + 255) / 256, grid = want < (int64_t)sms * 8 ? want : (int64_t)sms * 8;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint8_t* q = static_cast<const uint8_t*>(in->q);
    const int64_t ldq = fp8_ldq(in->cols), lds = fp8_lds(in->cols);
    if (dtype == CLEARMOE_BF16)
        return cuda_code(cm::launch(cm::dequantize_kernel<uint16_t>, dim3((unsigned)grid), 256, s, q, (const uint8_t*)in->scale, in->rows,
                                    in->cols, ldq, lds, (int)block_rows, static_cast<uint16_t*>(out), ld));
    return cuda_code(cm::launch(cm::dequantize_kernel<float>, dim3((unsigned)grid), 256, s, q, (const uint8_t*)in->scale, in->rows,
                                in->cols, ldq, lds, (int)block_rows, static_cast<float*>(out), ld));
}

}  // extern "C"
