// Pieces shared by the kernels of products in 4-bit blocks: instruction descriptor, tiles, outputs. The epilogue's
// arithmetic, the stores of fp32 and bf16 rows and the copy of scales to tensor memory are fp8_gemm.cuh's.
#pragma once

#include "fp4.cuh"
#include "fp8_gemm.cuh"

namespace cm {

constexpr int F4_BK = 256;  // columns of a stage: 128 bytes of q, two scale tiles
constexpr int F4_SF = 1024;  // bytes of a stage's scales for 128 rows

// Instruction descriptor of kind::mxf4: e2m1 A and W, UE8M0 scales of 32 columns; `half` selects the two scale bytes of
// each word that an MMA of 64 columns takes.
__device__ __forceinline__ uint32_t idesc_mxf4(int M, int N, int half) {
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (1u << 23) |
           ((uint32_t)(M >> 4) << 24) | ((uint32_t)(2 * half) << 29);
}

// Row boundaries of the groups, off[E + 1], held to ascend within the rows (f8_groups), and the row tiles before each,
// prefix[E + 1]. A group's tiles start at the scale tile that its first row lies in, so that scales come as they lie;
// rows of another group in its first and last tile are computed and not stored.
// By one warp, a group a lane: E + 1 loads one after the other took 2 us.
template <class Args>
__device__ __forceinline__ void f4_groups(const Args& a, int bm, int* off, int* prefix, int lane) {
    int v = lane <= a.E ? __ldcg(a.offsets + lane) : (int)a.M;
    v = max(v, 0);
#pragma unroll
    for (int o = 1; o <= CM_MAX_E; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v = max(v, u);
    }
    v = min(v, (int)a.M);
    const int end = __shfl_down_sync(0xFFFFFFFFu, v, 1);
    const int n = lane < a.E && end > v ? (end - (v & ~127) + bm - 1) / bm : 0;
    int sum = n;  // of the groups up to this one
#pragma unroll
    for (int o = 1; o <= CM_MAX_E; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += u;
    }
    if (lane <= a.E) {
        off[lane] = v;
        prefix[lane] = sum - n;
    }
}
// The maps of group 0's tiles, of a product with its kernel's parameters, on their way.
template <class Args>
__device__ __forceinline__ void f4_prefetch_maps(const Args& a) {
    const CUtensorMap* m[4] = {&a.tmA, &a.tmB[0], &a.tmSA, &a.tmSB[0]};
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m[i])) : "memory");
}
// A box on its way to L2, by the elected lane of a converged warp. Weights are asked for so before the kernel waits for its
// predecessor: nothing of them is read before that, and a write of the predecessor's goes to the same L2.
__device__ __forceinline__ void l2_prefetch_2d(const CUtensorMap* map, int32_t c0, int32_t c1) {
    asm volatile(
        "{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
        "@q cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];\n\t}" ::"l"(reinterpret_cast<uint64_t>(map)),
        "r"(c0), "r"(c1)
        : "memory");
}

// F8Walk over such tiles: rows [max(m0, lo), hi) of a tile are the group's. Without groups nothing is read of off and prefix.
template <bool GROUPED>
struct F4Walk {
    int mt, nt;  // row and column tile
    int e, m0, lo, hi, n0;
    int m_tiles, n_tiles, bm, bn, E, step_mt, step_nt;
    const int* off;
    const int* prefix;
    template <class Args>
    __device__ __forceinline__ F4Walk(int first, int step, const Args& a, int bm_, int bn_, const int* off_, const int* prefix_)
        : e(0), lo(0), hi((int)a.M), n_tiles((a.N + bn_ - 1) / bn_), bm(bm_), bn(bn_), E(a.E), off(off_), prefix(prefix_) {
        m_tiles = GROUPED ? prefix[E] : ((int)a.M + bm - 1) / bm;
        mt = first / n_tiles;
        nt = first - mt * n_tiles;
        step_mt = step / n_tiles;
        step_nt = step - step_mt * n_tiles;
        place();
    }
    __device__ __forceinline__ bool live() const { return mt < m_tiles; }
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
        n0 = nt * bn;
        if constexpr (GROUPED) {
            while (e + 1 < E && prefix[e + 1] <= mt) ++e;
            lo = off[e];
            m0 = (lo & ~127) + (mt - prefix[e]) * bm;
            hi = off[e + 1];
        } else {
            m0 = mt * bm;
        }
    }
};

// The tiles of one of `units` walkers: rounds in which each has one, then `rest` tiles. Where those are for half of the
// walkers at the most, each is two of half the width (HALVES).
template <bool GROUPED, bool HALVES>
struct F4PairWalk : F4Walk<GROUPED> {
    using Walk = F4Walk<GROUPED>;
    int left;     // tiles of this walker to go
    bool halved;  // the last one is a half
    template <class Args>
    __device__ __forceinline__ F4PairWalk(int unit, int units, const Args& a, int bm_, int bn_, const int* off_, const int* prefix_)
        : Walk(unit, units, a, bm_, bn_, off_, prefix_) {
        int rest = a.rest;
        left = whole(a, units, rest);
        halved = HALVES && 2 * rest <= units;
        const bool more = unit < (halved ? 2 * rest : rest);
        halved = halved && more;
        if (more) ++left;
        if (GROUPED && half()) turn(unit);
    }
    // Rounds in which each walker has a whole tile.
    template <class Args>
    __device__ __forceinline__ int whole(const Args& a, int units, int& rest) const {
        if constexpr (!GROUPED) return a.whole;
        const int tiles = this->m_tiles * this->n_tiles, rounds = tiles / units;
        rest = tiles - rounds * units;
        return rounds;
    }
    __device__ __forceinline__ bool live() const { return left > 0; }
    __device__ __forceinline__ bool half() const { return HALVES && left == 1 && halved; }
    __device__ __forceinline__ void next(int unit) {
        --left;
        Walk::next();
        if (half()) turn(unit);
    }
    // From the tile that would be the walker's in the last round to the one it has half of: walkers 2 i and 2 i + 1 have tile i.
    __device__ __forceinline__ void turn(int unit) {
        for (this->nt -= (unit + 1) >> 1; this->nt < 0; this->nt += this->n_tiles) --this->mt;
        this->e = 0;
        this->place();
        if (unit & 1) this->n0 += this->bn / 2;
    }
};

// The output row of row m of A (-1: none).
template <class Args>
__device__ __forceinline__ int f4_out_row(const Args& a, int m, int lo, int hi) {
    return m >= lo ? f8_out_row(a, m, hi) : -1;
}

// A row's 32 columns [nc, nc + 32) to a block, zeros past N.
template <class Args>
__device__ __forceinline__ uint4 f4_block(const Args& a, float (&v)[32], int nc, uint32_t& scale) {
    if (nc + 32 > a.N) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (nc + i >= a.N) v[i] = 0.f;
    }
    scale = fp4_scale_byte(abs_bits(f8_max_abs32(v)));
    const float inv = fp8_inverse_scale(scale);
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fp4_pack8_scaled(v + 8 * i, make_float2(inv, inv));
    return make_uint4(o[0], o[1], o[2], o[3]);
}
// B blocks side by side of output row `row` (-1: none), from column nc on (B == 2: a multiple of 64, as rows of q are long).
template <int B, class Args>
__device__ __forceinline__ void f4_store_blocks(const Args& a, const uint4* block, const uint32_t* scale, int row, int nc) {
    if (row < 0 || nc / 2 >= a.ldo) return;
    uint8_t* q = static_cast<uint8_t*>(a.out) + (int64_t)row * a.ldo + nc / 2;
    uint8_t* s = a.out_scale + fp4_scale_word(row, nc >> 7, a.ldos) + (nc >> 5 & 3);
    if constexpr (B == 2) {
        const uint32_t w[8] = {block[0].x, block[0].y, block[0].z, block[0].w, block[1].x, block[1].y, block[1].z, block[1].w};
        st_global_32(q, w);
        *reinterpret_cast<uint16_t*>(s) = (uint16_t)(scale[0] | scale[1] << 8);
    } else {
        *reinterpret_cast<uint4*>(q) = block[0];
        *s = (uint8_t)scale[0];
    }
}

// 32 rows' 32 columns [nc, nc + 32) (one row a lane: its output row, or -1) to out.
template <int KIND, class Args>
__device__ __forceinline__ void f4_store32(const Args& a, float (&v)[32], int row, int nc, bool wide, int lane) {
    if constexpr (KIND == FP4_OUT_FP4) {
        uint4 block[1];
        uint32_t scale[1];
        block[0] = f4_block(a, v, nc, scale[0]);
        f4_store_blocks<1>(a, block, scale, row, nc);
    } else {
        if ((Args::GROUPED && a.rows) || (wide && nc + 32 <= a.N)) {
            f8_store32<KIND>(a, v, row, nc, wide, lane);
            return;
        }
        // rows of any pitch in order, of which a group's first tile may leave out the first ones
        __syncwarp();
        f8_transpose(v, lane);
        const uint32_t live = __ballot_sync(0xFFFFFFFFu, row >= 0);
        if (!live) return;
        const int first = __ffs(live) - 1, end = nc + lane < a.N ? first + __popc(live) : 0;
        using T = std::conditional_t<KIND == FP8_OUT_BF16, uint16_t, float>;
        T* o = static_cast<T*>(a.out) + ((int64_t)__shfl_sync(0xFFFFFFFFu, row, first) - first) * a.ldo + nc + lane;
#pragma unroll
        for (int r = 0; r < 32; ++r, o += a.ldo) {
            if (r >= first && r < end) {
                if constexpr (KIND == FP8_OUT_BF16)
                    *o = f32_to_bf16(v[r]);
                else
                    *o = v[r];
            }
        }
    }
}

}  // namespace cm
