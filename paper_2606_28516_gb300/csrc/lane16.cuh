// Rows of bf16 or fp32 as the norm and the 4-bit quantiser read them: 16 elements a lane.
#pragma once

#include <type_traits>

#include "common.cuh"

namespace cm {

// x + r as stored. In bf16 one rounding of the exact sum, which that of the fp32 sum equals: a term whose last bit fp32
// drops is below 2^-16 of the other, and the nearest half way point 2^-10 away.
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// A lane's 16 elements of a row that LANES lanes read together. VEC: pieces of 16 bytes, P columns each, LANES P columns
// apart, so that a load's lanes read consecutive bytes; otherwise single ones, LANES apart.
template <typename T, bool VEC, int LANES>
struct Lane16 {
    static constexpr bool BF16 = sizeof(T) == 2;
    static constexpr int P = VEC ? (BF16 ? 8 : 4) : 1, N = 16 / P;
    using Piece = std::conditional_t<VEC, uint4, T>;
    Piece u[N];
    __device__ __forceinline__ static constexpr int at(int h) { return LANES * P * h; }  // piece h's column, from the first on

    // p: the first element's place; left: columns from there to the row's end
    __device__ __forceinline__ void load(const T* p, int left) {
        if (VEC || left > at(N - 1)) {  // whole warps of single elements without a test each
#pragma unroll
            for (int h = 0; h < N; ++h) {
                if (VEC) u[h] = Piece{};
                if (!VEC || at(h) < left) u[h] = __ldcg(reinterpret_cast<const Piece*>(p + at(h)));
            }
        } else {
#pragma unroll
            for (int h = 0; h < N; ++h) u[h] = at(h) < left ? __ldcg(reinterpret_cast<const Piece*>(p + at(h))) : Piece{};
        }
    }
    // The same by way of shared memory (VEC), a thread's pieces `pitch` apart.
    __device__ __forceinline__ static void ask(uint32_t to, uint32_t pitch, const T* p, int left) {
#pragma unroll
        for (int h = 0; h < N; ++h)
            if (at(h) < left) cp_async_16(to + h * pitch, p + at(h));
    }
    __device__ __forceinline__ void take(uint32_t from, uint32_t pitch, int left) {
        if constexpr (VEC) {
#pragma unroll
            for (int h = 0; h < N; ++h) {
                u[h] = make_uint4(0, 0, 0, 0);
                if (at(h) < left)
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(u[h].x), "=r"(u[h].y), "=r"(u[h].z), "=r"(u[h].w)
                                 : "r"(from + h * pitch)
                                 : "memory");
            }
        }
    }
    __device__ __forceinline__ void add(const Lane16& r) {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            if constexpr (VEC && BF16) {
                u[h].x = add_bf16x2(u[h].x, r.u[h].x), u[h].y = add_bf16x2(u[h].y, r.u[h].y);
                u[h].z = add_bf16x2(u[h].z, r.u[h].z), u[h].w = add_bf16x2(u[h].w, r.u[h].w);
            } else if constexpr (VEC) {
                float2 p = __fadd2_rn(make_float2(__uint_as_float(u[h].x), __uint_as_float(u[h].y)),
                                      make_float2(__uint_as_float(r.u[h].x), __uint_as_float(r.u[h].y)));
                float2 q = __fadd2_rn(make_float2(__uint_as_float(u[h].z), __uint_as_float(u[h].w)),
                                      make_float2(__uint_as_float(r.u[h].z), __uint_as_float(r.u[h].w)));
                u[h] = make_uint4(__float_as_uint(p.x), __float_as_uint(p.y), __float_as_uint(q.x), __float_as_uint(q.y));
            } else if constexpr (BF16) {
                u[h] = (T)add_bf16x2(u[h], r.u[h]);
            } else {
                u[h] += r.u[h];
            }
        }
    }
    __device__ __forceinline__ void store(T* p, int left) const {
#pragma unroll
        for (int h = 0; h < N; ++h)
            if (at(h) < left) *reinterpret_cast<Piece*>(p + at(h)) = u[h];
    }
    __device__ __forceinline__ void values(float2 (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (!VEC && BF16)
                v[i] = make_float2(bf16_to_f32(u[2 * i]), bf16_to_f32(u[2 * i + 1]));
            else if constexpr (!VEC)
                v[i] = make_float2(u[2 * i], u[2 * i + 1]);
            else if constexpr (BF16) {
                const uint4& p = u[i >> 2];
                const uint32_t w = (i & 3) == 0 ? p.x : (i & 3) == 1 ? p.y : (i & 3) == 2 ? p.z : p.w;
                v[i] = make_float2(bf16_lo(w), bf16_hi(w));
            } else {
                const uint4& p = u[i >> 1];
                v[i] = i & 1 ? make_float2(__uint_as_float(p.z), __uint_as_float(p.w)) : make_float2(__uint_as_float(p.x), __uint_as_float(p.y));
            }
        }
    }
};

}  // namespace cm
