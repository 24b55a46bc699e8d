// Operand handling shared by the two adapter kernels: 16 bytes a lane of
// either type, at any element alignment, and the matrix instructions on them.
#pragma once

#include "planes.h"

namespace onexn {

constexpr int kMaxRank = 128;

// One matrix-instruction step contracts 4 * V entries: lane group q = lane / 16
// holds entries q * V .. q * V + V - 1 of row (or column) lane % 16 of each
// operand.  bf16: one 16x16x32 instruction; fp32: four 16x16x4 ones, the t-th
// on entries {q * 4 + t}.  The result's lane holds rows q * 4 .. q * 4 + 3 of
// column lane % 16.
template <typename T> struct Mat;
template <> struct Mat<uint16_t> {
    static constexpr int V = 8;
    __device__ static f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    }
    // Column i of the V x V block whose rows the V registers hold.
    __device__ static u32x4 column(const u32x4 (&w)[V], int i) {
        u32x4 r;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            r[k] = __builtin_amdgcn_perm(w[2 * k + 1][i / 2], w[2 * k][i / 2], i % 2 ? 0x07060302 : 0x05040100);
        return r;
    }
};
template <> struct Mat<float> {
    static constexpr int V = 4;
    __device__ static f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[t]), __uint_as_float(b[t]), c, 0, 0, 0);
        return c;
    }
    __device__ static u32x4 column(const u32x4 (&w)[V], int i) { return u32x4{w[0][i], w[1][i], w[2][i], w[3][i]}; }
};

// Sixteen bytes at an address that is aligned to elements only.
template <typename T> struct Bytes16;
template <> struct Bytes16<uint16_t> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2), may_alias));
};
template <> struct Bytes16<float> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4), may_alias));
};

template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p) {
    return *reinterpret_cast<const typename Bytes16<T>::type*>(p);
}

// Sixteen bytes with their first `skip` elements (any count) replaced by zeros.
template <typename T>
__device__ __forceinline__ u32x4 without_first(u32x4 w, int32_t skip) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) w[k] = k < skip ? 0u : w[k];
        else w[k] &= (2 * k < skip ? 0u : 0xffffu) | (2 * k + 1 < skip ? 0u : 0xffff0000u);
    }
    return w;
}

// The three planes of eight floats: v is cut to its upper 16 bits, the remainder
// (exact) likewise, and the third holds what is left: v exactly, down to bf16's
// last subnormal bit, 2^-133.  Cut, unlike rounded, no finite value gets an
// infinite plane; an infinite one gets NaN in the second.
constexpr int kPlanes = 3;
__device__ __forceinline__ void cut_planes(const float (&v)[8], u32x4 (&p)[kPlanes]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float a = v[2 * k], b = v[2 * k + 1];
#pragma unroll
        for (int t = 0; t < kPlanes; ++t) {
            p[t][k] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
            a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
    }
}

}  // namespace onexn
