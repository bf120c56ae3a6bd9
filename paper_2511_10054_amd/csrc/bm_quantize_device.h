// Pieces of rows and of blocks on their way to 8 bits, shared by the kernels that quantize.
#pragma once
#include "bm_quantize.h"

namespace bm {

// Largest magnitude over the 16 lanes that share a block, as the bits of a non-negative float: for those the order of the
// numbers is the order of the bits, and a NaN is above everything.
__device__ __forceinline__ uint32_t row16_max_u32(uint32_t v) {
#define BM_DPP_MAX16(ctrl_)                                                                             \
    {                                                                                                   \
        const uint32_t o_ = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl_, 0xF, 0xF, false); \
        v = o_ > v ? o_ : v;                                                                            \
    }
    BM_DPP_MAX16(0xB1)     // quad_perm [1, 0, 3, 2]
    BM_DPP_MAX16(0x4E)     // quad_perm [2, 3, 0, 1]
    BM_DPP_MAX16(0x141)    // row_half_mirror
    BM_DPP_MAX16(0x140)    // row_mirror
#undef BM_DPP_MAX16
    return v;
}

__device__ __forceinline__ uint32_t max_bits(const float (&v)[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    return m;
}

// Eight consecutive values from p, zeros from the n-th on.  ALIGNED: p lies on a 16-byte boundary and n >= 8.
template <bool ALIGNED, typename T>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8]) {
    if (ALIGNED && sizeof(T) == 2) {
        const u32x4 u = ldg128(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = bf16_to_f32((uint16_t)(u[i] & 0xffffu));
            v[2 * i + 1] = bf16_to_f32((uint16_t)(u[i] >> 16));
        }
    } else if (ALIGNED) {
        const f32x4 a = *(const BM_GLOBAL f32x4 *)p, b = *((const BM_GLOBAL f32x4 *)p + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.0f;
            if (i < n) {
                if (sizeof(T) == 2) v[i] = bf16_to_f32(*(const BM_GLOBAL uint16_t *)(const void *)(p + i));
                else v[i] = ldg_f32(p + i);
            }
        }
    }
}

template <bool ALIGNED, typename T>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8]) {
    if (ALIGNED && sizeof(T) == 2) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        stg128(p, u);
    } else if (ALIGNED) {
        f32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
        *(BM_GLOBAL f32x4 *)p = a;
        *((BM_GLOBAL f32x4 *)p + 1) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) {
                if (sizeof(T) == 2) stg16(p + i, f32_to_bf16(v[i]));
                else *(BM_GLOBAL float *)(void *)(p + i) = v[i];
            }
    }
}

template <bool ALIGNED>
__device__ __forceinline__ void store_q8(uint8_t *p, int n, float (&v)[8], const Divisor &s) {
    raise(v, s);
    const uint32_t lo = e4m3x4(quotient(v[0], s), quotient(v[1], s), quotient(v[2], s), quotient(v[3], s));
    const uint32_t hi = e4m3x4(quotient(v[4], s), quotient(v[5], s), quotient(v[6], s), quotient(v[7], s));
    if (ALIGNED) {
        const u32x2 u = {lo, hi};
        *(BM_GLOBAL u32x2 *)p = u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) *(BM_GLOBAL uint8_t *)(p + i) = (uint8_t)((i < 4 ? lo >> (8 * i) : hi >> (8 * (i - 4))) & 0xffu);
    }
}

// Eight consecutive values as they lie in memory: 16-bit ones stay packed until they are converted (half the registers, and
// their largest magnitude is found two at a time on the bits).
template <typename T> struct Piece {
    float v[8];
    template <bool ALIGNED> __device__ __forceinline__ void load(const float *p, int n) { load8<ALIGNED>(p, n, v); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    __device__ __forceinline__ uint32_t max_of() const { return max_bits(v, 0); }
    __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i];
    }
};
template <> struct Piece<uint16_t> {
    u32x4 u;
    template <bool ALIGNED> __device__ __forceinline__ void load(const uint16_t *p, int n) {
        if (ALIGNED) {
            u = ldg128(p);
        } else {
            clear();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) u[i / 2] |= (uint32_t)*(const BM_GLOBAL uint16_t *)(p + i) << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ void clear() { u = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ uint32_t max_of() const {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        auto mag = [&](int i) { return __builtin_bit_cast(u16x2, u[i] & 0x7fff7fffu); };
        const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(0), mag(1)), __builtin_elementwise_max(mag(2), mag(3)));
        return (uint32_t)max(m[0], m[1]) << 16;
    }
    __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = __builtin_bit_cast(float, u[i] << 16);
            o[2 * i + 1] = __builtin_bit_cast(float, u[i] & 0xffff0000u);
        }
    }
};

// Block blk of 128 values of n_rows rows of kb blocks (fewer than 2^28 blocks), by 16 lanes that are together in a row of 16
template <bool ALIGNED, typename T>
__device__ __forceinline__ void quantize_row_block(const T *src, uint8_t *q, float *scale, uint32_t blk, long long n_rows, int cols, int kb) {
    const long long row = blk / (uint32_t)kb;
    const int j = (int)(blk - row * kb) * SCALE_BLOCK + (threadIdx.x & 15) * 8;
    const bool in = row < n_rows && j < cols;
    Piece<T> v;
    v.clear();
    const long long at = row * cols + j;
    if (in) v.template load<ALIGNED>(src + at, cols - j);
    const uint32_t m = row16_max_u32(v.max_of());
    if (!in) return;
    const float s = block_scale(m);
    float f[8];
    v.get(f);
    store_q8<ALIGNED>(q + at, cols - j, f, divisor(s));
    if ((threadIdx.x & 15) == 0) scale[blk] = s;
}

}  // namespace bm
