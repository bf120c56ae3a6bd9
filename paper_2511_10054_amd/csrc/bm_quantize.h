// 8-bit values with block scales: conversion shared by the quantizing kernels, and their launchers.
#pragma once
#include "bm_kernels.h"

namespace bm {

constexpr int SCALE_BLOCK = 128;         // values of a row (or of 128 rows) that share a scale
constexpr int MAX_NORM_D = 16384;        // a row lies in the registers of one workgroup

// Scale of a block from the bits of its largest magnitude: max(m / 448, 2^-126), NaN for an infinity or a NaN.
__device__ __forceinline__ float block_scale(uint32_t max_bits) {
    const float s = __builtin_bit_cast(float, max_bits) / 448.0f;
    if (max_bits >= 0x7f800000u) return __builtin_nanf("");
    return s < 0x1p-126f ? 0x1p-126f : s;
}

// A block's scale as a divisor.  Scales under 2^-64 are raised by 2^64, and the values with them (raise): both exact, and no
// remainder is rounded among the denormals.
struct Divisor {
    float s, inv, lift;
};
__device__ __forceinline__ Divisor divisor(float scale) {
    const float lift = scale < 0x1p-64f ? 0x1p64f : 1.0f, s = scale * lift;
    return Divisor{s, 1.0f / s, lift};
}

// (a branch that waves rarely take: as a product for every value it cost 2 % of bm_quantize by blocks)
template <int N>
__device__ __forceinline__ void raise(float (&v)[N], const Divisor &d) {
    if (__any(d.lift != 1.0f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= d.lift;
    }
}

// x / scale rounded to 32 bits, x raised: the product with the reciprocal is within two units in the last place, one step of the remainder
// makes it the rounded quotient.  Without it 16-bit inputs, whose quotients often lie exactly half way between two e4m3 values, fall
// to either side, and so they do in blocks under 1e-31 that are not raised.  The remainder is taken as y s - x, so that -0 stays -0.
__device__ __forceinline__ float quotient(float x, const Divisor &d) {
    const float y = x * d.inv;
    return fmaf(-fmaf(y, d.s, -x), d.inv, y);
}

// Four values (magnitudes up to 448) to e4m3, rounded to nearest even, the first in the lowest byte
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
}

struct NormParams {
    const void *x, *residual, *gamma;    // residual: or null
    void *residual_out, *y;              // or null
    uint8_t *q;                          // or null (then scale is not written)
    float *scale;
    int T, d;
    float eps;
};

// the launch's grid stays within its limits
inline bool quantize_grid_ok(int n, int rows, int cols, bool blocks) {
    const long long kb = ((long long)cols + SCALE_BLOCK - 1) / SCALE_BLOCK, rb = ((long long)rows + SCALE_BLOCK - 1) / SCALE_BLOCK;
    return blocks ? rb <= 65535 && n <= 65535 && kb < (1ll << 24)                   // 256 threads a block, under 2^32 along each side
                  : (long long)n * rows <= ((1ll << 28) - 16) / kb;                  // 16 threads a block, under 2^32 a launch
}

// Threads of a norm's workgroup: eight values each, in whole waves, twice eight past 8192
inline int norm_threads(int d) {
    const int nt = ((d + 7) / 8 + 63) / 64 * 64;
    return nt < 1024 ? nt : 1024;
}
inline bool norm_grid_ok(int T, int d) { return (long long)T * norm_threads(d) < (1ll << 32); }

int launch_add_rmsnorm(const NormParams &p, bool f32, hipStream_t st);
int launch_quantize(const void *src, bool f32, uint8_t *q, float *scale, int n, int rows, int cols, bool blocks, hipStream_t st);

}  // namespace bm
