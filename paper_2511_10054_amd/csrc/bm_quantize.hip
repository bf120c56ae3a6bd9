// Quantization to 8 bits (e4m3: sign, four exponent and three mantissa bits, no infinities) with one 32-bit scale for each block of 128
// values, alone (bm_quantize) and behind the residual's addition and the root-mean-square norm (bm_add_rmsnorm).
//
// Of a block with largest magnitude m:  s = max(m / 448, 2^-126),  q = e4m3(x / s), every rounding to nearest even and
// both quotients rounded to 32 bits.  s keeps q within e4m3's +-448 and 1 / s finite.  A block that holds an infinity or
// a NaN gets s = NaN and NaN throughout: what it stands for is no number either.
#include "bm_quantize_device.h"

namespace bm {

// ---------------------------------------------------------------------------------------------------------------------
// A scale for each 128 values of a row: 16 lanes of eight values each hold a block.  Bound by HBM, by the launch where rows are
// few: 16384 x 4096 of bf16 5.2 to 5.4 TB/s; 4095 x 1440 of fp32 6.3 us, of which the launch is 3.
// ---------------------------------------------------------------------------------------------------------------------
template <bool ALIGNED, typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T *src, uint8_t *q, float *scale, long long n_rows, int cols, int kb) {
    quantize_row_block<ALIGNED>(src, q, scale, (uint32_t)blockIdx.x * 16 + (threadIdx.x >> 4), n_rows, cols, kb);
}

// ---------------------------------------------------------------------------------------------------------------------
// A scale for each 128 x 128 block of a matrix: one workgroup a block, its 16384 values in registers between the
// search for the largest and the conversion (16-bit ones packed).  Bound by HBM: 16 x 1408 x 2048 of bf16 in 29 us, 4.8 TB/s, larger
// ones up to 5.7, 4 x 4096 x 4096 of fp32 in 60 us, 5.6 (a copy, with as many bytes written as read: 5.1).
// ---------------------------------------------------------------------------------------------------------------------
template <bool ALIGNED, typename T>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const T *src, uint8_t *q, float *scale, int rows, int cols) {
    __shared__ uint32_t s_max[4];
    const int tid = threadIdx.x;
    const int j = blockIdx.x * SCALE_BLOCK + (tid & 15) * 8, r0 = blockIdx.y * SCALE_BLOCK + (tid >> 4);
    const size_t base = (size_t)blockIdx.z * rows * cols;
    Piece<T> v[8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        v[i].clear();
        if (r < rows && j < cols) v[i].template load<ALIGNED>(src + base + (size_t)r * cols + j, cols - j);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, v[i].max_of());
    m = wave_max_u32(m);
    if ((tid & 63) == 0) s_max[tid >> 6] = m;
    __syncthreads();
    m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    const float s = block_scale(m);
    const Divisor by = divisor(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        float f[8];
        v[i].get(f);
        if (r < rows && j < cols) store_q8<ALIGNED>(q + base + (size_t)r * cols + j, cols - j, f, by);
    }
    if (tid == 0) scale[((size_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x] = s;
}

// ---------------------------------------------------------------------------------------------------------------------
// r = x + residual, n = r / sqrt(mean(r^2) + eps) * gamma, in 32 bits; r and n are rounded once where they are written,
// n's 8-bit form is made from the 32-bit values.  One workgroup a row, which stays in registers (NIT pieces of eight
// values a thread) between the sum and the outputs: every input is read once.  Bound by HBM: 8192 x 2048 of bf16 with all outputs
// in 31 us, 4.9 TB/s, 8192 x 4096 of fp32 in 103 us, 5.6 TB/s; one row by the launch and two trips to memory, 5.6 us.
// ---------------------------------------------------------------------------------------------------------------------
template <bool ALIGNED, typename T, int NIT>
__global__ void __launch_bounds__(1024) add_rmsnorm_kernel(NormParams p) {
    __shared__ float s_sum[16];
    const int tid = threadIdx.x, nt = blockDim.x, d = p.d;
    const size_t at = (size_t)blockIdx.x * d;
    const T *x = static_cast<const T *>(p.x) + at, *res = p.residual ? static_cast<const T *>(p.residual) + at : nullptr;
    const T *gamma = static_cast<const T *>(p.gamma);
    float v[NIT][8], g[NIT][8];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int j = (i * nt + tid) * 8;
        float r[8] = {};
#pragma unroll
        for (int u = 0; u < 8; ++u) v[i][u] = g[i][u] = 0.0f;
        if (j < d) {
            load8<ALIGNED>(x + j, d - j, v[i]);
            if (res) load8<ALIGNED>(res + j, d - j, r);
            load8<ALIGNED>(gamma + j, d - j, g[i]);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            v[i][u] += r[u];
            sum = fmaf(v[i][u], v[i][u], sum);
        }
    }
    sum = wave_sum(sum);
    if (nt > WAVE) {
        if ((tid & 63) == 0) s_sum[tid >> 6] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int w = 0; w < nt / WAVE; ++w) sum += s_sum[w];
    }
    const float rs = 1.0f / sqrtf(sum / (float)d + p.eps);
    const int kb = (d + SCALE_BLOCK - 1) / SCALE_BLOCK;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
        const int j = (i * nt + tid) * 8;
        if (p.residual_out && j < d) store8<ALIGNED>(static_cast<T *>(p.residual_out) + at + j, d - j, v[i]);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[i][u] = v[i][u] * rs * g[i][u];
        if (p.y && j < d) store8<ALIGNED>(static_cast<T *>(p.y) + at + j, d - j, v[i]);
        if (p.q) {
            // lanes past the row's end hold gamma = 0 and may have 0 * infinity there: they are left out
            const uint32_t m = row16_max_u32(j < d ? max_bits(v[i], 0) : 0u);
            if (j < d) {
                const float s = block_scale(m);
                store_q8<ALIGNED>(p.q + at + j, d - j, v[i], divisor(s));
                if ((tid & 15) == 0) p.scale[(size_t)blockIdx.x * kb + j / SCALE_BLOCK] = s;
            }
        }
    }
}

template <typename T>
static void launch_norm_t(const NormParams &p, hipStream_t st) {
    const bool al = p.d % 8 == 0 && aligned16(p.x) && aligned16(p.residual) && aligned16(p.gamma) && aligned16(p.residual_out) &&
                    aligned16(p.y) && ((uintptr_t)p.q & 7) == 0;
    const int nt = norm_threads(p.d);
    const bool two = p.d > nt * 8;
    if (al && !two) hipLaunchKernelGGL((add_rmsnorm_kernel<true, T, 1>), dim3(p.T), dim3(nt), 0, st, p);
    else if (al) hipLaunchKernelGGL((add_rmsnorm_kernel<true, T, 2>), dim3(p.T), dim3(nt), 0, st, p);
    else if (!two) hipLaunchKernelGGL((add_rmsnorm_kernel<false, T, 1>), dim3(p.T), dim3(nt), 0, st, p);
    else hipLaunchKernelGGL((add_rmsnorm_kernel<false, T, 2>), dim3(p.T), dim3(nt), 0, st, p);
}

int launch_add_rmsnorm(const NormParams &p, bool f32, hipStream_t st) {
    if (f32) launch_norm_t<float>(p, st);
    else launch_norm_t<uint16_t>(p, st);
    return launch_status(__func__);
}

template <typename T>
static void launch_quantize_t(const void *src, uint8_t *q, float *scale, int n, int rows, int cols, bool blocks, hipStream_t st) {
    const bool al = cols % 8 == 0 && aligned16(src) && ((uintptr_t)q & 7) == 0;
    const int kb = cols / SCALE_BLOCK + (cols % SCALE_BLOCK != 0);       // (the sum of cols and 127 can pass 2^31)
    const T *s = static_cast<const T *>(src);
    if (blocks) {
        const dim3 grid(kb, (rows + SCALE_BLOCK - 1) / SCALE_BLOCK, n);
        if (al) hipLaunchKernelGGL((quantize_blocks_kernel<true, T>), grid, dim3(256), 0, st, s, q, scale, rows, cols);
        else hipLaunchKernelGGL((quantize_blocks_kernel<false, T>), grid, dim3(256), 0, st, s, q, scale, rows, cols);
    } else {
        const long long n_rows = (long long)n * rows;
        const dim3 grid((unsigned)((n_rows * kb + 15) / 16));
        if (al) hipLaunchKernelGGL((quantize_rows_kernel<true, T>), grid, dim3(256), 0, st, s, q, scale, n_rows, cols, kb);
        else hipLaunchKernelGGL((quantize_rows_kernel<false, T>), grid, dim3(256), 0, st, s, q, scale, n_rows, cols, kb);
    }
}

int launch_quantize(const void *src, bool f32, uint8_t *q, float *scale, int n, int rows, int cols, bool blocks, hipStream_t st) {
    if (f32) launch_quantize_t<float>(src, q, scale, n, rows, cols, blocks, st);
    else launch_quantize_t<uint16_t>(src, q, scale, n, rows, cols, blocks, st);
    return launch_status(__func__);
}

}  // namespace bm
