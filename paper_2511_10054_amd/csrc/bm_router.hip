// Routing by softmax or sigmoid scores with a balance bias and groups of experts.
//
//   z = x W^T + bias,  s = softmax(z) or sigmoid(z),  c = s + balance
// A group's score is the sum of its one or two largest c; the experts of the best groups stay, of those the K of largest c
// are chosen, and their s - without the balance - become the weights.
//
// Two launches: the product writes the logits (fp32, T * E values that stay in the memory-side cache), then a wave a token
// scores, ranks and weighs.  The order of a logit's additions follows from d alone: eight parts of the reduction (whole
// 128-byte lines of a row), each a chain of matrix instructions, added as ((q0 + q1) + q2) + q3 with q_j = e_2j + e_2j+1.  A
// token's ids and weights are the same bits whatever batch it is part of.
#include "bm_router.h"

namespace bm {

namespace {

constexpr int PARTS = 8;                 // of the reduction

// What a line of 128 bytes holds, and its matrix instructions: lane l has row l % 16 and the 16 bytes l / 16 of a half line.
struct Bf16Line {
    static constexpr int VALUES = 64;
    static __device__ __forceinline__ f32x4 mac(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
    }
};
struct F32Line {
    static constexpr int VALUES = 32;
    static __device__ __forceinline__ f32x4 mac(u32x4 a, u32x4 b, f32x4 c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// 16 bytes of a row from byte `at` on, zeros behind its end.  WHOLE: the row's length and the addresses are multiples of 16 bytes.
template <bool WHOLE>
__device__ __forceinline__ u32x4 piece(const char *row, int at, int bytes) {
    if constexpr (WHOLE) {
        const u32x4 v = ldg128(row + (at < bytes ? at : 0));
        return at < bytes ? v : u32x4{0, 0, 0, 0};
    } else {                               // 4-byte values at any 4-byte address
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = at + 4 * i;
            v[i] = b < bytes ? (uint32_t)ldg_i32(row + b) : 0u;
        }
        return v;
    }
}

// ---------------------------------------------------------------------------
// The product for few tokens: a workgroup takes 16 tokens x 16 experts, a wave one eighth of the reduction with the loads of up to
// eight lines in flight.  Bound by latency.
// ---------------------------------------------------------------------------
template <typename L, bool WHOLE>
__global__ void __launch_bounds__(PARTS * 64) router_small_kernel(RouterParams p) {
    __shared__ f32x4 part[PARTS][64];
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16;
    const int bytes = p.d * (128 / L::VALUES), lines = (bytes + 127) >> 7;
    const char *xr = static_cast<const char *>(p.x) + (size_t)min(t0 + r16, p.T - 1) * bytes;
    const char *wr = static_cast<const char *>(p.w) + (size_t)min(e0 + r16, p.E - 1) * bytes;
    const int begin = wave * lines / PARTS, end = (wave + 1) * lines / PARTS;
    constexpr int AHEAD = WHOLE ? 8 : 2;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int l0 = begin; l0 < end; l0 += AHEAD) {
        u32x4 a[AHEAD][2], b[AHEAD][2];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = min(l0 + i, end - 1) * 128 + h * 64 + kq * 16;
                a[i][h] = piece<WHOLE>(xr, at, bytes);
                b[i][h] = piece<WHOLE>(wr, at, bytes);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (l0 + i >= end) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = L::mac(a[i][h], b[i][h], acc);
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
    f32x4 q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = part[2 * j][lane] + part[2 * j + 1][lane];
    const f32x4 sum = ((q[0] + q[1]) + q[2]) + q[3];
    const int e = e0 + r16;
    if (e >= p.E) return;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int t = t0 + 4 * kq + v;
        if (t < p.T) p.logits[(size_t)t * p.E + e] = sum[v];
    }
}

// ---------------------------------------------------------------------------
// Scores, groups, choice and weights: a wave a token, lane l holds experts l, l + 64, ..  Bound by latency, hidden by the
// other waves: 16 of them share a unit's schedulers.
// EC: experts a lane; PARTED: the logits are four parts.
// ---------------------------------------------------------------------------
constexpr int SELECT_WAVES = 4;

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int EC, bool PARTED>
__global__ void __launch_bounds__(SELECT_WAVES * 64) select_kernel(RouterParams p) {
    __shared__ float choice[SELECT_WAVES][EC * 64];
    const int lane = lane_id(), wave = threadIdx.x >> 6, t = blockIdx.x * SELECT_WAVES + wave;
    if (t >= p.T) return;
    const float NEVER = -__builtin_inff();
    float s[EC], c[EC];
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        const int e = lane + 64 * i;
        s[i] = NEVER;
        if (e < p.E) {
            const float *z = p.logits + (size_t)t * p.E + e;
            const size_t part = (size_t)p.T * p.E;
            float v = ldg_f32(z);
            if (PARTED) v = ((v + ldg_f32(z + part)) + ldg_f32(z + 2 * part)) + ldg_f32(z + 3 * part);
            s[i] = p.bias != nullptr ? v + ldg_f32(p.bias + e) : v;
        }
    }
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < EC; ++i) s[i] = 1.0f / (1.0f + expf(-s[i]));
    } else {
        float most = s[0];
#pragma unroll
        for (int i = 1; i < EC; ++i) most = fmaxf(most, s[i]);
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, WAVE));
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < EC; ++i) {
            s[i] = lane + 64 * i < p.E ? expf(s[i] - most) : 0.0f;
            sum += s[i];
        }
        sum = wave_sum(sum);               // a NaN among the logits makes every score one
#pragma unroll
        for (int i = 0; i < EC; ++i) s[i] = s[i] / sum;
    }
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        const int e = lane + 64 * i;
        c[i] = e < p.E ? (p.balance != nullptr ? s[i] + ldg_f32(p.balance + e) : s[i]) : NEVER;
        if (!(c[i] == c[i])) c[i] = NEVER;
    }
    if (p.keep_groups < p.n_groups) {
        // 2^n lanes a group, each the two largest of every 2^n-th expert, then of the lanes
        const int per = p.E / p.n_groups;
        int shift = 0;
        while ((p.n_groups << (shift + 1)) <= 64) ++shift;
        const int group = lane >> shift, sub = lane & ((1 << shift) - 1);
#pragma unroll
        for (int i = 0; i < EC; ++i) choice[wave][lane + 64 * i] = c[i];
        wave_lds_fence();
        float first = NEVER, second = NEVER;
        if (group < p.n_groups)
            for (int j = sub; j < per; j += 1 << shift) {
                const float v = choice[wave][group * per + j];
                second = fmaxf(second, fminf(first, v));
                first = fmaxf(first, v);
            }
        for (int m = 1; m < 1 << shift; m <<= 1) {
            const float f = __shfl_xor(first, m, WAVE), g = __shfl_xor(second, m, WAVE);
            second = fmaxf(fminf(first, f), fmaxf(second, g));
            first = fmaxf(first, f);
        }
        float score = p.group_top == 2 ? first + second : first;
        if (!(score == score)) score = NEVER;
        int better = 0;
        for (int g = 0; g < p.n_groups; ++g) {
            const float other = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, score), g << shift));
            better += (other > score || (other == score && g < group)) ? 1 : 0;
        }
        const unsigned long long kept = __ballot(better < p.keep_groups && group < p.n_groups);
#pragma unroll
        for (int i = 0; i < EC; ++i) {
            const int e = lane + 64 * i;
            if (e < p.E && !(kept >> ((e / per) << shift) & 1)) c[i] = NEVER;
        }
    }
    uint32_t key[EC];                      // 0: never chosen
#pragma unroll
    for (int i = 0; i < EC; ++i) key[i] = c[i] == NEVER ? 0u : float_to_ordered(c[i]);
    int32_t id = -1;
    float w = 0.0f, total = 0.0f;
    for (int k = 0; k < p.K; ++k) {
        uint32_t most = key[0];
#pragma unroll
        for (int i = 1; i < EC; ++i) most = max(most, key[i]);
        most = wave_max_u32(most);
        if (most == 0) break;
        int at = -1;
        float sw = 0.0f;
#pragma unroll
        for (int i = 0; i < EC; ++i) {     // the lowest index of those that hold the maximum
            const unsigned long long who = __ballot(key[i] == most);
            if (at < 0 && who != 0) {
                const int from = __builtin_ctzll(who);
                at = from + 64 * i;
                sw = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, s[i]), from));
                if (lane == from) key[i] = 0;
            }
        }
        if (lane == k) {
            id = at;
            w = sw;
        }
        total += sw;
    }
    if (p.renorm) w = w / (total < 0x1p-126f ? 0x1p-126f : total);
    if (lane < p.K) {
        p.ids[(size_t)t * p.K + lane] = id;
        p.weights[(size_t)t * p.K + lane] = w * p.scale;
    }
}

template <typename L, bool WHOLE>
void launch_product(const RouterParams &p, hipStream_t st) {
    hipLaunchKernelGGL((router_small_kernel<L, WHOLE>), dim3((p.E + 15) / 16, (p.T + 15) / 16), dim3(PARTS * 64), 0, st, p);
}

template <bool PARTED>
void launch_select(const RouterParams &p, hipStream_t st) {
    const dim3 grid((p.T + SELECT_WAVES - 1) / SELECT_WAVES), block(SELECT_WAVES * 64);
    if (p.E <= 64) hipLaunchKernelGGL((select_kernel<1, PARTED>), grid, block, 0, st, p);
    else if (p.E <= 128) hipLaunchKernelGGL((select_kernel<2, PARTED>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((select_kernel<4, PARTED>), grid, block, 0, st, p);
}

constexpr int CHUNK = 16384;             // tokens whose logits lie in the scratch at once

}  // namespace

size_t router_scratch_bytes(int T, int, int E, bool) { return (size_t)(T < CHUNK ? T : CHUNK) * E * 4; }

int launch_route_scored(const RouterParams &all, bool f32, hipStream_t st) {
    const size_t row = (size_t)all.d * (f32 ? 4 : 2);
    const bool whole = row % 16 == 0 && aligned16(all.x) && aligned16(all.w);
    for (int t0 = 0; t0 < all.T; t0 += CHUNK) {
        RouterParams p = all;
        p.T = all.T - t0 < CHUNK ? all.T - t0 : CHUNK;
        p.x = static_cast<const char *>(all.x) + t0 * row;
        p.ids = all.ids + (size_t)t0 * p.K;
        p.weights = all.weights + (size_t)t0 * p.K;
        if (!f32) launch_product<Bf16Line, true>(p, st);
        else if (whole) launch_product<F32Line, true>(p, st);
        else launch_product<F32Line, false>(p, st);
        launch_select<false>(p, st);
    }
    return launch_status(__func__);
}

}  // namespace bm
