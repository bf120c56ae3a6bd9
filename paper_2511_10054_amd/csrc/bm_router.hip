// Routing by softmax or sigmoid scores with a balance bias and groups of experts.
//
//   z = x W^T + bias,  s = softmax(z) or sigmoid(z),  c = s + balance
// A group's score is the sum of its one or two largest c; the experts of the best groups stay, of those the K of largest c
// are chosen, and their s - without the balance - become the weights.
//
// Two launches: the product writes parts of the logits (fp32, they stay in the memory-side cache), then a wave a token
// adds them, scores, ranks and weighs.  The order of a logit's additions follows from d alone: eight parts of the reduction (whole
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
        typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
        u32x4 v = {0, 0, 0, 0};
        if (at + 16 <= bytes) {
            v = *(const BM_GLOBAL u32x4_at4 *)(row + at);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const int b = at + 4 * i;
                if (b < bytes) v[i] = (uint32_t)ldg_i32(row + b);
            }
        }
        return v;
    }
}

// ---------------------------------------------------------------------------
// The product for few tokens: a wave takes 16 tokens x 16 experts and one eighth of the reduction, with the loads of up to
// eight lines in flight.  Bound by latency: a wave a workgroup spreads the router's matrix over the most units (at 1 token, 4096 ->
// 256, 2 MB over 128 of them).
// ---------------------------------------------------------------------------
template <typename L, bool WHOLE>
__global__ void __launch_bounds__(64) router_small_kernel(RouterParams p) {
    const int lane = threadIdx.x, r16 = lane & 15, kq = lane >> 4;
    const int e0 = blockIdx.x * 16, t0 = blockIdx.y * 16, part = blockIdx.z;
    const int bytes = p.d * (128 / L::VALUES), lines = (bytes + 127) >> 7;
    const char *xr = static_cast<const char *>(p.x) + (size_t)min(t0 + r16, p.T - 1) * bytes;
    const char *wr = static_cast<const char *>(p.w) + (size_t)min(e0 + r16, p.E - 1) * bytes;
    const int begin = part * lines / PARTS, end = (part + 1) * lines / PARTS;
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
    const int e = e0 + r16;
    if (e >= p.E) return;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int t = t0 + 4 * kq + v;
        if (t < p.T) p.logits[((size_t)part * p.T + t) * p.E + e] = acc[v];
    }
}

// ---------------------------------------------------------------------------
// The product for many tokens: 128 tokens x EB experts and TAKE of the eight parts of the reduction a workgroup of eight waves.
// Whole lines of both operands go straight into a ring of S LDS stages (8 rows an instruction); row r's 16-byte piece c lies at
// slot c ^ (r & 7), by the choice of the piece that a lane fetches: conflict-free reads.  One wait and one barrier a line: its
// stage has landed for every wave, and everybody is done with the stage that takes the next loads.
// Bound by the way from the second-level caches into LDS, whose rate is what is in flight over the time that a load takes: all
// experts in one workgroup, and as many stages as LDS holds.
// ---------------------------------------------------------------------------
#define BM_LDS __attribute__((address_space(3)))
constexpr int TILE_TOKENS = 128, TILE_WAVES = 8;
constexpr int LGKM0 = 0xc07f;            // s_waitcnt lgkmcnt(0), the other counters at their most

template <int EB>
struct RouterTile {
    static constexpr int WN = EB == 256 ? 4 : EB >= 64 ? 2 : 1, WM = TILE_WAVES / WN;     // waves along experts and tokens
    static constexpr int TM = TILE_TOKENS / WM / 16, TN = EB / WN / 16;                  // 16 x 16 blocks of a wave
    static constexpr int BLOCKS = (TILE_TOKENS + EB) / 8;                                // of 8 rows
    static constexpr int LOADS = (BLOCKS + TILE_WAVES - 1) / TILE_WAVES;                 // a wave and stage
    static constexpr int STAGES = EB == 128 ? 4 : 3, STAGE = BLOCKS * 64;                // 16-byte pieces of a stage
    static constexpr size_t LDS = (size_t)STAGES * STAGE * 16;
};

template <typename L, int EB, int TAKE>
__global__ void __launch_bounds__(TILE_WAVES * 64, 2) router_tile_kernel(RouterParams p) {
    using R = RouterTile<EB>;
    constexpr int S = R::STAGES, TM = R::TM, TN = R::TN;
    extern __shared__ u32x4 smem[];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, kq = lane >> 4;
    // Workgroups go round the eight dies: a die (two dies) for an eighth (a quarter) of the reduction, whose columns of the router's
    // matrix stay in its second-level cache, and a tile's tokens with all of the experts one after the other on one die
    constexpr int SLICES = PARTS / TAKE;
    const int die = blockIdx.x & 7, turn = blockIdx.x >> 3, slice = die % SLICES, part = slice * TAKE;
    const int expert_tiles = (p.E + EB - 1) / EB;
    const int e0 = turn % expert_tiles * EB, t0 = (turn / expert_tiles * TAKE + die / SLICES) * TILE_TOKENS;
    if (t0 >= p.T) return;
    const int bytes = p.d * (128 / L::VALUES), lines = (bytes + 127) >> 7;
    const int begin = part * lines / PARTS, middle = (part + 1) * lines / PARTS, end = (part + TAKE) * lines / PARTS;
    const char *from[R::LOADS];
    int to[R::LOADS], piece_at;
#pragma unroll
    for (int j = 0; j < R::LOADS; ++j) {
        int block = wave + TILE_WAVES * j;
        if (block >= R::BLOCKS) block = wave % R::BLOCKS;                // (a repeated load of what is there)
        const int row = block * 8 + (lane >> 3);
        from[j] = row < TILE_TOKENS ? static_cast<const char *>(p.x) + (size_t)min(t0 + row, p.T - 1) * bytes
                                    : static_cast<const char *>(p.w) + (size_t)min(e0 + row - TILE_TOKENS, p.E - 1) * bytes;
        to[j] = block * 64;
    }
    piece_at = ((lane & 7) ^ (lane >> 3)) * 16;
    auto load = [&](int l, int slot) {
        const int at = min(l, end - 1) * 128 + piece_at, within = at < bytes ? at : 0;   // (behind a row's end: cleared when read)
#pragma unroll
        for (int j = 0; j < R::LOADS; ++j)
            __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)(from[j] + within), (BM_LDS void *)(smem + slot * R::STAGE + to[j]), 16, 0, 0);
    };
    const int m0 = wave % R::WM * (TM * 16), n0 = TILE_TOKENS + wave / R::WM * (TN * 16);
    f32x4 acc[TM][TN], first[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = first[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Fragments of the two halves of a line: those of one are read while the other's are multiplied.  Between the halves stand a wait and
    // a barrier: the next line has landed for every wave, and this one's reads are done - its stage takes new loads.
    u32x4 a[2][TM], b[2][TN];
    int now = 0;
    auto read = [&](int h) {
        const u32x4 *st = smem + now * R::STAGE;
        const int c = (h * 4 + kq) ^ (r16 & 7);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[h][i] = st[(m0 + i * 16 + r16) * 8 + c];
#pragma unroll
        for (int j = 0; j < TN; ++j) b[h][j] = st[(n0 + j * 16 + r16) * 8 + c];
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](int h) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = L::mac(a[h][i], b[h][j], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // (The waits for LDS by the builtin, which the compiler knows: left to itself it has every half wait for the other half's reads too.)
    auto line = [&](int l) {
        __builtin_amdgcn_s_waitcnt(LGKM0);
        read(1);
        multiply(0);
        __builtin_amdgcn_s_waitcnt(LGKM0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S - 2) * R::LOADS) : "memory");
        load(l + S, now);
        now = now + 1 == S ? 0 : now + 1;
        read(0);
        multiply(1);
    };
    if (begin < end) {
#pragma unroll
        for (int i = 0; i < S; ++i) load(begin + i, i);
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((S - 1) * R::LOADS) : "memory");
        read(0);
        int l = begin;
        for (; l < min(middle, end - 1); ++l) line(l);
        if (TAKE == 2 && middle < end) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    first[i][j] = acc[i][j];
                    acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            for (; l < end - 1; ++l) line(l);
        }
        read(1);
        if (l * 128 + 128 > bytes) {                                     // the row ends in the last line
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = l * 128 + (h * 4 + kq) * 16 < bytes;
#pragma unroll
                for (int i = 0; i < TM; ++i) a[h][i] = in ? a[h][i] : u32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < TN; ++j) b[h][j] = in ? b[h][j] : u32x4{0, 0, 0, 0};
            }
        }
        multiply(0);
        multiply(1);
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");               // the last loads are through before the workgroup ends
    }
    // (a first part without lines: its sum is the zero that acc starts from)
    float *out = p.logits + (size_t)slice * p.T * p.E;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int e = e0 + n0 - TILE_TOKENS + j * 16 + r16;
        if (e >= p.E) continue;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int t = t0 + m0 + i * 16 + 4 * kq + v;
                if (t < p.T) out[(size_t)t * p.E + e] = TAKE == 2 ? first[i][j][v] + acc[i][j][v] : acc[i][j][v];
            }
    }
}

// ---------------------------------------------------------------------------
// Scores, groups, choice and weights: a wave a token, lane l holds the EC experts from l * EC on, sorted by falling choice, so
// that a round of the top-k looks at one value a lane and the lowest lane of equals holds the lowest expert.
// N: parts of the logits, the 8 of the reduction or its 4 quarters.
// ---------------------------------------------------------------------------
constexpr int SELECT_WAVES = 4;

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp(float old, float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float read_lane(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// Sum over the wave: inside rows of 16 lanes, then row by row into lane 63
__device__ __forceinline__ float row_sum(float v) {
    v += dpp<0xB1>(0.0f, v);               // lane ^ 1
    v += dpp<0x4E>(0.0f, v);               // lane ^ 2
    v += dpp<0x141>(0.0f, v);              // mirror inside a half row
    v += dpp<0x140>(0.0f, v);              // mirror inside the row
    v += dpp<0x142, 0xA>(0.0f, v);         // rows 1 and 3 get the row before
    v += dpp<0x143, 0xC>(0.0f, v);         // rows 2 and 3 get lane 31
    return read_lane(v, 63);
}

// e^x: 2^(x log2 e) with the rest of the product, which the instruction's argument has no room for (at 87 up to 63 * 2^-24 of the result).
// From 128 on the instruction gives infinity, or zero, and the rest of an infinity is no number.
__device__ __forceinline__ float exponential(float x) {
    const float hi = x * 0x1.715476p+0f, lo = fmaf(x, 0x1.715476p+0f, -hi) + x * 0x1.4ae0c0p-26f;    // log2 e in two parts
    const float e = __builtin_amdgcn_exp2f(hi);
    return fabsf(hi) < 128.0f ? fmaf(e, lo * 0x1.62e430p-1f, e) : e;                                 // 2^lo = 1 + lo log 2
}

struct Two {                               // the largest and second largest of a set
    float first, second;
    __device__ __forceinline__ void join(float f, float g) {
        second = fmaxf(fminf(first, f), fmaxf(second, g));
        first = fmaxf(first, f);
    }
};

// How many groups come before the one that starts at the lane `mine`, `lanes` lanes a group that all hold its two largest
__device__ __forceinline__ int better_groups(const RouterParams &p, const Two &two, int lanes, int mine) {
    float score = p.group_top == 2 ? two.first + two.second : two.first;
    if (!(score == score)) score = -__builtin_inff();
    int better = 0;
    for (int g = 0, l = 0; g < p.n_groups; ++g, l += lanes) {
        const float other = read_lane(score, l);
        better += (other > score || (other == score && l < mine)) ? 1 : 0;
    }
    return better;
}

// The lane's EC values of each part of a token's logits, of the bias and of the balance.  One branch for all of the loads: with one for
// each array the compiler has a load wait for those before.
template <int EC, int N, bool WHOLE>
__device__ __forceinline__ void load_lane(const RouterParams &p, int t, int lane, float (&part)[N][EC], float (&bias)[EC], float (&balance)[EC]) {
    const int E = p.E;
    const float *z = p.logits + (size_t)t * E;
    auto load = [&](const float *row, float (&v)[EC]) {
        if constexpr (WHOLE) {             // E is a multiple of 4, and rows are at 16-byte addresses
            const f32x4 q = *(const BM_GLOBAL f32x4 *)(row + min(lane * 4, E - 4));
#pragma unroll
            for (int i = 0; i < EC; ++i) v[i] = q[i % 4];
        } else {
#pragma unroll
            for (int i = 0; i < EC; ++i) v[i] = ldg_f32(row + min(lane * EC + i, E - 1));
        }
    };
#pragma unroll
    for (int n = 0; n < N; ++n) load(z + (size_t)n * p.T * E, part[n]);
    load(p.bias != nullptr ? p.bias : z, bias);            // (of none: values that are not used)
    load(p.balance != nullptr ? p.balance : z, balance);
}

template <int EC, int N>
__global__ void __launch_bounds__(SELECT_WAVES * 64) select_kernel(RouterParams p) {
    __shared__ float choice[SELECT_WAVES][EC * 64], score[SELECT_WAVES][EC * 64];
    const int lane = lane_id(), wave = threadIdx.x >> 6, t = blockIdx.x * SELECT_WAVES + wave;
    if (t >= p.T) return;
    const float NEVER = -__builtin_inff();
    const int E = p.E;
    float part[N][EC], s[EC], c[EC];
    if (EC == 4 && E % 4 == 0 && aligned16(p.bias) && aligned16(p.balance)) load_lane<EC, N, EC == 4>(p, t, lane, part, s, c);
    else load_lane<EC, N, false>(p, t, lane, part, s, c);
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        s[i] = p.bias != nullptr ? s[i] : 0.0f;
        c[i] = p.balance != nullptr ? c[i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        float q[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = N == 8 ? part[N / 4 * j][i] + part[N / 4 * j + N / 4 - 1][i] : part[N / 4 * j][i];
        const float z = ((q[0] + q[1]) + q[2]) + q[3];
        s[i] = lane * EC + i < E ? z + s[i] : NEVER;
    }
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < EC; ++i) s[i] = __builtin_amdgcn_rcpf(1.0f + exponential(-s[i]));
    } else {
        uint32_t key = 0;                  // (a NaN among the logits makes every score one, by the sum)
#pragma unroll
        for (int i = 0; i < EC; ++i) key = max(key, float_to_ordered(s[i]));
        const float most = ordered_to_float(wave_max_u32(key));
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < EC; ++i) {
            s[i] = lane * EC + i < E ? exponential(s[i] - most) : 0.0f;
            sum += s[i];
        }
        const float inv = 1.0f / row_sum(sum);
#pragma unroll
        for (int i = 0; i < EC; ++i) s[i] *= inv;
    }
    // choices as ordered integers (0: never chosen), sorted by the lane; order: which of its experts, a byte each
    uint32_t key[EC], order = 0;
    int at[EC];
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        at[i] = i;
        c[i] = s[i] + c[i];
        if (lane * EC + i >= E || !(c[i] == c[i])) c[i] = NEVER;
        key[i] = c[i] == NEVER ? 0u : float_to_ordered(c[i]);
        score[wave][lane * EC + i] = s[i];
    }
    const bool grouped = p.keep_groups < p.n_groups;
    const int per = p.per_group, lanes = p.lanes_per_group;                         // lanes: 0, or a power of two that holds a group
    if (grouped && lanes == 0) {
#pragma unroll
        for (int i = 0; i < EC; ++i) choice[wave][lane * EC + i] = c[i];
    }
#pragma unroll
    for (int pass = 0; pass < EC - 1; ++pass)                                       // (stable: equals stay in order)
#pragma unroll
        for (int i = 0; i < EC - 1 - pass; ++i) {
            const bool swap = key[i + 1] > key[i];
            const uint32_t k0 = key[i];
            const int a0 = at[i];
            key[i] = swap ? key[i + 1] : k0;
            at[i] = swap ? at[i + 1] : a0;
            key[i + 1] = swap ? k0 : key[i + 1];
            at[i + 1] = swap ? a0 : at[i + 1];
        }
    if (grouped && lanes > 0) {
        Two two{key[0] ? ordered_to_float(key[0]) : NEVER, EC > 1 && key[EC > 1] ? ordered_to_float(key[EC > 1]) : NEVER};
        if (lanes > 1) two.join(dpp<0xB1>(0.f, two.first), dpp<0xB1>(0.f, two.second));
        if (lanes > 2) two.join(dpp<0x4E>(0.f, two.first), dpp<0x4E>(0.f, two.second));
        if (lanes > 4) two.join(dpp<0x141>(0.f, two.first), dpp<0x141>(0.f, two.second));
        if (lanes > 8) two.join(dpp<0x140>(0.f, two.first), dpp<0x140>(0.f, two.second));
        if (lanes > 16) two.join(__shfl_xor(two.first, 16, WAVE), __shfl_xor(two.second, 16, WAVE));
        const int better = better_groups(p, two, lanes, lane & -lanes);
#pragma unroll
        for (int i = 0; i < EC; ++i) key[i] = better < p.keep_groups ? key[i] : 0u;
    } else if (grouped) {
        // any sizes: 2^n lanes a group, each the two largest of every 2^n-th expert, then of the lanes
        int shift = 0;
        while ((p.n_groups << (shift + 1)) <= 64) ++shift;
        const int group = lane >> shift, sub = lane & ((1 << shift) - 1);
        wave_lds_fence();
        Two two{NEVER, NEVER};
        if (group < p.n_groups)
            for (int j = sub; j < per; j += 1 << shift) two.join(choice[wave][group * per + j], NEVER);
        for (int m = 1; m < 1 << shift; m <<= 1) two.join(__shfl_xor(two.first, m, WAVE), __shfl_xor(two.second, m, WAVE));
        const int better = better_groups(p, two, 1 << shift, group << shift);
        const unsigned long long kept = __ballot(better < p.keep_groups && group < p.n_groups);
#pragma unroll
        for (int i = 0; i < EC; ++i)
            if (key[i] && !(kept >> (((lane * EC + at[i]) / per) << shift) & 1)) key[i] = 0;
        // those that are out move behind the others, which stay in order
#pragma unroll
        for (int pass = 0; pass < EC - 1; ++pass)
#pragma unroll
            for (int i = 0; i < EC - 1 - pass; ++i) {
                const bool swap = key[i] == 0;
                const int a0 = at[i];
                key[i] = swap ? key[i + 1] : key[i];
                at[i] = swap ? at[i + 1] : at[i];
                key[i + 1] = swap ? 0u : key[i + 1];
                at[i + 1] = swap ? a0 : at[i + 1];
            }
    }
#pragma unroll
    for (int i = 0; i < EC; ++i) order |= (uint32_t)at[i] << 8 * i;
    int id = -1;                           // of slot `lane`
    for (int k = 0; k < p.K; ++k) {
        const uint32_t most = wave_max_u32(key[0]);
        if (most == 0) break;
        const int from = __builtin_ctzll(__ballot(key[0] == most));
        const int e = EC == 1 ? from : from * EC + (__builtin_amdgcn_readlane((int)order, from) & 0xff);
        id = lane == k ? e : id;
        if (lane == from) {
#pragma unroll
            for (int i = 0; i < EC; ++i) key[i] = i + 1 < EC ? key[(i + 1) % EC] : 0u;
            order >>= 8;
        }
    }
    wave_lds_fence();
    float w = id >= 0 ? score[wave][id] : 0.0f;
    if (p.renorm) {
        const float total = row_sum(w);
        w = w / (total < 0x1p-126f ? 0x1p-126f : total);
    }
    if (lane < p.K) {
        p.ids[(size_t)t * p.K + lane] = id;
        p.weights[(size_t)t * p.K + lane] = w * p.scale;
    }
}

template <int N>
void launch_select(RouterParams p, hipStream_t st) {
    p.per_group = p.E / p.n_groups;
    const int ec = p.E <= 64 ? 1 : p.E <= 128 ? 2 : 4, lanes = p.per_group % ec == 0 ? p.per_group / ec : 0;
    p.lanes_per_group = (lanes & (lanes - 1)) == 0 ? lanes : 0;
    const dim3 grid((p.T + SELECT_WAVES - 1) / SELECT_WAVES), block(SELECT_WAVES * 64);
    if (p.E <= 64) hipLaunchKernelGGL((select_kernel<1, N>), grid, block, 0, st, p);
    else if (p.E <= 128) hipLaunchKernelGGL((select_kernel<2, N>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((select_kernel<4, N>), grid, block, 0, st, p);
}

template <typename L, int EB, int TAKE>
void launch_tile(const RouterParams &p, hipStream_t st) {
    const int tiles = (p.T + TILE_TOKENS * TAKE - 1) / (TILE_TOKENS * TAKE);      // of each die
    hipLaunchKernelGGL((router_tile_kernel<L, EB, TAKE>), dim3((p.E + EB - 1) / EB * tiles * 8), dim3(TILE_WAVES * 64), RouterTile<EB>::LDS, st, p);
}

constexpr int CHUNK = 16384;             // tokens whose logits lie in the scratch at once

// From how many logits on the product is tiled: small | tiled product, us of the whole call.  bf16: 4096 -> 256 experts at 32 / 64 / 128 / 256
// tokens 7.3 8.2 10.2 14.2 | 8.7 8.8 9.0 9.7, 2048 -> 128 at 64 / 128 / 256 6.6 7.7 9.9 | 7.1 7.5 8.0, 2048 -> 64 at 128 / 256 / 512
// 6.1 7.1 9.1 | 6.7 7.0 7.4, 4096 -> 8 at 1024 / 2048 6.8 8.8 | 7.6 7.8.  fp32: 2048 -> 256 at 128 / 256 10.7 14.8 | 12.1 12.8,
// 2048 -> 128 at 256 / 512 10.5 14.6 | 11.9 12.8, 1440 -> 60 at 512 / 1024 9.3 13.7 | 9.7 10.3.  The lines by logits alone: at the bf16 one
// 4096 -> 256 (64 tokens) loses 0.6 us, 2048 -> 128, 2048 -> 64 and 4096 -> 8 win 0.2 to 1.0.  Rows or arrays off 16-byte addresses have no
// tiled product: fp32, 1000 / 2048 tokens, 2047 -> 256 40 71 (2048 -> 256: 21 34), 1443 -> 60 12.3 19.1 (1440 -> 60: 10.1 11.5).
bool wants_tiles(int T, int E, bool f32) { return (long long)T * E >= (f32 ? 40960 : 16384); }

// A tiled product's workgroup takes one of the eight parts of the reduction, or of large batches two: half of the parts to write and to
// read, but half of the workgroups.  One | two, us: 4096 -> 256 at 1024 / 2048 / 4096 tokens 14.2 20.5 26.7 | 23.3 25.5 31.0,
// 4096 -> 8 at 4096 9.4 | 13.6; fewer lines: 2048 -> 128 at 2048 / 4096 12.5 19.1 | 13.3 14.9, 2048 -> 64 9.2 12.6 | 9.4 10.7;
// fp32: 2048 -> 128 at 4096 32.1 | 46.8, 1440 -> 60 16.9 | 20.8.
constexpr int EIGHTHS = 4096;
bool by_eighths(int T, int lines, bool f32) { return T <= (f32 || lines >= 64 ? EIGHTHS : EIGHTHS / 2); }

// All experts in one workgroup, or fewer where that leaves units idle
template <typename L>
void launch_tiles(const RouterParams &p, bool eighths, hipStream_t st) {
    const int tiles = (p.T + TILE_TOKENS - 1) / TILE_TOKENS;
    if (!eighths) {
        if (p.E <= 32) launch_tile<L, 32, 2>(p, st);
        else if (p.E <= 64) launch_tile<L, 64, 2>(p, st);
        else if (p.E <= 128) launch_tile<L, 128, 2>(p, st);
        else launch_tile<L, 256, 2>(p, st);
        return;
    }
    auto fits = [&](int eb) { return p.E <= eb || tiles * ((p.E + eb - 1) / eb) * 8 <= 256; };
    if (fits(32)) launch_tile<L, 32, 1>(p, st);
    else if (fits(64)) launch_tile<L, 64, 1>(p, st);
    else if (fits(128)) launch_tile<L, 128, 1>(p, st);
    else launch_tile<L, 256, 1>(p, st);
}

}  // namespace

// A larger batch needs no less: eight parts of each logit of a small batch, four of a large one
size_t router_scratch_bytes(int T, int E) {
    const size_t few = (size_t)(T < EIGHTHS ? T : EIGHTHS) * PARTS, many = (size_t)(T < CHUNK ? T : CHUNK) * (PARTS / 2);
    return (few > many ? few : many) * E * 4;
}

int launch_route_scored(const RouterParams &all, bool f32, hipStream_t st) {
    const size_t row = (size_t)all.d * (f32 ? 4 : 2);
    const bool whole = row % 16 == 0 && aligned16(all.x) && aligned16(all.w);
    const bool tiled = whole && wants_tiles(all.T, all.E, f32), eighths = !tiled || by_eighths(all.T, (int)((row + 127) / 128), f32);
    // as many tokens at a time as the scratch has room for
    const int chunk = (int)(router_scratch_bytes(all.T, all.E) / ((size_t)(eighths ? PARTS : PARTS / 2) * all.E * 4));
    for (int t0 = 0; t0 < all.T; t0 += chunk) {
        RouterParams p = all;
        p.T = all.T - t0 < chunk ? all.T - t0 : chunk;
        p.x = static_cast<const char *>(all.x) + t0 * row;
        p.ids = all.ids + (size_t)t0 * p.K;
        p.weights = all.weights + (size_t)t0 * p.K;
        if (tiled) {
            if (f32) launch_tiles<F32Line>(p, eighths, st);
            else launch_tiles<Bf16Line>(p, eighths, st);
            if (eighths) launch_select<PARTS>(p, st);
            else launch_select<PARTS / 2>(p, st);
            continue;
        }
        const dim3 grid((p.E + 15) / 16, (p.T + 15) / 16, PARTS), block(64);
        if (!f32) hipLaunchKernelGGL((router_small_kernel<Bf16Line, true>), grid, block, 0, st, p);
        else if (whole) hipLaunchKernelGGL((router_small_kernel<F32Line, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((router_small_kernel<F32Line, false>), grid, block, 0, st, p);
        launch_select<PARTS>(p, st);
    }
    return launch_status(__func__);
}

}  // namespace bm
