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
// The product for many tokens: 128 tokens x EB experts and a quarter (two parts) of the reduction a workgroup of eight waves.
// Whole lines of both operands go straight into a ring of S LDS stages (8 rows an instruction); row r's 16-byte piece c lies at
// slot c ^ (r & 7), by the choice of the piece that a lane fetches: conflict-free reads.  One wait and one barrier a line: its
// stage has landed for every wave, and everybody is done with the stage that takes the next loads.
// Bound by the way from the second-level caches into LDS, whose rate is what is in flight over the time that a load takes: all
// experts in one workgroup, and as many stages as LDS holds.
// ---------------------------------------------------------------------------
#define BM_LDS __attribute__((address_space(3)))
constexpr int TILE_TOKENS = 128, TILE_WAVES = 8;

template <int EB>
struct RouterTile {
    static constexpr int WN = EB == 256 ? 4 : EB >= 64 ? 2 : 1, WM = TILE_WAVES / WN;     // waves along experts and tokens
    static constexpr int TM = TILE_TOKENS / WM / 16, TN = EB / WN / 16;                  // 16 x 16 blocks of a wave
    static constexpr int BLOCKS = (TILE_TOKENS + EB) / 8;                                // of 8 rows
    static constexpr int LOADS = (BLOCKS + TILE_WAVES - 1) / TILE_WAVES;                 // a wave and stage
    static constexpr int STAGES = EB == 128 ? 4 : 3, STAGE = BLOCKS * 64;                // 16-byte pieces of a stage
    static constexpr size_t LDS = (size_t)STAGES * STAGE * 16;
};

template <typename L, int EB>
__global__ void __launch_bounds__(TILE_WAVES * 64, 2) router_tile_kernel(RouterParams p) {
    using R = RouterTile<EB>;
    constexpr int S = R::STAGES, TM = R::TM, TN = R::TN;
    extern __shared__ u32x4 smem[];
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, kq = lane >> 4;
    // workgroups go round the eight dies: two dies a quarter (its columns of the router's matrix stay in their second-level caches),
    // and a tile's tokens with all of the experts one after the other on one die
    const int die = blockIdx.x & 7, turn = blockIdx.x >> 3, quarter = die & 3, part = quarter * 2;
    const int expert_tiles = (p.E + EB - 1) / EB;
    const int e0 = turn % expert_tiles * EB, t0 = (turn / expert_tiles * 2 + (die >> 2)) * TILE_TOKENS;
    if (t0 >= p.T) return;
    const int bytes = p.d * (128 / L::VALUES), lines = (bytes + 127) >> 7;
    const int begin = part * lines / PARTS, middle = (part + 1) * lines / PARTS, end = (part + 2) * lines / PARTS;
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
    if (begin < end) {
#pragma unroll
        for (int i = 0; i < S - 1; ++i) load(begin + i, i);
        int now = 0, free = S - 1;
        for (int l = begin; l < end; ++l) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S - 2) * R::LOADS) : "memory");
            load(l + S - 1, free);
            const u32x4 *st = smem + now * R::STAGE;
            if (l == middle)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        first[i][j] = acc[i][j];
                        acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                    }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 a[TM], b[TN];
                const int c = (h * 4 + kq) ^ (r16 & 7);
#pragma unroll
                for (int i = 0; i < TM; ++i) a[i] = st[(m0 + i * 16 + r16) * 8 + c];
#pragma unroll
                for (int j = 0; j < TN; ++j) b[j] = st[(n0 + j * 16 + r16) * 8 + c];
                if (l * 128 + 128 > bytes) {                             // the row ends in this line
                    const bool in = l * 128 + (h * 4 + kq) * 16 < bytes;
#pragma unroll
                    for (int i = 0; i < TM; ++i) a[i] = in ? a[i] : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < TN; ++j) b[j] = in ? b[j] : u32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = L::mac(a[i], b[j], acc[i][j]);
            }
            free = now;
            now = now + 1 == S ? 0 : now + 1;
        }
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");               // the last loads are through before the workgroup ends
    }
    // (a first part without lines: its sum is the zero that acc starts from)
    float *out = p.logits + (size_t)quarter * p.T * p.E;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int e = e0 + n0 - TILE_TOKENS + j * 16 + r16;
        if (e >= p.E) continue;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int t = t0 + m0 + i * 16 + 4 * kq + v;
                if (t < p.T) out[(size_t)t * p.E + e] = first[i][j][v] + acc[i][j][v];
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

struct Two {                               // the largest and second largest of a set
    float first, second;
    __device__ __forceinline__ void join(float f, float g) {
        second = fmaxf(fminf(first, f), fmaxf(second, g));
        first = fmaxf(first, f);
    }
};

// The lane's value v of EC, from a row of n values at a 4-byte address; whole: n is a multiple of EC and the row is at a multiple of
// EC values
template <int EC>
__device__ __forceinline__ void load_lane(const float *row, int lane, int n, bool whole, float (&v)[EC]) {
    if (EC == 4 && whole) {
        const f32x4 q = *(const BM_GLOBAL f32x4 *)(row + min(lane * 4, n - 4));
#pragma unroll
        for (int i = 0; i < EC; ++i) v[i] = q[i % 4];
    } else {
#pragma unroll
        for (int i = 0; i < EC; ++i) v[i] = ldg_f32(row + min(lane * EC + i, n - 1));
    }
}

template <int EC, int N>
__global__ void __launch_bounds__(SELECT_WAVES * 64) select_kernel(RouterParams p) {
    __shared__ float choice[SELECT_WAVES][EC * 64];
    const int lane = lane_id(), wave = threadIdx.x >> 6, t = blockIdx.x * SELECT_WAVES + wave;
    if (t >= p.T) return;
    const float NEVER = -__builtin_inff();
    const int E = p.E;
    const bool whole = E % 4 == 0;
    float part[N][EC], s[EC], c[EC];
#pragma unroll
    for (int n = 0; n < N; ++n) load_lane<EC>(p.logits + ((size_t)n * p.T + t) * E, lane, E, whole, part[n]);
#pragma unroll
    for (int i = 0; i < EC; ++i) s[i] = c[i] = 0.0f;
    if (p.bias != nullptr) load_lane<EC>(p.bias, lane, E, whole && aligned16(p.bias), s);
    if (p.balance != nullptr) load_lane<EC>(p.balance, lane, E, whole && aligned16(p.balance), c);
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
        for (int i = 0; i < EC; ++i) s[i] = 1.0f / (1.0f + expf(-s[i]));
    } else {
        uint32_t key = 0;                  // (a NaN among the logits makes every score one, by the sum)
#pragma unroll
        for (int i = 0; i < EC; ++i) key = max(key, float_to_ordered(s[i]));
        const float most = ordered_to_float(wave_max_u32(key));
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < EC; ++i) {
            s[i] = lane * EC + i < E ? expf(s[i] - most) : 0.0f;
            sum += s[i];
        }
        sum = row_sum(sum);
#pragma unroll
        for (int i = 0; i < EC; ++i) s[i] = s[i] / sum;
    }
    // choices as ordered integers (0: never chosen), sorted by the lane
    uint32_t key[EC];
    int at[EC];
#pragma unroll
    for (int i = 0; i < EC; ++i) {
        at[i] = lane * EC + i;
        c[i] = s[i] + c[i];
        if (at[i] >= E || !(c[i] == c[i])) c[i] = NEVER;
        key[i] = c[i] == NEVER ? 0u : float_to_ordered(c[i]);
    }
    const bool grouped = p.keep_groups < p.n_groups;
    const int per = E / p.n_groups;
    const int lanes = EC == 1 ? per : per % EC == 0 ? per / EC : 0;
    const bool in_lanes = grouped && lanes > 0 && (lanes & (lanes - 1)) == 0;      // a group is a power of two of lanes
    if (grouped && !in_lanes) {
#pragma unroll
        for (int i = 0; i < EC; ++i) choice[wave][lane * EC + i] = c[i];
    }
#pragma unroll
    for (int pass = 0; pass < EC - 1; ++pass)                                       // (stable: equals stay in order)
#pragma unroll
        for (int i = 0; i < EC - 1 - pass; ++i) {
            const bool swap = key[i + 1] > key[i];
            const uint32_t k0 = key[i];
            const float s0 = s[i];
            const int a0 = at[i];
            key[i] = swap ? key[i + 1] : k0;
            s[i] = swap ? s[i + 1] : s0;
            at[i] = swap ? at[i + 1] : a0;
            key[i + 1] = swap ? k0 : key[i + 1];
            s[i + 1] = swap ? s0 : s[i + 1];
            at[i + 1] = swap ? a0 : at[i + 1];
        }
    if (in_lanes) {
        Two two{key[0] ? ordered_to_float(key[0]) : NEVER, EC > 1 && key[EC > 1] ? ordered_to_float(key[EC > 1]) : NEVER};
        if (lanes > 1) two.join(dpp<0xB1>(0.f, two.first), dpp<0xB1>(0.f, two.second));
        if (lanes > 2) two.join(dpp<0x4E>(0.f, two.first), dpp<0x4E>(0.f, two.second));
        if (lanes > 4) two.join(dpp<0x141>(0.f, two.first), dpp<0x141>(0.f, two.second));
        if (lanes > 8) two.join(dpp<0x140>(0.f, two.first), dpp<0x140>(0.f, two.second));
        if (lanes > 16) two.join(__shfl_xor(two.first, 16, WAVE), __shfl_xor(two.second, 16, WAVE));
        float score = p.group_top == 2 ? two.first + two.second : two.first;
        if (!(score == score)) score = NEVER;
        int better = 0;
        for (int g = 0, l = 0; g < p.n_groups; ++g, l += lanes) {
            const float other = read_lane(score, l);
            better += (other > score || (other == score && l < (lane & -lanes))) ? 1 : 0;
        }
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
        float score = p.group_top == 2 ? two.first + two.second : two.first;
        if (!(score == score)) score = NEVER;
        int better = 0;
        for (int g = 0; g < p.n_groups; ++g) {
            const float other = read_lane(score, g << shift);
            better += (other > score || (other == score && g < group)) ? 1 : 0;
        }
        const unsigned long long kept = __ballot(better < p.keep_groups && group < p.n_groups);
#pragma unroll
        for (int i = 0; i < EC; ++i)
            if (key[i] && !(kept >> ((at[i] / per) << shift) & 1)) key[i] = 0;
        // those that are out move behind the others, which stay in order
#pragma unroll
        for (int pass = 0; pass < EC - 1; ++pass)
#pragma unroll
            for (int i = 0; i < EC - 1 - pass; ++i) {
                const bool swap = key[i] == 0;
                const float s0 = s[i];
                const int a0 = at[i];
                key[i] = swap ? key[i + 1] : key[i];
                s[i] = swap ? s[i + 1] : s[i];
                at[i] = swap ? at[i + 1] : at[i];
                key[i + 1] = swap ? 0u : key[i + 1];
                s[i + 1] = swap ? s0 : s[i + 1];
                at[i + 1] = swap ? a0 : at[i + 1];
            }
    }
    int32_t id = -1;
    float w = 0.0f, total = 0.0f;
    for (int k = 0; k < p.K; ++k) {
        const uint32_t most = wave_max_u32(key[0]);
        if (most == 0) break;
        const int from = __builtin_ctzll(__ballot(key[0] == most));
        const float sw = read_lane(s[0], from);
        const int e = __builtin_amdgcn_readlane(at[0], from);
        total += sw;
        id = lane == k ? e : id;
        w = lane == k ? sw : w;
        if (lane == from) {
#pragma unroll
            for (int i = 0; i < EC; ++i) {
                key[i] = i + 1 < EC ? key[(i + 1) % EC] : 0u;
                s[i] = s[(i + 1) % EC];
                at[i] = at[(i + 1) % EC];
            }
        }
    }
    if (p.renorm) w = w / (total < 0x1p-126f ? 0x1p-126f : total);
    if (lane < p.K) {
        p.ids[(size_t)t * p.K + lane] = id;
        p.weights[(size_t)t * p.K + lane] = w * p.scale;
    }
}

template <int N>
void launch_select(const RouterParams &p, hipStream_t st) {
    const dim3 grid((p.T + SELECT_WAVES - 1) / SELECT_WAVES), block(SELECT_WAVES * 64);
    if (p.E <= 64) hipLaunchKernelGGL((select_kernel<1, N>), grid, block, 0, st, p);
    else if (p.E <= 128) hipLaunchKernelGGL((select_kernel<2, N>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((select_kernel<4, N>), grid, block, 0, st, p);
}

template <typename L, int EB>
void launch_tile(const RouterParams &p, hipStream_t st) {
    const int pairs = (p.T + 2 * TILE_TOKENS - 1) / (2 * TILE_TOKENS);     // of token tiles: one for each half of the dies
    hipLaunchKernelGGL((router_tile_kernel<L, EB>), dim3((p.E + EB - 1) / EB * pairs * 8), dim3(TILE_WAVES * 64), RouterTile<EB>::LDS, st, p);
}

template <typename L>
void launch_tiles(const RouterParams &p, hipStream_t st) {
    if (p.E <= 32) launch_tile<L, 32>(p, st);
    else if (p.E <= 64) launch_tile<L, 64>(p, st);
    else if (p.E <= 128) launch_tile<L, 128>(p, st);
    else launch_tile<L, 256>(p, st);
}

constexpr int CHUNK = 16384;             // tokens whose logits lie in the scratch at once
constexpr int TILED_FROM = 1024;

}  // namespace

// A larger batch needs no less: eight parts of each logit of a small batch, four of a large one
size_t router_scratch_bytes(int T, int E) {
    const size_t few = (size_t)(T < TILED_FROM - 1 ? T : TILED_FROM - 1) * PARTS, many = (size_t)(T < CHUNK ? T : CHUNK) * (PARTS / 2);
    return (few > many ? few : many) * E * 4;
}

int launch_route_scored(const RouterParams &all, bool f32, hipStream_t st) {
    const size_t row = (size_t)all.d * (f32 ? 4 : 2);
    const bool whole = row % 16 == 0 && aligned16(all.x) && aligned16(all.w);
    // (rows of other lengths and addresses: the product for few tokens, as many at a time as the scratch has room for)
    const int chunk = whole ? CHUNK : (int)(router_scratch_bytes(all.T, all.E) / ((size_t)PARTS * all.E * 4));
    for (int t0 = 0; t0 < all.T; t0 += chunk) {
        RouterParams p = all;
        p.T = all.T - t0 < chunk ? all.T - t0 : chunk;
        p.x = static_cast<const char *>(all.x) + t0 * row;
        p.ids = all.ids + (size_t)t0 * p.K;
        p.weights = all.weights + (size_t)t0 * p.K;
        const dim3 grid((p.E + 15) / 16, (p.T + 15) / 16, PARTS), block(64);
        if (whole && all.T >= TILED_FROM) {
            if (f32) launch_tiles<F32Line>(p, st);
            else launch_tiles<Bf16Line>(p, st);
            launch_select<PARTS / 2>(p, st);
            continue;
        }
        if (!f32) hipLaunchKernelGGL((router_small_kernel<Bf16Line, true>), grid, block, 0, st, p);
        else if (whole) hipLaunchKernelGGL((router_small_kernel<F32Line, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((router_small_kernel<F32Line, false>), grid, block, 0, st, p);
        launch_select<PARTS>(p, st);
    }
    return launch_status(__func__);
}

}  // namespace bm
