// Grouped products of 8-bit rows with 8-bit matrices, a 32-bit scale for each 128 values of a row and for each 128 x 128
// block of a matrix:
//   c[i][n] = sum_kb sa[i][kb] * sw[n / 128][kb] * sum_{k in block kb} a[i][k] * w[n][k]
// The inner sum is one v_mfma_f32_16x16x128 (its 128 products are exact, its sum is held in 32 bits); the outer one is a
// fused multiply-add per value in 32 bits.  Weights are the matrix instruction's row operand and tokens its column
// operand, so that a lane's four results belong to one token and a block of weights: one scale for all four.
#include "bm_products.h"

namespace bm {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Eight e4m3 values as fp16 (exact: three mantissa bits, exponents down to 2^-9)
__device__ __forceinline__ f16x8 widen8(int a, int b) {
    const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// A lane's 32 values of a block of 128: as they are, or as fp16
template <bool WIDE> struct Operand;
template <> struct Operand<false> {
    i32x8 v;
    __device__ __forceinline__ void set(i32x8 x) { v = x; }
};
template <> struct Operand<true> {
    f16x8 v[4];
    __device__ __forceinline__ void set(i32x8 x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = widen8(x[2 * i], x[2 * i + 1]);
    }
};
__device__ __forceinline__ f32x4 block_product(const Operand<false> &a, const Operand<false> &b) {
    const f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, z, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 block_product(const Operand<true> &a, const Operand<true> &b) {
    f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) r = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[i], b.v[i], r, 0, 0, 0);
    return r;
}

#define BM_LDS __attribute__((address_space(3)))
// At most n direct loads of this wave are still in flight and its LDS accesses are done; then all waves meet.
// (s_waitcnt of gfx9: vmcnt[3:0] | expcnt 7 << 4 | lgkmcnt 0 << 8 | vmcnt[5:4] << 14)
#define BM_WAIT_AND_MEET(n)                                                             \
    {                                                                                   \
        __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (((n) >> 4) << 14));         \
        asm volatile("s_barrier" ::: "memory");                                         \
    }

// One workgroup's tile: rows [row0, row0 + BM) of a group that ends at row_end, columns [n0, ..).
struct Tile {
    int group, row0, row_end, nt;
};

// Which tile a workgroup has.  Tiles are numbered group by group, inside a group by column tile and then by row tile
// (neighbours share their weights), and each XCD takes a contiguous share: workgroups go round-robin to the XCDs.  Every
// wave derives the groups' tile counts itself from the offsets (clamped: whatever they hold, no tile leaves the rows).
template <int BM>
__device__ __forceinline__ bool find_tile(const ProductParams &p, int n_nt, Tile &t) {
    const int lane = lane_id();
    constexpr int CH = (BM_MAX_E + 8 + WAVE - 1) / WAVE;
    int lo[CH], hi[CH], first[CH], total = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int g = c * WAVE + lane;
        lo[c] = hi[c] = 0;
        if (g < p.n_groups) {
            lo[c] = p.offsets ? min(max(ldg_i32(p.offsets + g), 0), p.rows) : 0;
            hi[c] = p.offsets ? min(max(ldg_i32(p.offsets + g + 1), lo[c]), p.rows) : p.rows;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        first[c] = total;
        if (c * WAVE < p.n_groups) {
            const int mine = (hi[c] - lo[c] + BM - 1) / BM;
            int sum = mine;
#pragma unroll
            for (int s = 1; s < WAVE; s <<= 1) {
                const int o = __shfl_up(sum, s, WAVE);
                sum += lane >= s ? o : 0;
            }
            first[c] = total + sum - mine;
            total += __builtin_amdgcn_readlane(sum, WAVE - 1);
        }
    }
    const long long tiles = (long long)total * n_nt, per_xcd = (tiles + 7) >> 3;
    const long long lid = (long long)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((long long)(blockIdx.x >> 3) >= per_xcd || lid >= tiles) return false;
    const int m = (int)(lid / n_nt);           // the row tiles before it belong to whole groups before it
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int n = (hi[c] - lo[c] + BM - 1) / BM;
        const unsigned long long hit = __ballot(n > 0 && first[c] <= m && m < first[c] + n);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            const int f = __builtin_amdgcn_readlane(first[c], src), nn = __builtin_amdgcn_readlane(n, src);
            const int in = (int)(lid - (long long)f * n_nt);
            t.group = c * WAVE + src;
            t.nt = in / nn;
            t.row0 = __builtin_amdgcn_readlane(lo[c], src) + (in % nn) * BM;
            t.row_end = __builtin_amdgcn_readlane(hi[c], src);
            return true;
        }
    }
    return false;
}

}  // namespace

// BM tokens x BN weight rows (DUAL: BN / 2 of the gate, BN / 2 of the up matrix) per workgroup of NW waves, WNN of them along
// the weight rows.  Steps of 128 along the reduction go through a ring of S stages in LDS, filled with direct loads (a row's
// 128 bytes are one cache line; 8 rows an instruction).  Piece p of row r lies in slot p ^ ((r >> 1) & 7), so that the 16
// rows of an operand read fall into different banks.
template <int BM, int BN, int NW, int WNN, int S, bool DUAL, bool WIDE>
__global__ void __launch_bounds__(NW * 64) product_kernel(ProductParams p) {
    constexpr int WMN = NW / WNN;
    constexpr int TB = BM / WMN / 16, WB = BN / WNN / 16;      // 16-token and 16-row blocks of a wave
    constexpr int HB = DUAL ? WB / 2 : WB;                     // of these, blocks of different columns
    constexpr int COLS = DUAL ? BN / 2 : BN;
    constexpr int WI = BN / NW / 8;                            // weight loads of a wave and stage
    constexpr int TR = BM / NW, TI = TR >= 8 ? TR / 8 : 1;     // token rows and loads of a wave and stage
    constexpr int PER = WI + TI + 1;                           // with the tokens' scales
    constexpr int STAGE = (BN + BM) * 128;
    static_assert(WI * 8 * NW == BN && TB * 16 * WMN == BM && WB * 16 * WNN == BN && (TR >= 8 ? TR % 8 == 0 : TR > 0), "tile shape");
    static_assert(!DUAL || COLS == SCALE_BLOCK, "a tile quantizes whole blocks");
    static_assert((S - 2) * PER < 64, "the wait counts up to 63 loads");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[S * STAGE];
    __shared__ float s_sa[S * BM];
    __shared__ float s_sw[DUAL ? 2 : (BN + SCALE_BLOCK - 1) / SCALE_BLOCK + 1][MAX_PRODUCT_KD / SCALE_BLOCK];
    __shared__ float s_amax[DUAL ? WNN : 1][DUAL ? BM : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WNN, wn = wave % WNN;
    const int q4 = lane >> 4, l16 = lane & 15;
    const int N = p.N, Kd = p.Kd, kb_n = (Kd + SCALE_BLOCK - 1) / SCALE_BLOCK, nb_n = (N + SCALE_BLOCK - 1) / SCALE_BLOCK;
    Tile t;
    if (!find_tile<BM>(p, (N + COLS - 1) / COLS, t)) return;
    const int g = __builtin_amdgcn_readfirstlane(t.group), row0 = t.row0, row_end = t.row_end;
    const int n0 = t.nt * COLS;
    const bool routed = g < p.E;
    const size_t ge = routed ? g : g - p.E;
    const uint8_t *b0 = (routed ? p.b0 : p.sb0) + ge * N * Kd, *b1 = DUAL ? (routed ? p.b1 : p.sb1) + ge * N * Kd : nullptr;
    const float *bs0 = (routed ? p.bs0 : p.sbs0) + ge * nb_n * kb_n, *bs1 = DUAL ? (routed ? p.bs1 : p.sbs1) + ge * nb_n * kb_n : nullptr;

    // weight scales of the tile's blocks
    {
        constexpr int NBT = DUAL ? 2 : (BN + SCALE_BLOCK - 1) / SCALE_BLOCK + 1;
        for (int i = tid; i < NBT * kb_n; i += NW * 64) {
            const int j = i / kb_n, kb = i - j * kb_n;
            s_sw[j][kb] = DUAL ? ldg_f32((j ? bs1 : bs0) + (size_t)(n0 / SCALE_BLOCK) * kb_n + kb)
                               : ldg_f32(bs0 + (size_t)min(n0 / SCALE_BLOCK + j, nb_n - 1) * kb_n + kb);
        }
    }

    // addresses of this wave's loads: whole rows of 128 bytes, 8 an instruction
    const uint8_t *wp[WI], *tp[TI];
    int wpc[WI], tpc[TI];
#pragma unroll
    for (int j = 0; j < WI; ++j) {
        const int pos = wave * (WI * 8) + j * 8 + (lane >> 3);        // row in the stage
        const int b = (pos >> 4) % WB, m = pos & 15, w = (pos >> 4) / WB;
        const int bb = DUAL ? b % HB : b;
        // a lane's results of all blocks are consecutive columns
        const int n = min(n0 + w * (16 * HB) + (m >> 2) * (4 * HB) + bb * 4 + (m & 3), N - 1);
        wpc[j] = (lane & 7) ^ ((pos >> 1) & 7);
        wp[j] = (DUAL && b >= HB ? b1 : b0) + (size_t)n * Kd + wpc[j] * 16;
    }
    auto source_row = [&](int r) {                                     // row of a for row r of the tile (past the end: the last one)
        const int pos = min(row0 + r, row_end - 1);
        const int src = p.row_map ? ldg_i32(p.row_map + pos) / p.map_div : pos;
        return min(max(src, 0), p.a_rows - 1);
    };
    const bool tl = TR >= 8 || lane < TR * 8;                          // lanes with a token piece
#pragma unroll
    for (int j = 0; j < TI; ++j) {
        const int pos = wave * TR + j * 8 + (TR >= 8 ? lane >> 3 : min(lane >> 3, TR - 1));
        tpc[j] = (lane & 7) ^ ((pos >> 1) & 7);
        tp[j] = p.a + (size_t)source_row(pos) * Kd + tpc[j] * 16;
    }
    const bool sl = lane < TR;                                         // lanes with a token's scale
    const float *sp = p.a_scale + (size_t)source_row(wave * TR + min(lane, TR - 1)) * kb_n;

    auto issue = [&](int kt) {
        const int st = kt % S;
        uint8_t *base = smem + st * STAGE;
        const int k0 = kt * 128;
        const bool cut = k0 + 128 > Kd;                                // pieces past the row's end: a piece of the row instead
#pragma unroll
        for (int j = 0; j < WI; ++j) {
            const uint8_t *src = wp[j] + k0;
            if (cut && k0 + wpc[j] * 16 >= Kd) src -= wpc[j] * 16;
            __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)src, (BM_LDS void *)(base + (wave * (WI * 8) + j * 8) * 128), 16, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < TI; ++j) {
            const uint8_t *src = tp[j] + k0;
            if (cut && k0 + tpc[j] * 16 >= Kd) src -= tpc[j] * 16;
            if (tl) __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)src, (BM_LDS void *)(base + (BN + wave * TR + j * 8) * 128), 16, 0, 0);
        }
        if (sl) __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)(sp + kt), (BM_LDS void *)(s_sa + st * BM + wave * TR), 4, 0, 0);
    };

    f32x4 acc[WB][TB];
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
        for (int i = 0; i < TB; ++i) acc[b][i] = 0.0f;

    const int live = min(row_end - row0, BM) - wm * (TB * 16);        // tokens of this wave's blocks
    const int nb_live = (live + 15) / 16;
    // the wave's blocks of columns lie in one block of 128
    const int sw_i = DUAL ? 0 : (n0 % SCALE_BLOCK + wn * (16 * HB)) / SCALE_BLOCK;

    const int KT = kb_n;
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
        if (s < KT) issue(s);
    for (int kt = 0; kt < KT; ++kt) {
        if (KT - kt > S - 2) BM_WAIT_AND_MEET((S - 2) * PER)
        else BM_WAIT_AND_MEET(0)
        if (kt + S - 1 < KT) issue(kt + S - 1);
        const int st = kt % S;
        const uint8_t *ws = smem + st * STAGE, *ts = ws + BN * 128;
        auto frag = [&](const uint8_t *rows, int pos) {
            const int x = (pos >> 1) & 7;
            const u32x4 lo = *reinterpret_cast<const u32x4 *>(rows + pos * 128 + ((q4 ^ x) * 16));
            const u32x4 hi = *reinterpret_cast<const u32x4 *>(rows + pos * 128 + (((q4 + 4) ^ x) * 16));
            i32x8 f;
#pragma unroll
            for (int i = 0; i < 4; ++i) { f[i] = (int)lo[i]; f[4 + i] = (int)hi[i]; }
            return f;
        };
        Operand<WIDE> wf[WB];
#pragma unroll
        for (int b = 0; b < WB; ++b) wf[b].set(frag(ws, (wn * WB + b) * 16 + l16));
        const float sw0 = s_sw[sw_i][kt], sw1 = DUAL ? s_sw[1][kt] : 0.0f;
        const int rem = Kd - kt * 128;
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            if (i < nb_live) {
                const int pos = wm * (TB * 16) + i * 16 + l16;
                i32x8 tf = frag(ts, pos);
                if (rem < 128) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        tf[u] = q4 * 16 < rem ? tf[u] : 0;
                        tf[4 + u] = q4 * 16 + 64 < rem ? tf[4 + u] : 0;
                    }
                }
                Operand<WIDE> to;
                to.set(tf);
                const float sa = s_sa[st * BM + pos];
                const float f0 = sa * sw0, f1 = sa * sw1;
#pragma unroll
                for (int b = 0; b < WB; ++b) {
                    const f32x4 r = block_product(wf[b], to);
                    const float f = DUAL && b >= HB ? f1 : f0;
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[b][i][v] = fmaf(r[v], f, acc[b][i][v]);
                }
            }
        }
    }

    const int col = n0 + wn * (16 * HB) + q4 * (4 * HB);              // this lane's 4 * HB columns
    if (!DUAL) {
        if (col >= N) return;                                          // N is a multiple of 32: all of them or none
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            const int r = wm * (TB * 16) + i * 16 + l16;
            if (row0 + r >= row_end) continue;
            const size_t at = (size_t)(row0 + r) * N + col;
            if (p.c_f32) {
#pragma unroll
                for (int b = 0; b < WB; ++b) *(BM_GLOBAL f32x4 *)(static_cast<float *>(p.c) + at + 4 * b) = acc[b][i];
            } else {
#pragma unroll
                for (int b = 0; b < WB; ++b) {
                    const u32x2 o = {pack_bf16x2(acc[b][i][0], acc[b][i][1]), pack_bf16x2(acc[b][i][2], acc[b][i][3])};
                    *(BM_GLOBAL u32x2 *)(static_cast<uint16_t *>(p.c) + at + 4 * b) = o;
                }
            }
        }
        return;
    }
    // h in place of the gate's sums; the largest magnitude of a token's 128 columns over lanes and waves
    const bool in = col < N;
#pragma unroll
    for (int i = 0; i < TB; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int b = 0; b < HB; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float h = in ? silu(acc[b][i][v]) * acc[HB + b < WB ? HB + b : 0][i][v] : 0.0f;
                acc[b][i][v] = h;
                m = max(m, __builtin_bit_cast(uint32_t, h) & 0x7fffffffu);
            }
        m = max(m, (uint32_t)__shfl_xor((int)m, 16, WAVE));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32, WAVE));
        if (q4 == 0) s_amax[wn][wm * (TB * 16) + i * 16 + l16] = __builtin_bit_cast(float, m);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TB; ++i) {
        const int r = wm * (TB * 16) + i * 16 + l16;
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < WNN; ++w) m = max(m, __builtin_bit_cast(uint32_t, s_amax[w][r]));
        if (row0 + r >= row_end) continue;
        const float s = block_scale(m), inv = 1.0f / s;
        if (wn == 0 && q4 == 0) p.c_scale[(size_t)(row0 + r) * nb_n + n0 / SCALE_BLOCK] = s;
        if (!in) continue;
        uint8_t *c = static_cast<uint8_t *>(p.c) + (size_t)(row0 + r) * N + col;
#pragma unroll
        for (int b = 0; b < HB; ++b)
            *(BM_GLOBAL uint32_t *)(c + 4 * b) = e4m3x4(quotient(acc[b][i][0], s, inv), quotient(acc[b][i][1], s, inv),
                                                        quotient(acc[b][i][2], s, inv), quotient(acc[b][i][3], s, inv));
    }
}

// Workgroups of a launch: a bound on the row tiles of any grouping of the rows, times the column tiles.
static unsigned product_grid(const ProductParams &p, int bm, int cols) {
    const long long groups = p.n_groups < p.rows ? p.n_groups : p.rows;
    const long long tiles = (p.rows / bm + groups) * ((p.N + cols - 1) / cols);
    return (unsigned)((tiles + 7) / 8 * 8);
}

bool product_grid_ok(long long rows, int N, int n_groups) {
    return (rows / 16 + n_groups) * ((N + 31) / 32) < (1ll << 31) - 8;       // no tile is smaller
}

template <int BM, int BN, int NW, int WNN, int S, bool DUAL, bool WIDE>
static void launch_tiles(const ProductParams &p, hipStream_t st) {
    hipLaunchKernelGGL((product_kernel<BM, BN, NW, WNN, S, DUAL, WIDE>), dim3(product_grid(p, BM, DUAL ? BN / 2 : BN)), dim3(NW * 64), 0, st, p);
}

int launch_product(const ProductParams &p, hipStream_t st) {
    const long long avg = p.rows / p.n_groups;
    if (p.c_f32) {
        if (avg >= 128) launch_tiles<256, 256, 8, 4, 2, false, true>(p, st);
        else launch_tiles<64, 64, 4, 4, 4, false, true>(p, st);
    } else {
        if (avg >= 128) launch_tiles<256, 256, 8, 4, 2, false, false>(p, st);
        else launch_tiles<64, 64, 4, 4, 4, false, false>(p, st);
    }
    return launch_status(__func__);
}

int launch_swiglu(const ProductParams &p, hipStream_t st) {
    const long long avg = p.rows / p.n_groups;
    if (avg >= 128) launch_tiles<256, 256, 8, 4, 2, true, true>(p, st);
    else launch_tiles<64, 256, 8, 8, 3, true, true>(p, st);
    return launch_status(__func__);
}

}  // namespace bm
