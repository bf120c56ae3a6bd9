// Grouped products of 8-bit rows with 8-bit matrices, a 32-bit scale for each 128 values of a row and for each 128 x 128
// block of a matrix:
//   c[i][n] = sum_kb sa[i][kb] * sw[n / 128][kb] * sum_{k in block kb} a[i][k] * w[n][k]
// The inner sum is made by matrix instructions, the outer one by a fused multiply-add per value in 32 bits.  Weights are the
// matrix instruction's row operand and tokens its column operand, so that a lane's four results belong to one token and
// a block of weights: one scale for all four.
//
// Two forms of the inner sum.  v_mfma_f32_16x16x128 multiplies e4m3 as it is, 8192 flop a cycle and unit, but cuts each of the
// eight products that it adds at once below 2^-13 of the largest of them (measured: 1.4e-5 of the result's 2-norm, whatever
// the instruction's shape; magnitudes get smaller: where all products have one sign, the mean result is 7e-5 too small over random bytes,
// 3e-6 over normal values): it serves results that are rounded to bf16.  Results in 32 bits - sums that stay so, and h, whose
// scales are 32-bit numbers - widen e4m3 to fp16, which is exact, for v_mfma_f32_16x16x32_f16 at half the rate (7e-8).
#include "bm_product_rings.h"
#include "bm_products.h"

namespace bm {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Two e4m3 values, of the lower or the upper 16 bits, as fp16 (exact: three mantissa bits, exponents down to 2^-9)
__device__ __forceinline__ f16x2 widen2(uint32_t a, bool high) {
    return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
}
__device__ __forceinline__ f16x8 join8(f16x2 p, f16x2 q, f16x2 r, f16x2 s) { return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]}; }
__device__ __forceinline__ f16x8 widen8(uint32_t a, uint32_t b) { return join8(widen2(a, false), widen2(a, true), widen2(b, false), widen2(b, true)); }

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
// Two blocks of weights with the same tokens, their chains of matrix instructions interleaved
__device__ __forceinline__ void block_products(const Operand<false> &a0, const Operand<false> &a1, const Operand<false> &b, f32x4 &r0, f32x4 &r1) {
    r0 = block_product(a0, b);
    r1 = block_product(a1, b);
}
__device__ __forceinline__ void block_products(const Operand<true> &a0, const Operand<true> &a1, const Operand<true> &b, f32x4 &r0, f32x4 &r1) {
    r0 = r1 = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(a0.v[i], b.v[i], r0, 0, 0, 0);
        r1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(a1.v[i], b.v[i], r1, 0, 0, 0);
    }
}

#define BM_LDS __attribute__((address_space(3)))
// BYTES of every lane from base + offset + step into LDS, in the order of the lanes; offset + step + BYTES stay below 2^32 - 1, where the
// buffer ends.  A buffer instruction: behind a global one that writes LDS the compiler holds every use of an LDS read until all
// reads before it are done (2 to 4 % of the large products).
template <int BYTES>
__device__ __forceinline__ void fetch(const void *base, uint32_t offset, uint32_t step, void *lds) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, -1, 0x00027000);
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (BM_LDS void *)lds, 16, (int)offset, (int)step, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (BM_LDS void *)lds, 4, (int)offset, (int)step, 0, 0);
}
// At most n direct loads of this wave are still in flight and its LDS accesses are done; then all waves meet.
// (s_waitcnt of gfx9: vmcnt[3:0] | expcnt 7 << 4 | lgkmcnt 0 << 8 | vmcnt[5:4] << 14)
#define BM_WAIT_AND_MEET(n)                                                             \
    {                                                                                   \
        __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (((n) >> 4) << 14));         \
        asm volatile("s_barrier" ::: "memory");                                         \
    }
// The same for a wave whose LDS is its own
#define BM_WAIT_OWN(n)                                                                  \
    {                                                                                   \
        __builtin_amdgcn_s_waitcnt(((n) & 15) | (7 << 4) | (((n) >> 4) << 14));         \
        asm volatile("" ::: "memory");                                                  \
    }

// The tile of a workgroup: rows [row0, ..) of a group that ends at row_end, column tile nt.
struct Tile {
    int group, row0, row_end, nt;
};

// The groups' row ranges and tile counts, in LDS.  Offsets are clamped to the rows and raised to the largest before them: whatever
// they hold, groups do not overlap and no tile leaves the rows.
struct TileTable {
    int first[BM_MAX_E + 8 + 1];        // tiles of height bm before the group; [n_groups]: all
    int lo[BM_MAX_E + 8 + 1];           // first row; the group ends where the next begins
};

// Called by one wave; the workgroup has to meet before the table is read.
__device__ __forceinline__ void build_tile_table(const ProductParams &p, int bm, TileTable &tt) {
    const int lane = lane_id();
    int total = 0, last = p.offsets ? min(max(ldg_i32(p.offsets), 0), p.rows) : 0;
    for (int c = 0; c < p.n_groups; c += WAVE) {
        const int g = c + lane;
        int hi = last;
        if (g < p.n_groups) hi = p.offsets ? min(max(ldg_i32(p.offsets + g + 1), last), p.rows) : p.rows;
#pragma unroll
        for (int s = 1; s < WAVE; s <<= 1) {
            const int o = __shfl_up(hi, s, WAVE);
            hi = lane >= s ? max(hi, o) : hi;
        }
        const int before = __shfl_up(hi, 1, WAVE), lo = lane ? before : last;
        const int mine = (hi - lo + bm - 1) / bm;
        int sum = mine;
#pragma unroll
        for (int s = 1; s < WAVE; s <<= 1) {
            const int o = __shfl_up(sum, s, WAVE);
            sum += lane >= s ? o : 0;
        }
        if (g < p.n_groups) {
            tt.first[g] = total + sum - mine;
            tt.lo[g] = lo;
        }
        total += __builtin_amdgcn_readlane(sum, WAVE - 1);
        last = __builtin_amdgcn_readlane(hi, WAVE - 1);
    }
    if (lane == 0) {
        tt.first[p.n_groups] = total;
        tt.lo[p.n_groups] = last;
    }
}

// Tiles are numbered group by group, inside a group by column tile and then by row tile (neighbours share their weights).
__device__ __forceinline__ Tile tile_at(const ProductParams &p, const TileTable &tt, int bm, int n_nt, int lid) {
    const int lane = lane_id(), m = lid / n_nt;        // the row tiles before it belong to whole groups before it
    Tile t{};
    for (int c = 0; c < p.n_groups; c += WAVE) {
        const int g = min(c + lane, p.n_groups - 1);
        const int f = tt.first[g], n = tt.first[g + 1] - f;
        const unsigned long long hit = __ballot(c + lane < p.n_groups && f <= m && m < f + n);
        if (hit) {
            const int src = __ffsll(hit) - 1, f0 = __builtin_amdgcn_readlane(f, src), rows_n = __builtin_amdgcn_readlane(n, src);
            const int in = lid - f0 * n_nt;
            t.group = c + src;
            t.nt = in / rows_n;
            t.row0 = __builtin_amdgcn_readfirstlane(tt.lo[t.group]) + (in % rows_n) * bm;
            t.row_end = __builtin_amdgcn_readfirstlane(tt.lo[t.group + 1]);
            break;
        }
    }
    return t;
}

// Every XCD takes a contiguous share of the tiles; workgroups go round-robin to the XCDs, so blockIdx.x % 8 names it.
struct Share {
    int begin, end, step;
};
__device__ __forceinline__ Share my_share(int tiles) {
    const int per_xcd = (tiles + 7) >> 3, from = min((int)(blockIdx.x & 7) * per_xcd, tiles);
    return Share{from + (int)(blockIdx.x >> 3), min(from + per_xcd, tiles), (int)(gridDim.x >> 3)};
}

// Row of a for output row `row` of a group that ends at row_end (past the end: the last one's)
__device__ __forceinline__ int row_of_id(const ProductParams &p, int id) { return min(max(id / p.map_div, 0), p.a_rows - 1); }
__device__ __forceinline__ int source_row(const ProductParams &p, int row, int row_end) {
    const int pos = min(row, row_end - 1);
    return p.row_map ? row_of_id(p, ldg_i32(p.row_map + pos)) : min(pos, p.a_rows - 1);
}

// Sixteen values of row pos of a stage
__device__ __forceinline__ u32x4 lds_piece(const uint8_t *rows, int pos, int piece) {
    return *reinterpret_cast<const u32x4 *>(rows + pos * 128 + ((piece ^ ((pos >> 1) & 7)) * 16));
}
// A lane's 32 values of row pos of a stage: pieces q4 and q4 + 4 (any order serves, the same for both operands)
__device__ __forceinline__ i32x8 lds_operand(const uint8_t *rows, int pos, int q4) {
    const u32x4 lo = lds_piece(rows, pos, q4), hi = lds_piece(rows, pos, q4 + 4);
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// The block of 128 at which a streaming tile's walk along the reduction begins (it goes round).  Workgroups that start together
// would otherwise read the same offset of their rows at the same time, which lie a power of two apart in many layers, and
// meet in few memory channels (5 % of the gate/up product of one token).  A function of the group and the columns: in tiles of one
// shape a row's sum does not depend on the rows beside it.
__device__ __forceinline__ int entry_block(const Tile &t, int kb_n) { return (t.group * 7 + t.nt * 5) % kb_n; }

// Four consecutive values of c
__device__ __forceinline__ void store4(const ProductParams &p, size_t at, f32x4 v) {
    if (p.c_f32) *(BM_GLOBAL f32x4 *)(static_cast<float *>(p.c) + at) = v;
    else *(BM_GLOBAL u32x2 *)(static_cast<uint16_t *>(p.c) + at) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// The group's matrices and their scales
struct Matrices {
    const uint8_t *w0, *w1;
    const float *s0, *s1;
};
template <bool DUAL>
__device__ __forceinline__ Matrices matrices_of(const ProductParams &p, int group) {
    const int kb_n = (p.Kd + SCALE_BLOCK - 1) / SCALE_BLOCK, nb_n = (p.N + SCALE_BLOCK - 1) / SCALE_BLOCK;
    const bool routed = group < p.E;
    const size_t g = routed ? group : group - p.E, at = g * p.N * p.Kd, sat = g * nb_n * kb_n;
    return Matrices{(routed ? p.b0 : p.sb0) + at, DUAL ? (routed ? p.b1 : p.sb1) + at : nullptr,
                    (routed ? p.bs0 : p.sbs0) + sat, DUAL ? (routed ? p.bs1 : p.sbs1) + sat : nullptr};
}

__device__ uint4 zero_piece;             // where pieces of tokens past the row's end come from

}  // namespace

// ---------------------------------------------------------------------------------------------------------------------
// Tiles of BM tokens x BN weight rows (DUAL: 128 of the gate, 128 of the up matrix) on 8 waves, WNN of them along the weight
// rows.  The reduction goes in steps of 128 through two rings in LDS, SW stages of weights and ST of tokens, filled with
// direct loads: a row's 128 bytes are one cache line, 8 rows an instruction.  Piece p of row r lies in slot p ^ ((r >> 1) & 7),
// so that the 16 rows of an operand read fall into different banks.
//
// A workgroup takes one tile after the other and its loads run ahead across them: the last steps of a tile fetch the first
// blocks of the next, whose rows and scales were fetched at the tile's beginning.  A step waits for the loads that it needs
// and leaves those behind them in flight (AHEAD; loads return in order).  Other loads in between make the wait stricter for these,
// but are covered by it themselves only if as many of a step's loads follow them: the next tile's row ids, asked for in step 0,
// are not where a walk is as short as four stages, and are then waited for by themselves (TileRings; 8 gathered rows in each of 64
// groups, 512 -> 640: 15.9 us; 640 -> 640, which need no such wait: 17.6).
//   step s:  tokens of step s and weights of step s have landed -> all waves meet (so the stages read in step s - 1 are
//   free) -> load the tokens of step s + ST - 1 and the weights of step s + SW - 1 -> multiply.
// NEAR: the reduction is a multiple of 128, at least MIN_STEPS blocks, and a is smaller than 4 GiB: no piece is cut, addresses are
// 32-bit offsets (which leaves room for tiles of 192 tokens).
// SPREAD (128 and 192 rows): the loads of a step stand between its matrix instructions.  Issued together they held a wave for 900 of
// 6300 cycles, since a unit takes 64 bytes a cycle of them.  Past the last tile they fetch the tile's beginning once more.
// Bounds.  Few rows: the weights' bytes, read once, 4.6 TB/s at 128 rows of 4096 -> 14336 in 8 groups.  Many rows: the matrix units at
// the clock that their power leaves.  14336 -> 4096 of 8192 rows: 531 us, 1.81 PFLOP/s (a library's product of 8192^3 in e4m3: 2.7).
// With e4m3 widened, 4096 -> 14336 of 8192 rows: 1637 us, 1.17 PFLOP/s (in fp16: 1.59), matrix units busy 57 % of the cycles and vector
// units 62 %, the clock at 2.17 of 2.4 GHz; tiles of 128 rows with instructions of 32 x 32 took 3 % fewer cycles, at 1.93 GHz, and were no
// faster.  What is spilled (13 registers of the 192 x 256 gate/up form, 19 of its form with cut blocks, 1 to 6 of three products) is read
// again where a tile ends or the next begins, never in a step.
// Everything lies in one LDS array: of several, the compiler tells apart which one direct loads fill, and holds every read
// of that one until no load is in flight.
// ---------------------------------------------------------------------------------------------------------------------
template <int BM, int BN, int WMN, int WNN, int KG, int SW, int ST, int PER_UNIT, bool DUAL, bool WIDE, bool NEAR>
__global__ void __launch_bounds__(WMN * WNN * KG * 64, WMN * WNN * KG * PER_UNIT / 4) tiles_kernel(ProductParams p) {
    constexpr int NW = WMN * WNN;                              // waves of each of the KG parts of the reduction
    constexpr int TB = BM / WMN / 16, WB = BN / WNN / 16;      // 16-token and 16-row blocks of a wave
    constexpr int HB = DUAL ? WB / 2 : WB;                     // of these, blocks of different columns
    constexpr int COLS = DUAL ? BN / 2 : BN;
    using Rings = TileRings<BM, BN, NW, SW, ST>;
    constexpr int WI = Rings::WI, TR = Rings::TR, TI = Rings::TI, PER = Rings::PER, AHEAD = Rings::AHEAD;
    constexpr int PART = BM <= 64 ? 1 : TB;                    // blocks that are multiplied or, where no token is theirs, left out together
    // loads are issued between the matrix instructions, where these leave enough places
    constexpr bool SPREAD = BM > 64 && PER_UNIT == 1 && PER <= (WIDE ? TB * 4 : TB * WB / 2);
    static_assert(TB * 16 * WMN == BM && WB * 16 * WNN == BN, "tile shape");
    constexpr int MAX_KB = MAX_PRODUCT_KD / SCALE_BLOCK;
    constexpr int W_BYTES = SW * KG * BN * 128, T_BYTES = ST * KG * BM * 128, EXCHANGE = KG > 1 ? (KG - 1) * NW * 1024 : 0;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[W_BYTES + T_BYTES + EXCHANGE + (ST * KG * BM + 4 * MAX_KB + BM + (DUAL ? WNN * BM : 0)) * 4 + sizeof(TileTable)];
    uint8_t *const w_ring = lds, *const t_ring = lds + W_BYTES;
    f32x4 *const s_part = reinterpret_cast<f32x4 *>(t_ring + T_BYTES);            // [KG - 1][NW][64] sums on their way to the first part
    float *const s_sa = reinterpret_cast<float *>(t_ring + T_BYTES + EXCHANGE);   // [ST][KG][BM] tokens' scales
    float *const s_sw = s_sa + ST * KG * BM;                                           // [2 tiles][2][MAX_KB] weight blocks' scales
    int *const s_id = reinterpret_cast<int *>(s_sw + 4 * MAX_KB);                 // [BM] row_map of the next tile
    uint32_t *const s_amax = reinterpret_cast<uint32_t *>(s_id + BM);             // [WNN][BM]
    TileTable &tt = *reinterpret_cast<TileTable *>(s_amax + (DUAL ? WNN * BM : 0));

    const int lane = lane_id(), all = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), kg = all / NW, wave = all % NW;
    const int wm = wave / WNN, wn = wave % WNN, q4 = lane >> 4, l16 = lane & 15;
    const int N = p.N, Kd = p.Kd, kb_n = (Kd + SCALE_BLOCK - 1) / SCALE_BLOCK, nb_n = (N + SCALE_BLOCK - 1) / SCALE_BLOCK;
    const int n_nt = (N + COLS - 1) / COLS, KT = NEAR ? kb_n / KG : max((kb_n + KG - 1) / KG, MIN_STEPS);

    if (all == 0) build_tile_table(p, BM, tt);
    BM_WAIT_AND_MEET(0)
    const Share share = my_share(__builtin_amdgcn_readfirstlane(tt.first[p.n_groups]) * n_nt);
    if (share.begin >= share.end) return;

    // ---- loading side: the tile whose weights are fetched, the tile whose tokens are fetched ----
    Matrices wt;                                               // at the tile's first row
    uint32_t wo[WI];                                           // 32 bits: 256 rows of at most 32768 bytes
    int w_entry = 0;
    const uint8_t *tp[NEAR ? 1 : TI];
    const float *sp = nullptr;
    uint32_t to[NEAR ? TI : 1], so = 0;
    int t_entry = 0;
    auto w_piece = [&](int j) { return (lane & 7) ^ (((wave * (WI * 8) + j * 8 + (lane >> 3)) >> 1) & 7); };
    auto t_pos = [&](int j) { return wave * TR + j * 8 + (TR >= 8 ? lane >> 3 : min(lane >> 3, TR - 1)); };
    auto t_piece = [&](int j) { return (lane & 7) ^ ((t_pos(j) >> 1) & 7); };
    auto entry_of = [&](const Tile &t) { return BM <= 64 ? entry_block(t, KT) : 0; };
    auto aim_weights = [&](const Tile &t) {
        const int n0 = t.nt * COLS;
        wt = matrices_of<DUAL>(p, t.group);
        wt.w0 += (size_t)n0 * Kd;
        if (DUAL) wt.w1 += (size_t)n0 * Kd;
        w_entry = entry_of(t);
#pragma unroll
        for (int j = 0; j < WI; ++j) {
            const int pos = wave * (WI * 8) + j * 8 + (lane >> 3);                // row in the stage
            const int b = (pos >> 4) % WB, m = pos & 15, w = (pos >> 4) / WB, bb = DUAL ? b % HB : b;
            // a lane's results of all blocks are consecutive columns
            const int n = min(w * (16 * HB) + (m >> 2) * (4 * HB) + bb * 4 + (m & 3), N - 1 - n0);
            wo[j] = (uint32_t)n * (uint32_t)Kd + w_piece(j) * 16;
        }
    };
    // a lane finds one of its wave's rows: by its id in LDS (row r of the tile at s_id[r]), or by row_map
    auto aim_tokens = [&](const Tile &t, bool ids) {
        const int mine = wave * TR + min(lane, TR - 1);
        const int row = ids && p.row_map ? row_of_id(p, s_id[mine]) : source_row(p, t.row0 + mine, t.row_end);
#pragma unroll
        for (int j = 0; j < TI; ++j) {
            const int r = __shfl(row, t_pos(j) - wave * TR, WAVE);
            if constexpr (NEAR) to[j] = (uint32_t)r * (uint32_t)Kd + t_piece(j) * 16;
            else tp[j] = p.a + (size_t)r * Kd + t_piece(j) * 16;
        }
        if constexpr (NEAR) so = (uint32_t)row * (uint32_t)kb_n;
        else sp = p.a_scale + (size_t)row * kb_n;
        t_entry = entry_of(t);
    };
    auto block_at = [&](int step, int entry) { return (step + entry < KT ? step + entry : step + entry - KT) * KG + kg; };
    // Pieces past the row's end: of weights any piece of the row, of tokens zeros.  Blocks past the last one: the first, and zeros.
    auto load_weight = [&](int step, int slot, int j) {
        const int kt = block_at(step, w_entry), k0 = NEAR || kt < kb_n ? kt * 128 : 0;
        const int pos = wave * (WI * 8) + j * 8, pc = w_piece(j) * 16;
        const uint8_t *from = DUAL && (pos >> 4) % WB >= HB ? wt.w1 : wt.w0;
        const uint32_t off = NEAR || k0 + pc < Kd ? wo[j] : wo[j] - pc;
        fetch<16>(from, off, k0, w_ring + (slot * KG + kg) * (BN * 128) + pos * 128);
    };
    auto load_token = [&](int step, int slot, int j) {
        const int kt = block_at(step, t_entry), k0 = kt * 128;
        if (j < TI) {
            uint8_t *lds_at = t_ring + (slot * KG + kg) * (BM * 128) + (wave * TR + j * 8) * 128;
            if (TR >= 8 || lane < TR * 8) {
                if constexpr (NEAR) {
                    fetch<16>(p.a, to[j], k0, lds_at);
                } else {
                    const uint8_t *src = k0 + t_piece(j) * 16 < Kd ? tp[j] + k0 : reinterpret_cast<const uint8_t *>(&zero_piece);
                    __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)src, (BM_LDS void *)lds_at, 16, 0, 0);
                }
            }
        } else {
            float *lds_at = s_sa + (slot * KG + kg) * BM + wave * TR;
            if (lane < TR) {
                if constexpr (NEAR) fetch<4>(p.a_scale, so * 4, kt * 4, lds_at);
                else __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)(sp + min(kt, kb_n - 1)), (BM_LDS void *)lds_at, 4, 0, 0);
            }
        }
    };
    auto load_weights = [&](int step, int slot) {
#pragma unroll
        for (int j = 0; j < WI; ++j) load_weight(step, slot, j);
    };
    auto load_tokens = [&](int step, int slot) {
#pragma unroll
        for (int j = 0; j <= TI; ++j) load_token(step, slot, j);
    };
    // What a tile needs beside its operands: the scales of its weight blocks (a wave fetches 64 of one of two rows) and its rows' ids
    auto load_meta = [&](const Tile &t, int buf, bool ids) {
        const int j = all >> 2, kb = (all & 3) * 64 + lane, nb = min(t.nt * COLS / SCALE_BLOCK + (DUAL ? 0 : j), nb_n - 1);
        const Matrices m = matrices_of<DUAL>(p, t.group);
        const float *s = (DUAL && j ? m.s1 : m.s0) + (size_t)nb * kb_n;
        if (j < 2 && kb < kb_n)
            fetch<4>(s, kb * 4, 0, s_sw + (buf * 2 + j) * MAX_KB + (all & 3) * 64);
        if (ids && p.row_map && lane < TR)
            fetch<4>(p.row_map + t.row0, (uint32_t)min(wave * TR + lane, t.row_end - 1 - t.row0) * 4, 0, s_id + wave * TR);
    };

    int lid = share.begin;
    Tile cur = tile_at(p, tt, BM, n_nt, lid), next{};
    aim_weights(cur);
    aim_tokens(cur, false);
    load_meta(cur, 0, false);
    int w_slot = 0, t_slot = 0;                                // next stages to fill
    auto advance = [](int &slot, int n) { slot = slot + 1 == n ? 0 : slot + 1; };
#pragma unroll
    for (int s = 1 - SW; s < 0; ++s) {
        if (s + ST - 1 >= 0) { load_tokens(s + ST - 1, t_slot); advance(t_slot, ST); }
        load_weights(s + SW - 1, w_slot);
        advance(w_slot, SW);
    }
    int w_read = 0, t_read = 0, buf = 0;                       // stages and scales that are read

    while (true) {
        const bool more = lid + share.step < share.end;
        const int live = min(cur.row_end - cur.row0, BM) - wm * (TB * 16), entry = entry_of(cur);
        f32x4 acc[WB][TB];
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
            for (int i = 0; i < TB; ++i) acc[b][i] = 0.0f;

        for (int step = 0; step < KT; ++step) {
            if (SPREAD || more || step + SW - 2 < KT) BM_WAIT_AND_MEET(AHEAD)
            else BM_WAIT_AND_MEET(0)
            if (step == 0 && more) {
                next = tile_at(p, tt, BM, n_nt, lid + share.step);
                load_meta(next, buf ^ 1, true);
            }
            if (more && step + ST - 1 == KT) {
                if constexpr (Rings::ids_need_wait(MIN_STEPS))
                    if (Rings::ids_need_wait(KT)) BM_WAIT_OWN(Rings::BEHIND_IDS)
                aim_tokens(next, true);
            }
            if (more && step + SW - 1 == KT) aim_weights(next);
            const int t_step = step + ST - 1 < KT ? step + ST - 1 : step + ST - 1 - KT, w_step = step + SW - 1 < KT ? step + SW - 1 : step + SW - 1 - KT;
            const int t_fill = t_slot, w_fill = w_slot;
            auto load_part = [&](int j) {
                if (j <= TI) load_token(t_step, t_fill, j);
                else if (j < PER) load_weight(w_step, w_fill, j - TI - 1);
            };
            if (SPREAD || more || step + ST - 1 < KT) {
                if (!SPREAD) load_tokens(t_step, t_slot);
                advance(t_slot, ST);
            }
            if (SPREAD || more || step + SW - 1 < KT) {
                if (!SPREAD) load_weights(w_step, w_slot);
                advance(w_slot, SW);
            }
            const uint8_t *ws = w_ring + (w_read * KG + kg) * (BN * 128), *ts = t_ring + (t_read * KG + kg) * (BM * 128);
            const float *sa_at = s_sa + (t_read * KG + kg) * BM + wm * (TB * 16) + l16;
            const int kt = NEAR ? block_at(step, entry) : min(block_at(step, entry), kb_n - 1);
            // DUAL: the gate's and the up matrix's scale; else one of the two blocks of 128 columns, the wave's
            const float sw0 = s_sw[(buf * 2 + (DUAL ? 0 : wn * (16 * HB) / SCALE_BLOCK)) * MAX_KB + kt];
            const float sw1 = DUAL ? s_sw[(buf * 2 + 1) * MAX_KB + kt] : sw0;
            if (BM > 64 && live <= 0) {
                if (SPREAD) {
                    load_tokens(t_step, t_fill);
                    load_weights(w_step, w_fill);
                }
                advance(w_read, SW);
                advance(t_read, ST);
                continue;
            }
            if constexpr (WIDE && BM > 64) {
                // Beside every matrix instruction stand the widening of the next values of the tokens (in the first 16 tokens, of the
                // weights too) and the addition of one result of the 16 tokens before: a unit works at a matrix instruction for 16
                // cycles and takes two others of the same wave meanwhile, not three (20.6).  A wave goes first until its first 16
                // tokens are done, so that the two waves of a unit drift apart (2 %)
                const int pos0 = wm * (TB * 16) + l16;
                __builtin_amdgcn_s_setprio(1);
                u32x4 raw[2] = {lds_piece(ts, pos0, q4), lds_piece(ts, pos0, q4 + 4)}, wr[WB][2];
                float sa[TB];
#pragma unroll
                for (int i = 0; i < TB; ++i) sa[i] = sa_at[i * 16];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int b = 0; b < WB; ++b) wr[b][h] = lds_piece(ws, (wn * WB + b) * 16 + l16, q4 + 4 * h);
                __builtin_amdgcn_sched_barrier(0);
                f16x8 wf[WB][4], tf[2];
                f32x4 r[2][WB];
#pragma unroll
                for (int b = 0; b < WB; ++b) wf[b][0] = widen8(wr[b][0][0], wr[b][0][1]);
                tf[0] = widen8(raw[0][0], raw[0][1]);
                f16x2 part[4];
                float f0 = 0.0f, f1 = 0.0f;
#pragma unroll
                for (int n = 0; n < TB; ++n) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int h = ((k + 1) & 3) >> 1, u = ((k + 1) & 1) * 2;
#pragma unroll
                        for (int b = 0; b < WB; ++b) {
                            r[n & 1][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wf[b][k], tf[k & 1], k ? r[n & 1][b] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
                            if (n + 1 < TB || k < 3)
#pragma unroll
                                for (int c = b * 4 / WB; c < (b + 1) * 4 / WB; ++c) part[c] = widen2(raw[h][u + (c >> 1)], c & 1);
                            if (n == 0 && k < 3) wf[b][k + 1] = widen8(wr[b][h][u], wr[b][h][u + 1]);
                            if (n > 0) acc[b][n - 1][k] = fmaf(r[(n + 1) & 1][b][k], DUAL && b >= HB ? f1 : f0, acc[b][n - 1][k]);
                            if (b == 0 && (k & 1) && n + 1 < TB) raw[k >> 1] = lds_piece(ts, pos0 + (n + 1) * 16, q4 + 4 * (k >> 1));
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        if (SPREAD) load_part(n * 4 + k);
                        tf[(k + 1) & 1] = join8(part[0], part[1], part[2], part[3]);
                    }
                    if (n == 0) __builtin_amdgcn_s_setprio(0);
                    f0 = sa[n] * sw0;
                    f1 = sa[n] * sw1;
                }
#pragma unroll
                for (int b = 0; b < WB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[b][TB - 1][v] = fmaf(r[(TB + 1) & 1][b][v], DUAL && b >= HB ? f1 : f0, acc[b][TB - 1][v]);
            } else {
                Operand<WIDE> wf[WB];
#pragma unroll
                for (int b = 0; b < WB; ++b) wf[b].set(lds_operand(ws, (wn * WB + b) * 16 + l16, q4));
#pragma unroll
                for (int i0 = 0; i0 < TB; i0 += PART) {
                    if (BM <= 64 && live <= i0 * 16) break;              // (in large tiles the branch costs 60 spilled registers)
                    // operands of the next 16 tokens are read, and the results of the block before are added, under the matrix
                    // instructions of the present one
                    const int pos0 = wm * (TB * 16) + i0 * 16 + l16;
                    i32x8 raw = lds_operand(ts, pos0, q4);
                    float sa[PART];
#pragma unroll
                    for (int i = 0; i < PART; ++i) sa[i] = sa_at[(i0 + i) * 16];
                    f32x4 r[2][2];
                    Operand<WIDE> tf;
                    auto add = [&](int n) {
                        const float f = sa[n / WB] * (DUAL && n % WB >= HB ? sw1 : sw0);
#pragma unroll
                        for (int v = 0; v < 4; ++v) acc[n % WB][i0 + n / WB][v] = fmaf(r[n >> 1 & 1][n & 1][v], f, acc[n % WB][i0 + n / WB][v]);
                    };
#pragma unroll
                    for (int n = 0; n < PART * WB; n += 2) {
                        if (n % WB == 0) {
                            tf.set(raw);
                            if (n / WB + 1 < PART) raw = lds_operand(ts, pos0 + (n / WB + 1) * 16, q4);
                        }
                        block_products(wf[n % WB], wf[n % WB + 1], tf, r[n >> 1 & 1][0], r[n >> 1 & 1][1]);
                        if (SPREAD) load_part(n >> 1);
                        if (n > 0) {
                            add(n - 2);
                            add(n - 1);
                        }
                    }
                    add(PART * WB - 2);
                    add(PART * WB - 1);
                }
            }
            advance(w_read, SW);
            advance(t_read, ST);
        }

        // the parts of the reduction, added in order: one block of 16 x 16 of every wave at a time
        if constexpr (KG > 1) {
#pragma unroll
            for (int i = 0; i < TB; ++i)
#pragma unroll
                for (int b = 0; b < WB; ++b) {
                    if (kg > 0) s_part[((kg - 1) * NW + wave) * 64 + lane] = acc[b][i];
                    BM_WAIT_AND_MEET(63)
                    if (kg == 0)
#pragma unroll
                        for (int k = 0; k < KG - 1; ++k) acc[b][i] += s_part[(k * NW + wave) * 64 + lane];
                    BM_WAIT_AND_MEET(63)
                }
        }
        // ---- write-out: a lane holds 4 * HB consecutive columns of each of its tokens (N is a multiple of 32: all in or none) ----
        const int n0 = cur.nt * COLS, col = n0 + wn * (16 * HB) + q4 * (4 * HB), first = wm * (TB * 16) + l16;
        if constexpr (!DUAL) {
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                const int r = cur.row0 + first + i * 16;
                if (kg > 0 || r >= cur.row_end || col >= N) continue;
#pragma unroll
                for (int b = 0; b < WB; ++b) store4(p, (size_t)r * N + col + 4 * b, acc[b][i]);
            }
        } else {
            // h = silu(gate) * up in place of the gate's sums; the largest magnitude of a token's 128 columns over lanes and waves
            // (as bits: their order is that of non-negative numbers); the scale; the conversion
            const bool in = col < N;
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                uint32_t m = 0;
#pragma unroll
                for (int b = 0; b < HB; ++b)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float h = in ? silu(acc[b][i][v]) * acc[HB + b][i][v] : 0.0f;
                        acc[b][i][v] = h;
                        m = max(m, __builtin_bit_cast(uint32_t, h) & 0x7fffffffu);
                    }
                m = max(m, (uint32_t)__shfl_xor((int)m, 16, WAVE));
                m = max(m, (uint32_t)__shfl_xor((int)m, 32, WAVE));
                if (q4 == 0 && kg == 0) s_amax[wn * BM + first + i * 16] = m;
            }
            BM_WAIT_AND_MEET(63)                              // LDS only: loads go on
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                const int at = first + i * 16, r = cur.row0 + at;
                uint32_t m = 0;
#pragma unroll
                for (int w = 0; w < WNN; ++w) m = max(m, s_amax[w * BM + at]);
                if (kg > 0 || r >= cur.row_end) continue;
                const float s = block_scale(m);
                const Divisor by = divisor(s);
                if (wn == 0 && q4 == 0) p.c_scale[(size_t)r * nb_n + cur.nt] = s;
                if (!in) continue;
                uint8_t *c = static_cast<uint8_t *>(p.c) + (size_t)r * N + col;
#pragma unroll
                for (int b = 0; b < HB; ++b) {
                    float v[4] = {acc[b][i][0], acc[b][i][1], acc[b][i][2], acc[b][i][3]};
                    raise(v, by);
                    *(BM_GLOBAL uint32_t *)(c + 4 * b) = e4m3x4(quotient(v[0], by), quotient(v[1], by), quotient(v[2], by), quotient(v[3], by));
                }
            }
        }
        if (!more) {
            if (SPREAD) BM_WAIT_OWN(0)                        // no load may land in LDS that is another's by then
            return;
        }
        cur = next;
        lid += share.step;
        buf ^= 1;
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// One product of few rows a group: the weights' bytes are what counts.  Every wave streams 32 weight rows through a ring of its
// own in LDS - whole cache lines, no barrier in the loop; wave k takes every fourth block of 128, so that the workgroup reads
// consecutive lines, and the parts are added in order at the end.
// Tokens go straight to registers, as far ahead as the weights: loads return in order, and waiting for a nearer one would
// wait for all weights in flight.  Their scales lie in LDS from the start (from memory in the loop they cost as many bytes
// from the L2 as the tokens: a line for four).  Measured at 1 row, 4096 -> 4096: 8.5 to 9.4 us, of which 5 are the launch and the first
// and last bytes' way; 14336 -> 4096, two groups of one row: 21.7 to 23.3 us, 5.0 to 5.4 TB/s.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int STREAM_WAVES = 4;
constexpr int STREAM_SCALES = 32 * 112;          // tokens x blocks of 128 whose scales fit beside the ring

template <int TB, bool WIDE>
__device__ __forceinline__ void stream_tile(const ProductParams &p, const Tile &t, int rows, uint8_t *ring, const float *s_sw, const float *s_sa,
                                            const uint8_t *b0) {
    constexpr int WB = 2, S = 4, PER = 4 + 2 * TB;              // stages; loads of a step
    static_assert((S - 2) * PER < 64, "the wait counts up to 63 loads");
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int q4 = lane >> 4, l16 = lane & 15;
    const int N = p.N, Kd = p.Kd, kb_n = (Kd + SCALE_BLOCK - 1) / SCALE_BLOCK;
    const int row0 = t.row0, row_end = row0 + rows, n0 = t.nt * 32;      // the tile's rows, fewer than the matrix instruction's
    uint8_t *mine = ring + wave * (S * 4096);

    const uint8_t *const rows_at = b0 + (size_t)n0 * Kd;
    uint32_t wo[4];
    const int piece = (lane & 7) ^ ((lane >> 4) & 3);             // of rows 8 j + lane / 8: (row >> 1) & 7 is 4 (j & 1) more
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int pos = j * 8 + (lane >> 3), b = pos >> 4, m = pos & 15;
        const int n = min((m >> 2) * 8 + b * 4 + (m & 3), N - 1 - n0);         // a lane's results: consecutive columns
        wo[j] = (uint32_t)n * (uint32_t)Kd + ((piece ^ (4 * (j & 1))) * 16);
    }
    const uint8_t *tp[TB];
#pragma unroll
    for (int i = 0; i < TB; ++i) tp[i] = p.a + (size_t)source_row(p, row0 + i * 16 + l16, row_end) * Kd + q4 * 16;
    u32x4 tlo[S][TB], thi[S][TB];
    f32x4 acc[WB][TB];
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
        for (int i = 0; i < TB; ++i) acc[b][i] = 0.0f;

    const int steps = (kb_n - wave + STREAM_WAVES - 1) / STREAM_WAVES, entry = entry_block(t, kb_n);
    auto block_of = [&](int step) {
        const int kt = wave + min(step, steps - 1) * STREAM_WAVES + entry;      // past the end: the last one again
        return kt < kb_n ? kt : kt - kb_n;
    };
    auto issue = [&](int step, int st, u32x4 (&lo)[TB], u32x4 (&hi)[TB]) {
        const int k0 = block_of(step) * 128;
        // pieces past the row's end: the row's piece 0 of this block instead (arithmetic, no branch around a load)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int pc = (piece ^ (4 * (j & 1))) * 16, back = k0 + pc >= Kd ? pc : 0;
            fetch<16>(rows_at, wo[j] - back, k0, mine + st * 4096 + j * 1024);
        }
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            const int at = q4 * 16, lo_at = k0 + at >= Kd ? k0 - at : k0, hi_at = k0 + at + 64 >= Kd ? k0 - at : k0 + 64;
            lo[i] = ldg128(tp[i] + lo_at);
            hi[i] = ldg128(tp[i] + hi_at);
        }
    };
    // Loads are issued without a condition (the compiler counts those in flight behind the tokens, and would wait for all of
    // them where two paths meet); the few past the end come from the L2
#pragma unroll
    for (int s = 0; s < S - 1; ++s) issue(s, s, tlo[s], thi[s]);
    for (int s0 = 0; s0 < steps; s0 += S) {
#pragma unroll
        for (int st = 0; st < S; ++st) {
            const int step = s0 + st;
            if (step >= steps) break;
            BM_WAIT_OWN((S - 2) * PER)
            constexpr int LAST = S - 1;
            issue(step + LAST, (st + LAST) % S, tlo[(st + LAST) % S], thi[(st + LAST) % S]);      // the stage read last
            const int kt = block_of(step);
            const uint8_t *ws = mine + st * 4096;
            Operand<WIDE> wf[WB];
#pragma unroll
            for (int b = 0; b < WB; ++b) wf[b].set(lds_operand(ws, b * 16 + l16, q4));
            const float sw = s_sw[kt];
            const int rem = Kd - kt * 128;
#pragma unroll
            for (int i = 0; i < TB; ++i) {
                u32x4 lo = tlo[st][i], hi = thi[st][i];
#pragma unroll
                for (int u = 0; u < 4; ++u) {                          // pieces past the row's end count nothing
                    lo[u] = q4 * 16 < rem ? lo[u] : 0u;
                    hi[u] = q4 * 16 + 64 < rem ? hi[u] : 0u;
                }
                Operand<WIDE> to;
                to.set(i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]});
                const float f = s_sa[min(i * 16 + l16, rows - 1) * kb_n + kt] * sw;
#pragma unroll
                for (int b = 0; b < WB; ++b) {
                    const f32x4 r = block_product(wf[b], to);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[b][i][v] = fmaf(r[v], f, acc[b][i][v]);
                }
            }
        }
    }
    BM_WAIT_OWN(0)                                                     // nothing may land in LDS that others use, or behind the end
    constexpr int PAIRS = WB * TB;
    auto put = [&](int b, int i, f32x4 v) {
        const int col = n0 + q4 * 8 + b * 4, r = row0 + i * 16 + l16;
        if (col < N && r < row_end) store4(p, (size_t)r * N + col, v);
    };
    __syncthreads();                                                   // every ring is done with: the parts take its place
    float *red = reinterpret_cast<float *>(ring);                      // [wave][pair of blocks][lane], four at a time
#pragma unroll
    for (int pair = 0; pair < PAIRS; ++pair) *reinterpret_cast<f32x4 *>(red + ((wave * PAIRS + pair) * 64 + lane) * 4) = acc[pair / TB][pair % TB];
    __syncthreads();
    for (int pair = wave; pair < PAIRS; pair += STREAM_WAVES) {
        f32x4 sum = 0.0f;
#pragma unroll
        for (int k = 0; k < STREAM_WAVES; ++k) sum += *reinterpret_cast<const f32x4 *>(red + ((k * PAIRS + pair) * 64 + lane) * 4);
        put(pair / TB, pair % TB, sum);
    }
}

template <bool WIDE>
__global__ void __launch_bounds__(STREAM_WAVES * WAVE, 2) stream_kernel(ProductParams p, int bm) {
    constexpr int COLS = 32, RING = STREAM_WAVES * 4 * 4096, MAX_KB = MAX_PRODUCT_KD / SCALE_BLOCK;
    __shared__ __attribute__((aligned(1024))) uint8_t ring[RING + (MAX_KB + STREAM_SCALES) * 4];
    float *const s_sw = reinterpret_cast<float *>(ring + RING), *const s_sa = s_sw + MAX_KB;
    TileTable &tt = *reinterpret_cast<TileTable *>(ring);                   // gone when the ring is filled
    if (threadIdx.x < WAVE) build_tile_table(p, bm, tt);
    __syncthreads();
    const int n_nt = (p.N + COLS - 1) / COLS;
    const Share share = my_share(__builtin_amdgcn_readfirstlane(tt.first[p.n_groups]) * n_nt);
    if (share.begin >= share.end) return;
    const Tile t = tile_at(p, tt, bm, n_nt, share.begin);
    const Matrices m = matrices_of<false>(p, t.group);
    const int rows = min(t.row_end - t.row0, bm), kb_n = (p.Kd + SCALE_BLOCK - 1) / SCALE_BLOCK;
    for (int kb = threadIdx.x; kb < kb_n; kb += STREAM_WAVES * WAVE) s_sw[kb] = ldg_f32(m.s0 + (size_t)(t.nt * COLS / SCALE_BLOCK) * kb_n + kb);
    for (int r = threadIdx.x >> 6; r < rows; r += STREAM_WAVES) {
        const float *src = p.a_scale + (size_t)source_row(p, t.row0 + r, t.row_end) * kb_n;
        for (int k = threadIdx.x & 63; k < kb_n; k += 64) s_sa[r * kb_n + k] = ldg_f32(src + k);
    }
    __syncthreads();
    if (rows <= 16) stream_tile<1, WIDE>(p, t, rows, ring, s_sw, s_sa, m.w0);
    else stream_tile<2, WIDE>(p, t, rows, ring, s_sw, s_sa, m.w0);
}

// A bound on the row tiles of any grouping of the rows, times the column tiles.
static long long tiles_bound(long long rows, int N, int n_groups, int bm, int cols) {
    const long long groups = n_groups < rows ? n_groups : rows;
    return (rows / bm + groups) * ((N + cols - 1) / cols);
}

bool product_grid_ok(long long rows, int N, int n_groups) {
    return tiles_bound(rows, N, n_groups, 8, 32) < (1ll << 31) - 8;       // no tile is smaller
}

template <int BM, int BN, int WMN, int WNN, int KG, int SW, int ST, int PER_UNIT, bool DUAL, bool WIDE>
static void launch_tiles(const ProductParams &p, hipStream_t st) {
    const long long tiles = (tiles_bound(p.rows, p.N, p.n_groups, BM, DUAL ? BN / 2 : BN) + 7) / 8 * 8;
    const dim3 grid((unsigned)(tiles < 256 * PER_UNIT ? tiles : 256 * PER_UNIT)), block(WMN * WNN * KG * 64);
    // 32-bit offsets into a, whole steps (see tiles_kernel)
    const bool near = p.Kd % (KG * SCALE_BLOCK) == 0 && p.Kd >= MIN_STEPS * KG * SCALE_BLOCK && (long long)p.a_rows * p.Kd < (1ll << 32);
    if (near) hipLaunchKernelGGL((tiles_kernel<BM, BN, WMN, WNN, KG, SW, ST, PER_UNIT, DUAL, WIDE, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((tiles_kernel<BM, BN, WMN, WNN, KG, SW, ST, PER_UNIT, DUAL, WIDE, false>), grid, block, 0, st, p);
}

template <bool WIDE>
static void launch_stream(const ProductParams &p, hipStream_t st) {
    const int kb_n = (p.Kd + SCALE_BLOCK - 1) / SCALE_BLOCK, bm = 32 * kb_n <= STREAM_SCALES ? 32 : 8;
    const long long tiles = (tiles_bound(p.rows, p.N, p.n_groups, bm, 32) + 7) / 8 * 8;
    hipLaunchKernelGGL((stream_kernel<WIDE>), dim3((unsigned)tiles), dim3(STREAM_WAVES * WAVE), 0, st, p, bm);
}

// Tiles by the rows a group has on average (groups of experts that are not resident are empty: the live ones have more).  A
// larger tile reads its operands fewer times and computes on more rows that are none; with fewer than a tile for each of the 256
// units the smaller one wins.  Measured in us, 14336 -> 4096 of 8 groups, rows a group and tiles of 192 | 128 | 64 | 32 rows:
//   256: 211 251 273 369    128: 203 149 183 221    64: 304 145 158 161    32: 278 145 110 119    8: 174 114 88 68
// and 768 -> 2048 of 128 groups:
//   512: 208 240 298 433     64: 55 46 53 72        32: 46 36 35 43        16: 50 35 31 34        4: 33 21 20 19
// Tiles of 128 rows: 256 columns for long reductions of 8-bit instructions (14336 -> 4096 of 1024 rows in 8 groups: 134 us against 147),
// else 128 and two workgroups a unit (768 -> 2048 of 8192 rows in 128 groups: 46 against 49; of 512 rows, 14336 -> 4096 in fp32: 149 against 187).
// Fewer than 256 tiles of 128 rows, but more of 64: a unit each and four stages (1000 x 2080 x 1440 in fp32 | bf16: 22.8 | 17.3 us against
// 25.4 | 18.4 on 64 rows; 1800 x 2048 x 4096: 47.2 | 32.4 against 54.2 | 37.3; with 256 tiles of 64 rows these win, 512 x 4096 x 4096: 34.9
// against 39.8).
// Tiles of 32 rows: at 2048 -> .. and beyond the reduction is worth two parts within a workgroup (14336 -> 4096 of 16 rows: 56 us
// against 69; of 512 rows, 768 -> 2048: 59 against 43).  Up to 128 tiles the streaming kernel takes 9.4 us for 1 x 4096 x 4096 against
// 17, 18.5 for 64 x 1024 x 8192 against 34; with more it is even (58.6 against 60 for 16 rows of 14336 -> 4096 in 8 groups).
template <bool WIDE>
static void launch_product_t(const ProductParams &p, hipStream_t st) {
    const long long avg = p.rows / p.n_groups;
    auto tiles = [&](int bm, int bn) { return tiles_bound(p.rows, p.N, p.n_groups, bm, bn); };
    const bool few_tiles = avg >= 128 && p.rows * (long long)((p.N + 127) / 128) > 256 * 64;
    const bool long_rows = !WIDE && p.Kd >= 4096 && avg >= 128 && tiles(128, 256) >= 256;
    if (avg >= 256 && tiles(192, 256) >= 256) launch_tiles<192, 256, 2, 4, 1, 3, 2, 1, false, WIDE>(p, st);
    else if (long_rows) {
        if constexpr (!WIDE) launch_tiles<128, 256, 2, 4, 1, 3, 3, 1, false, false>(p, st);
    } else if (avg >= 48 && tiles(128, 128) >= 256) launch_tiles<128, 128, 2, 4, 1, 2, 2, 2, false, WIDE>(p, st);
    else if (few_tiles) launch_tiles<128, 128, 2, 4, 1, 4, 4, 1, false, WIDE>(p, st);
    else if (avg >= (p.Kd >= 2048 ? 32 : 16) && tiles(64, 128) >= 256) launch_tiles<64, 128, 2, 4, 1, 3, 3, 2, false, WIDE>(p, st);
    else if (p.Kd >= 2048 && tiles(32, 128) <= 128) launch_stream<WIDE>(p, st);
    else if (p.Kd >= 2048) launch_tiles<32, 128, 1, 4, 2, 3, 3, 1, false, WIDE>(p, st);
    else launch_tiles<32, 128, 2, 4, 1, 3, 3, 2, false, WIDE>(p, st);
}

int launch_product(const ProductParams &p, hipStream_t st) {
    if (p.c_f32) launch_product_t<true>(p, st);
    else launch_product_t<false>(p, st);
    return launch_status(__func__);
}

// As above, with 128 columns of both matrices a tile.  Measured in us, gate/up 4096 -> 14336 of 8 groups, rows a group and tiles
// of 192 | 128 | 32 rows:   1024: 1670 . .    256: 534 549 731    128: 324 330 416    64: . 218 240    16: 186 169 130
// and 2048 -> 768 of 128 groups:   512: 472 490 670    128: . 153 198    64: . 110 104    32: 104 80 69
// From 96 rows a group (64 for long reductions) the least of rounds over the units times what a step of 128 takes, in us (2.1 and 1.55 for
// tiles of 192 and 128; of 32 rows 0.85, two on a unit 1.45), decides: 300 rows 4096 -> 4096 take 74 | 56 | 49 us, 1024 rows 81 | 67 | 102, 2000 rows
// 2880 -> 2880 75 | 95 | 116, 4 groups of 300 rows 2048 -> 768 42 | 32 | 21.
// Tiles of 32 rows: four stages and one workgroup a unit, or two and two.  The first wins where tiles are fewer than units (two rows,
// 4096 -> 14336: 41 us against 49) and in the last round of long reductions, whose tiles have a unit each (4096 -> 8192, 640 tiles: 121
// against 130, 768: 138 against 139, 1024: 183 against 182); the second where a second round would hold few tiles (2048 -> 768 of 512 rows in
// 128 groups, half of them empty: 46 against 37) and with more rows a tile (4096 -> 14336 of 128 rows in 8 groups: 137 against 130; of one
// group of 128 rows 72 against 54).
int launch_swiglu(const ProductParams &p, hipStream_t st) {
    const long long avg = p.rows / p.n_groups;
    const double groups = p.n_groups < p.rows ? p.n_groups : p.rows, columns = (p.N + SCALE_BLOCK - 1) / SCALE_BLOCK;
    auto tiles = [&](int bm) { return ((double)p.rows / bm + 0.5 * groups) * columns; };      // half a tile of every group is no row
    auto rounds = [](double tiles, int at_once) { return tiles > at_once ? tiles / at_once : 1.0; };
    const double t32 = tiles(32) <= 256 ? 0.85 : 1.45 * rounds(tiles(32), 512), t128 = 1.55 * rounds(tiles(128), 256), t192 = 2.1 * rounds(tiles(192), 256);
    const bool many = avg >= (p.Kd >= 4096 ? 64 : 96);
    if (avg >= 256 && t192 <= t128 && t192 <= t32) launch_tiles<192, 256, 2, 4, 1, 3, 2, 1, true, true>(p, st);
    else if (many && t128 <= t32) launch_tiles<128, 256, 2, 4, 1, 3, 3, 1, true, true>(p, st);
    else if (avg < 32 && tiles_bound(p.rows, p.N, p.n_groups, 32, SCALE_BLOCK) <= (p.Kd >= 4096 ? 1024 : 512)) launch_tiles<32, 256, 1, 8, 1, 4, 4, 1, true, true>(p, st);
    else launch_tiles<32, 256, 1, 8, 1, 2, 2, 2, true, true>(p, st);
    return launch_status(__func__);
}

}  // namespace bm
