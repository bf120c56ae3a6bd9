// Low-rank adapters of many requests beside a shared projection:
//   y[t] = base[t] + scale[a] * B[a] (A[a] x[t]),   a = the adapter of row t
//
// Three launches: rows are grouped by adapter (chunks of 1024 rows, each on its own), u = A x of a tile of up to 64 rows of one
// adapter (the reduction cut into parts over the chip), then B u is added to base on the way to y.  Up to 64 rows group themselves in
// the other two, and a few rows of a small rank take one launch.  A and B are read once for each tile, x once, base and y once: many
// rows are bound by base and y (8192 rows of 2048 -> 4096, rank 16: 134 MB in 29 us, a copy's rate; 46 us in all where the inputs lie in
// the memory-side cache, 57 where they do not), few by launches and trips to memory.  u is held in fp32.
#include "bm_adapters.h"

namespace bm {

namespace {

// A line of 128 bytes of a row and its matrix instructions: lane l has row l % 16 and the 16 bytes l / 16 of a half line.
struct Bf16Line {
    static constexpr int VALUES = 64, SIZE = 2;
    static __device__ __forceinline__ f32x4 mac(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
    }
};
struct F32Line {
    static constexpr int VALUES = 32, SIZE = 4;
    static __device__ __forceinline__ f32x4 mac(u32x4 a, u32x4 b, f32x4 c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// 16 bytes at an address that is a multiple of SIZE bytes
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
template <int SIZE>
__device__ __forceinline__ u32x4 load_any(const char *at) {
    if constexpr (SIZE == 4) return *(const BM_GLOBAL u32x4_at4 *)at;
    else return *(const BM_GLOBAL u32x4_at2 *)at;
}
template <int SIZE>
__device__ __forceinline__ void store_any(char *at, u32x4 v) {
    if constexpr (SIZE == 4) *(BM_GLOBAL u32x4_at4 *)at = v;
    else *(BM_GLOBAL u32x4_at2 *)at = v;
}

// 16 bytes of a row, its values from `at` on (a multiple of 16 bytes), zeros from value `end` on.  WHOLE: the row is at a 16-byte
// address and holds a multiple of 16 bytes; the values behind `end`, which lie in the row, are read and cleared.
template <typename L, bool WHOLE>
__device__ __forceinline__ u32x4 piece(const char *row, int at, int end, int row_end) {
    constexpr int PER = 16 / L::SIZE;
    u32x4 v = {0, 0, 0, 0};
    if constexpr (WHOLE) {
        v = ldg128(row + (size_t)(at < row_end ? at : 0) * L::SIZE);
        if (at >= end) v = u32x4{0, 0, 0, 0};
        else if (at + PER > end) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (at + i >= end) {
                    if constexpr (L::SIZE == 4) v[i] = 0;
                    else v[i / 2] &= i % 2 ? 0x0000ffffu : 0xffff0000u;
                }
        }
    } else if (at + PER <= end) {
        v = load_any<L::SIZE>(row + (size_t)at * L::SIZE);
    } else {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (at + i < end) {
                if constexpr (L::SIZE == 4) v[i] = *(const BM_GLOBAL uint32_t *)(row + (size_t)(at + i) * 4);
                else v[i / 2] |= (uint32_t)*(const BM_GLOBAL uint16_t *)(row + (size_t)(at + i) * 2) << 16 * (i % 2);
            }
    }
    return v;
}

__device__ __forceinline__ int rank_of(const AdapterParams &p, int a) {
    return p.ranks == nullptr ? p.rank : min(max(ldg_i32(p.ranks + a), 0), p.rank);
}

// ---------------------------------------------------------------------------
// The chunk's rows in the order of their adapters, rows of one adapter in their own order, and tiles of up to 64 of them.
// A row's place among its adapter's rows: those of its wave before it by ballots, and those of earlier waves from counts.
// Neighbouring tiles - often of one adapter - go to different dies.  (Runs of them on one die read that adapter's matrices once a die,
// and took 53 us instead of 46 for 8192 rows of 2048 -> 4096, rank 16.)
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(ADAPTER_CHUNK) adapter_group_kernel(AdapterParams p) {
    constexpr int MOST = ADAPTER_CHUNK / 64, KEYS = BM_MAX_ADAPTERS + 8;
    __shared__ uint16_t count[MOST][KEYS];
    __shared__ int first_row[KEYS], first_tile[KEYS];
    __shared__ int wave_rows[MOST], wave_tiles[MOST];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, waves = blockDim.x >> 6, chunk = blockIdx.x;
    const int row = chunk * ADAPTER_CHUNK + tid, keys = p.n + 1;
    for (int k = tid; k < keys; k += blockDim.x)
        for (int w = 0; w < waves; ++w) count[w][k] = 0;
    int key = -1;
    if (row < p.rows) {
        key = ldg_i32(p.adapter + row);
        if ((unsigned)key >= (unsigned)p.n) key = p.in_place ? -1 : p.n;
    }
    __syncthreads();
    int rank = 0;
    for (unsigned long long left = __ballot(key >= 0); left != 0;) {
        const int first = __builtin_ctzll(left), k = __builtin_amdgcn_readlane(key, first);
        const unsigned long long same = __ballot(key == k);
        if (key == k) rank = __popcll(same & ((1ull << lane) - 1));
        if (lane == first) count[wave][k] = (uint16_t)__popcll(same);
        left &= ~same;
    }
    __syncthreads();
    // per key: the rows of earlier waves, then rows and tiles of the keys before it
    int rows_so_far = 0, tiles_so_far = 0;
    for (int k0 = 0; k0 < keys; k0 += blockDim.x) {
        const int k = k0 + tid;
        int total = 0;
        if (k < keys)
            for (int w = 0; w < waves; ++w) {
                const int c = count[w][k];
                count[w][k] = (uint16_t)total;
                total += c;
            }
        const int tiles = (total + ADAPTER_TILE - 1) / ADAPTER_TILE;
        int r = total, t = tiles;          // inclusive sums over the wave
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int ro = __shfl_up(r, d, WAVE), to = __shfl_up(t, d, WAVE);
            if (lane >= d) { r += ro; t += to; }
        }
        if (lane == 63) { wave_rows[wave] = r; wave_tiles[wave] = t; }
        __syncthreads();
        int before_rows = rows_so_far, before_tiles = tiles_so_far;
        for (int w = 0; w < waves; ++w) {
            const int wr = wave_rows[w], wt = wave_tiles[w];
            if (w < wave) { before_rows += wr; before_tiles += wt; }
            rows_so_far += wr;
            tiles_so_far += wt;
        }
        if (k < keys) {
            first_row[k] = before_rows + r - total;
            first_tile[k] = before_tiles + t - tiles;
        }
        __syncthreads();
    }
    AdapterTile *const out = p.tiles + (size_t)chunk * p.max_tiles;
    for (int k = tid; k < keys; k += blockDim.x) {
        const int start = first_row[k], t0 = first_tile[k];
        const int total = (k + 1 < keys ? first_row[k + 1] : rows_so_far) - start;
        for (int i = 0; i * ADAPTER_TILE < total; ++i) out[t0 + i] = AdapterTile{k, start + i * ADAPTER_TILE, min(ADAPTER_TILE, total - i * ADAPTER_TILE), 0};
    }
    for (int i = tiles_so_far + tid; i < p.max_tiles; i += blockDim.x) out[i] = AdapterTile{0, 0, 0, 0};
    if (key >= 0) p.order[(size_t)chunk * ADAPTER_CHUNK + first_row[key] + count[wave][key] + rank] = row;
}

// ---------------------------------------------------------------------------
// A workgroup's tile: its adapter and its rows, in LDS.  Up to 64 rows need no grouping: every wave finds the tile by ballots, which takes
// less than the launch and the round trip to memory of a kernel for it.
// ---------------------------------------------------------------------------
constexpr int WAVES = 4;
constexpr int WANTED = 256, MAX_SPLITS = 8;       // workgroups of the launch, parts of the reduction at most

struct TileView {
    int adapter, count;           // adapter n: rows without one
    size_t place;                 // FEW: a row's place in u is its number, else place + its number in the tile
};

template <bool FEW>
__device__ __forceinline__ bool find_tile(const AdapterParams &p, int *rows, TileView &view) {
    const int tid = threadIdx.x, lane = lane_id();
    if constexpr (FEW) {
        int key = -1;
        if (lane < p.rows) {
            key = ldg_i32(p.adapter + lane);
            if ((unsigned)key >= (unsigned)p.n) key = p.in_place ? -1 : p.n;
        }
        unsigned long long left = __ballot(key >= 0), mine = 0;
        for (int i = 0; i <= (int)blockIdx.x; ++i) {
            left &= ~mine;
            if (left == 0) return false;
            view.adapter = __builtin_amdgcn_readlane(key, __builtin_ctzll(left));
            mine = __ballot(key == view.adapter);
        }
        view.count = __popcll(mine);
        view.place = 0;
        if (tid < 64 && key == view.adapter) rows[__popcll(mine & ((1ull << lane) - 1))] = lane;
    } else {
        const int chunk = blockIdx.z;
        const AdapterTile t = p.tiles[(size_t)chunk * p.max_tiles + blockIdx.x];
        if (t.count == 0) return false;
        view.adapter = t.adapter;
        view.count = t.count;
        view.place = (size_t)chunk * ADAPTER_CHUNK + t.start;
        if (tid < t.count) rows[tid] = ldg_i32(p.order + view.place + tid);
    }
    return true;
}
template <bool FEW>
__device__ __forceinline__ size_t place_in_u(const TileView &view, const int *rows, int i) { return FEW ? (size_t)rows[i] : view.place + i; }

__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------
// u = A x of a tile and a part of the reduction.  Matrix rows are A's, columns the tile's rows: a lane ends with four neighbouring values
// of u.  NR: blocks of 16 ranks.
// Up to 16 rows: the four waves take every fourth line each, straight from memory, and add their sums as (w0 + w2) + (w1 + w3).
// More: whole lines of x and A go straight into a ring of LDS stages (row r's 16-byte piece c at slot c ^ (r & 7)), one wait and one
// barrier a line; the waves share the tile's 64 rows and the ranks.  Direct loads for 64 rows and 128 ranks as well left a wave a
// SIMD for their registers: 2000 rows of 4096 -> 128 in 28.8 us.
// ---------------------------------------------------------------------------
#define BM_LDS __attribute__((address_space(3)))

template <typename L, bool WHOLE, bool FEW, int NR, int TS>
__device__ __forceinline__ void shrink_few(const AdapterParams &p, const TileView &tile, const int *rows, int split, f32x4 (*sums)[64]) {
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const int lines = (p.Kd + L::VALUES - 1) / L::VALUES;
    const int begin = (int)((long long)split * lines / p.splits), end = (int)((long long)(split + 1) * lines / p.splits);
    const int blocks = (rank_of(p, tile.adapter) + 15) >> 4;                  // of ranks that count
    const char *xr[TS], *ar[NR];
#pragma unroll
    for (int i = 0; i < TS; ++i) xr[i] = static_cast<const char *>(p.x) + (size_t)rows[min(i * 16 + r16, tile.count - 1)] * p.x_stride * L::SIZE;
#pragma unroll
    for (int j = 0; j < NR; ++j)
        ar[j] = static_cast<const char *>(p.a) + ((size_t)tile.adapter * p.rank + min(j * 16 + r16, p.rank - 1)) * p.Kd * L::SIZE;
    f32x4 acc[NR][TS];
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int i = 0; i < TS; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int l = begin + wave; l < end; l += WAVES) {
        u32x4 xv[TS][2], av[NR][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = l * L::VALUES + (h * 4 + kq) * (16 / L::SIZE);
#pragma unroll
            for (int i = 0; i < TS; ++i) xv[i][h] = piece<L, WHOLE>(xr[i], at, p.Kd, p.Kd);
#pragma unroll
            for (int j = 0; j < NR; ++j)
                if (j < blocks) av[j][h] = piece<L, WHOLE>(ar[j], at, p.Kd, p.Kd);
        }
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if (j >= blocks) break;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < TS; ++i) acc[j][i] = L::mac(av[j][h], xv[i][h], acc[j][i]);
        }
    }
    if (wave >= 2)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int i = 0; i < TS; ++i) sums[((wave - 2) * NR + j) * TS + i][lane] = acc[j][i];
    __syncthreads();
    if (wave < 2)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int i = 0; i < TS; ++i) {
                f32x4 &other = sums[(wave * NR + j) * TS + i][lane];
                acc[j][i] += other;
                if (wave == 1) other = acc[j][i];
            }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < TS; ++i) {
        if (i * 16 + r16 >= tile.count) continue;
        float *u = p.u + (split * (size_t)p.u_rows + place_in_u<FEW>(tile, rows, i * 16 + r16)) * p.width;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            if (j >= blocks) break;
            *(BM_GLOBAL f32x4 *)(u + j * 16 + kq * 4) = acc[j][i] + sums[(NR + j) * TS + i][lane];
        }
    }
}

template <int NR>
struct Ring {
    static constexpr int RB = NR * 16, ROWS = ADAPTER_TILE;
    static constexpr int WN = NR >= 4 ? 2 : 1, WM = WAVES / WN;                          // waves along ranks and rows
    static constexpr int TM = ROWS / WM / 16, TN = NR / WN;                              // 16 x 16 blocks of a wave
    static constexpr int BLOCKS = (ROWS + RB) / 8, LOADS = (BLOCKS + WAVES - 1) / WAVES; // of 8 rows; a wave and stage
    static constexpr int STAGES = NR == 8 ? 3 : 4, STAGE = BLOCKS * 64;   // 16-byte pieces of a stage: two workgroups a unit
};

template <typename L, bool FEW, int NR>
__device__ __forceinline__ void shrink_ring(const AdapterParams &p, const TileView &tile, const int *rows, int split, u32x4 *smem) {
    using R = Ring<NR>;
    constexpr int S = R::STAGES, TM = R::TM, TN = R::TN;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, kq = lane >> 4;
    const int bytes = p.Kd * L::SIZE, lines = (bytes + 127) >> 7, rank = rank_of(p, tile.adapter);
    const int begin = (int)((long long)split * lines / p.splits), end = (int)((long long)(split + 1) * lines / p.splits);
    if (begin >= end || rank == 0) return;                                   // (splits <= lines: no part is empty)
    const char *from[R::LOADS];
    int to[R::LOADS];
#pragma unroll
    for (int j = 0; j < R::LOADS; ++j) {
        int block = wave + WAVES * j;
        if (block >= R::BLOCKS) block = wave % R::BLOCKS;                    // (a repeated load of what is there)
        const int row = block * 8 + (lane >> 3);
        from[j] = row < R::ROWS ? static_cast<const char *>(p.x) + (size_t)rows[min(row, tile.count - 1)] * p.x_stride * L::SIZE
                                : static_cast<const char *>(p.a) + ((size_t)tile.adapter * p.rank + min(row - R::ROWS, rank - 1)) * bytes;
        to[j] = block * 64;
    }
    const int piece_at = ((lane & 7) ^ (lane >> 3)) * 16;
    auto load = [&](int l, int slot) {
        const int at = min(l, end - 1) * 128 + piece_at, within = at < bytes ? at : 0;   // (behind a row's end: cleared when read)
#pragma unroll
        for (int j = 0; j < R::LOADS; ++j)
            __builtin_amdgcn_global_load_lds((const BM_GLOBAL void *)(from[j] + within), (BM_LDS void *)(smem + slot * R::STAGE + to[j]), 16, 0, 0);
    };
    const int m0 = wave % R::WM * (TM * 16), n0 = wave / R::WM * (TN * 16);
    const bool idle = m0 >= tile.count || n0 >= rank;                        // (the wave's part of the tile holds nothing)
    f32x4 acc[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S - 1; ++i) load(begin + i, i);
    int now = 0, free = S - 1;
    for (int l = begin; l < end; ++l) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S - 2) * R::LOADS) : "memory");
        load(l + S - 1, free);
        const u32x4 *st = smem + now * R::STAGE;
        if (!idle)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 x[TM], a[TN];
                const int c = (h * 4 + kq) ^ (r16 & 7);
#pragma unroll
                for (int i = 0; i < TM; ++i) x[i] = st[(m0 + i * 16 + r16) * 8 + c];
#pragma unroll
                for (int j = 0; j < TN; ++j) a[j] = st[(R::ROWS + n0 + j * 16 + r16) * 8 + c];
                if (l * 128 + 128 > bytes) {                                 // the row ends in this line
                    const bool in = l * 128 + (h * 4 + kq) * 16 < bytes;
#pragma unroll
                    for (int i = 0; i < TM; ++i) x[i] = in ? x[i] : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < TN; ++j) a[j] = in ? a[j] : u32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[j][i] = L::mac(a[j], x[i], acc[j][i]);
            }
        free = now;
        now = now + 1 == S ? 0 : now + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");                       // the last loads are through before the workgroup ends
    if (idle) return;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int row = m0 + i * 16 + r16;
        if (row >= tile.count) continue;
        float *u = p.u + (split * (size_t)p.u_rows + place_in_u<FEW>(tile, rows, row)) * p.width + n0 + kq * 4;
#pragma unroll
        for (int j = 0; j < TN; ++j)
            if (n0 + j * 16 < rank) *(BM_GLOBAL f32x4 *)(u + j * 16) = acc[j][i];
    }
}

template <typename L, bool WHOLE, bool FEW, int NR>
__global__ void __launch_bounds__(WAVES * 64) adapter_shrink_kernel(AdapterParams p) {
    using R = Ring<NR>;
    constexpr int TS = WHOLE || NR >= 8 ? 1 : NR >= 4 ? 2 : ADAPTER_TILE / 16;               // blocks of 16 rows at a time straight from memory
    __shared__ u32x4 smem[WHOLE ? R::STAGES * R::STAGE : 2 * NR * TS * 64];
    static_assert(R::STAGES * R::STAGE >= 2 * NR * 64, "holds the waves' sums of up to 16 rows");
    __shared__ int rows[ADAPTER_TILE];
    TileView tile;
    if (!find_tile<FEW>(p, rows, tile) || tile.adapter >= p.n) return;
    __syncthreads();
    f32x4(*sums)[64] = reinterpret_cast<f32x4(*)[64]>(smem);
    if constexpr (WHOLE) {
        if (tile.count > 16) {
            // by the adapter's own rank: what lies behind it is neither loaded nor multiplied
            const int rank = rank_of(p, tile.adapter);
            if (NR >= 2 && rank <= 16) shrink_ring<L, FEW, 1>(p, tile, rows, blockIdx.y, smem);
            else if (NR >= 4 && rank <= 32) shrink_ring<L, FEW, NR >= 2 ? 2 : 1>(p, tile, rows, blockIdx.y, smem);
            else if (NR >= 8 && rank <= 64) shrink_ring<L, FEW, NR >= 4 ? 4 : 1>(p, tile, rows, blockIdx.y, smem);
            else shrink_ring<L, FEW, NR>(p, tile, rows, blockIdx.y, smem);
        }
        else shrink_few<L, true, FEW, NR, 1>(p, tile, rows, blockIdx.y, sums);
    } else {
        // other lengths and addresses
        for (int i = 0; i < tile.count; i += 16 * TS) {
            TileView part{tile.adapter, min(16 * TS, tile.count - i), tile.place + i};
            shrink_few<L, false, FEW, NR, TS>(p, part, rows + i, blockIdx.y, sums);
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------------------
// y = base + scale * B u of a tile and a range of columns.  Matrix rows are B's, columns the tile's rows.  Two matrix blocks cover
// 32 columns, their rows dealt so that a lane ends with eight neighbouring ones: block j, row 4 q + v is column
// (j / 2) * 32 + q * 8 + (j % 2) * 4 + v.  A wave takes 64 columns, 32 with ranks beyond 32.
// bf16: u goes to the matrix unit as the sum of two bf16 values, each the rest of those before it rounded (16 bits of u), of three
// (all 24) where y is fp32, which would show the difference: 1.6e-6 of an fp32 y with two, rank 128.  Up to 16 ranks the
// first two lie in one instruction's 32.
// ---------------------------------------------------------------------------
constexpr int RANGE = 256;               // columns of a workgroup
constexpr int expand_waves(int nr) { return nr >= 4 ? 8 : 4; }

// The values of u in the form of the matrix operand: [part][k block][row block][lane] 16 bytes
template <typename L, bool YF32, int NR>
struct Expanded {
    static constexpr bool F32 = L::SIZE == 4;
    static constexpr int KB = F32 ? NR : (NR + 1) / 2;       // blocks of 16 (fp32) or 32 ranks
    static constexpr int PARTS = F32 ? 1 : NR == 1 ? (YF32 ? 2 : 1) : (YF32 ? 3 : 2);
    static constexpr int WAVES = expand_waves(NR), H = RANGE / WAVES / 32;   // waves, 32 columns at a time of each
    u32x4 v[PARTS][KB][ADAPTER_TILE / 16][64];
};

// The bf16 values of a pair, and what they leave of it.  The largest number of bf16 is below fp32's: what lies above it, infinities and
// what is no number leave the rest to the last part, which is rounded as it comes.
template <bool LAST>
__device__ __forceinline__ uint32_t take_bf16(float &a, float &b) {
    if constexpr (LAST) return pack_bf16x2(a, b);
    constexpr float MOST = 0x1.fep127f;
    const uint32_t v = pack_bf16x2(__builtin_amdgcn_fmed3f(a, -MOST, MOST), __builtin_amdgcn_fmed3f(b, -MOST, MOST));
    a -= __builtin_bit_cast(float, v << 16);
    b -= __builtin_bit_cast(float, v & 0xffff0000u);
    return v;
}

// A lane's values of u (eight ranks, four in fp32) in their places
template <typename L, bool YF32, int NR>
__device__ __forceinline__ void put_u(float (&v)[8], int kb, int i, int lane, Expanded<L, YF32, NR> &out) {
    using X = Expanded<L, YF32, NR>;
    const int kq = lane >> 4;
    if constexpr (X::F32) {
        out.v[0][kb][i][lane] = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
    } else {
        constexpr int VALUES = NR == 1 ? X::PARTS + 1 : X::PARTS;
        u32x4 part[VALUES];
#pragma unroll
        for (int j = 0; j < VALUES; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) part[j][c] = j + 1 < VALUES ? take_bf16<false>(v[2 * c], v[2 * c + 1]) : take_bf16<true>(v[2 * c], v[2 * c + 1]);
        if constexpr (NR == 1) {                             // ranks 0 to 15 twice: the first part, then the second
            out.v[0][0][i][lane] = kq < 2 ? part[0] : part[1];
            if constexpr (YF32) out.v[1][0][i][lane] = kq < 2 ? part[2] : u32x4{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int j = 0; j < X::PARTS; ++j) out.v[j][kb][i][lane] = part[j];
        }
    }
}

template <typename L, bool YF32, bool FEW, int NR>
__device__ __forceinline__ void stage_u(const AdapterParams &p, const TileView &tile, const int *rows, int rank, Expanded<L, YF32, NR> &out) {
    using X = Expanded<L, YF32, NR>;
    constexpr int AHEAD = 4;                                 // (with 8 of them a unit holds fewer waves: 8192 rows 2048 -> 4096 48 -> 52 us)
    constexpr int Q = X::F32 ? 1 : 2;                        // pieces of four ranks: 8 ranks in bf16, 4 in fp32
    const size_t step = (size_t)p.u_rows * p.width;
    const int blocks = (tile.count + 15) >> 4, kbs = (rank + (X::F32 ? 15 : 31)) / (X::F32 ? 16 : 32);
    for (int at = threadIdx.x; at < kbs * blocks * 64; at += X::WAVES * 64) {
        const int lane = at & 63, i = (at >> 6) % blocks, kb = (at >> 6) / blocks;
        const int kq = lane >> 4, row = min(i * 16 + (lane & 15), tile.count - 1);
        const int r0 = X::F32 ? kb * 16 + kq * 4 : NR == 1 ? (kq & 1) * 8 : kb * 32 + kq * 8;
        const float *u = p.u + place_in_u<FEW>(tile, rows, row) * p.width;
        f32x4 sum[Q];
        int from[Q];
#pragma unroll
        for (int h = 0; h < Q; ++h) {
            sum[h] = f32x4{0.f, 0.f, 0.f, 0.f};
            from[h] = r0 + 4 * h < rank ? r0 + 4 * h : 0;    // (blocks of 16 ranks behind the last one are not written)
        }
        for (int s0 = 0; s0 < p.splits; s0 += AHEAD) {       // so many parts' loads on their way
            f32x4 w[AHEAD][Q];
#pragma unroll
            for (int s = 0; s < AHEAD; ++s)
#pragma unroll
                for (int h = 0; h < Q; ++h) w[s][h] = *(const BM_GLOBAL f32x4 *)(u + min(s0 + s, p.splits - 1) * step + from[h]);
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                if (s0 + s >= p.splits) break;
#pragma unroll
                for (int h = 0; h < Q; ++h) sum[h] += w[s][h];
            }
        }
        float v[8];
#pragma unroll
        for (int h = 0; h < Q; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c) v[4 * h + c] = r0 + 4 * h + c < rank ? sum[h][c] : 0.0f;
        put_u<L, YF32, NR>(v, kb, i, lane, out);
    }
}

// Eight values of a row of base or y from column n on (a multiple of 8), as they lie in memory
template <bool YF32>
struct Eight {
    u32x4 v[YF32 ? 2 : 1];
    template <bool WHOLE>
    __device__ __forceinline__ void load(const char *row, int n, int end) {
        constexpr int SIZE = YF32 ? 4 : 2, PER = 16 / SIZE;
#pragma unroll
        for (int i = 0; i < 8 / PER; ++i) {
            const int at = n + i * PER;
            if constexpr (WHOLE) {
                v[i] = ldg128(row + (size_t)(at < end ? at : 0) * SIZE);
            } else if (at + PER <= end) {
                v[i] = load_any<SIZE>(row + (size_t)at * SIZE);
            } else {
                v[i] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int c = 0; c < PER; ++c)
                    if (at + c < end) {
                        if constexpr (YF32) v[i][c] = (uint32_t)ldg_i32(row + (size_t)(at + c) * 4);
                        else v[i][c / 2] |= (uint32_t)*(const BM_GLOBAL uint16_t *)(row + (size_t)(at + c) * 2) << 16 * (c % 2);
                    }
            }
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void store(char *row, int n, int end) const {
        constexpr int SIZE = YF32 ? 4 : 2, PER = 16 / SIZE;
#pragma unroll
        for (int i = 0; i < 8 / PER; ++i) {
            const int at = n + i * PER;
            if constexpr (WHOLE) {
                if (at < end) stg128(row + (size_t)at * SIZE, v[i]);
            } else if (at + PER <= end) {
                store_any<SIZE>(row + (size_t)at * SIZE, v[i]);
            } else {
#pragma unroll
                for (int c = 0; c < PER; ++c)
                    if (at + c < end) {
                        if constexpr (YF32) *(BM_GLOBAL uint32_t *)(row + (size_t)(at + c) * 4) = v[i][c];
                        else stg16(row + (size_t)(at + c) * 2, (uint16_t)(v[i][c / 2] >> 16 * (c % 2)));
                    }
            }
        }
    }
    // + scale * (a, b)
    __device__ __forceinline__ void add(float scale, f32x4 a, f32x4 b) {
        float f[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint32_t bits = YF32 ? v[c / 4 % (YF32 ? 2 : 1)][c % 4] : v[0][c / 2 % 4] >> 16 * (c % 2) << 16;
            const float base = __builtin_bit_cast(float, bits);
            f[c] = fmaf(scale, c < 4 ? a[c % 4] : b[c % 4], base);
        }
        if constexpr (YF32) {
#pragma unroll
            for (int c = 0; c < 8; ++c) v[c / 4][c % 4] = __builtin_bit_cast(uint32_t, f[c]);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) v[0][c] = pack_bf16x2(f[2 * c], f[2 * c + 1]);
        }
    }
};

template <typename L, bool WHOLE, bool YF32, bool YWHOLE, bool FEW, int NR>
__global__ void __launch_bounds__(expand_waves(NR) * 64) adapter_expand_kernel(AdapterParams p) {
    using X = Expanded<L, YF32, NR>;
    constexpr int BLOCKS = ADAPTER_TILE / 16, YSIZE = YF32 ? 4 : 2, H = X::H;
    __shared__ X s;
    __shared__ int rows[ADAPTER_TILE];
    TileView tile;
    if (!find_tile<FEW>(p, rows, tile)) return;
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const bool none = tile.adapter >= p.n;                   // rows without an adapter: base goes to y
    const int rank = none ? 0 : rank_of(p, tile.adapter);
    const float scale = none || p.scale == nullptr ? 1.0f : ldg_f32(p.scale + tile.adapter);
    const int n0 = blockIdx.y * RANGE + wave * (32 * H), blocks = (tile.count + 15) >> 4;
    // everything that does not wait for u is on its way before it: B's rows, and base's of all of the tile
    u32x4 bv[X::KB][2 * H];
    if (rank > 0 && n0 < p.N) {
#pragma unroll
        for (int j = 0; j < 2 * H; ++j) {
            const int col = n0 + (j / 2) * 32 + (r16 >> 2) * 8 + (j % 2) * 4 + (r16 & 3);
            const char *row = static_cast<const char *>(p.b) + ((size_t)tile.adapter * p.N + min(col, p.N - 1)) * p.rank * L::SIZE;
#pragma unroll
            for (int kb = 0; kb < X::KB; ++kb) {
                const int r0 = X::F32 ? kb * 16 + kq * 4 : NR == 1 ? (kq & 1) * 8 : kb * 32 + kq * 8;
                if (kb == 0 || kb * (X::F32 ? 16 : 32) < rank) bv[kb][j] = piece<L, WHOLE>(row, r0, rank, p.rank);
            }
        }
    }
    __syncthreads();
    Eight<YF32> v[BLOCKS][H];
    int row[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
        if (i < blocks) {
            row[i] = rows[min(i * 16 + r16, tile.count - 1)];
            const char *from = static_cast<const char *>(p.base) + (size_t)row[i] * p.base_stride * YSIZE;
#pragma unroll
            for (int h = 0; h < H; ++h) v[i][h].template load<YWHOLE>(from, n0 + h * 32 + kq * 8, p.N);
        }
    if (rank > 0) {
        stage_u<L, YF32, FEW, NR>(p, tile, rows, rank, s);
        __syncthreads();
    }
    if (n0 >= p.N) return;
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        if (i >= blocks) break;
        if (rank > 0) {
            f32x4 acc[2 * H];
#pragma unroll
            for (int j = 0; j < 2 * H; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < X::KB; ++kb) {
                if (kb > 0 && kb * (X::F32 ? 16 : 32) >= rank) break;
#pragma unroll
                for (int part = 0; part < X::PARTS; ++part) {
                    const u32x4 uv = s.v[part][kb][i][lane];
#pragma unroll
                    for (int j = 0; j < 2 * H; ++j) acc[j] = L::mac(bv[kb][j], uv, acc[j]);
                }
            }
#pragma unroll
            for (int h = 0; h < H; ++h) v[i][h].add(scale, acc[2 * h], acc[2 * h + 1]);
        }
        char *to = static_cast<char *>(p.y) + (size_t)row[i] * p.y_stride * YSIZE;
        if (i * 16 + r16 < tile.count)
#pragma unroll
            for (int h = 0; h < H; ++h) v[i][h].template store<YWHOLE>(to, n0 + h * 32 + kq * 8, p.N);
    }
}

// ---------------------------------------------------------------------------
// A few rows of a small rank in one launch (one_launch): every workgroup of 256 columns makes u for itself, eight waves every eighth
// line each.  A is read once for every 256 columns, from the second-level cache; the launch and the round trip of u through memory
// that this saves take longer (one row 4096 -> 4096, rank 16: 8.2 us in two launches, see one_launch).
// ---------------------------------------------------------------------------
constexpr int ONE_WAVES = 8, ONE_ROWS = 16;
constexpr int ONE_MOST = 16, ONE_BYTES = 128 << 10, ONE_GRID = 256;     // rows; bytes of an adapter's A; workgroups
static_assert(ONE_MOST <= ONE_ROWS, "a tile's rows");

template <typename L, bool YF32>
__global__ void __launch_bounds__(ONE_WAVES * 64) adapter_one_kernel(AdapterParams p) {
    using X = Expanded<L, YF32, 1>;
    __shared__ X s;
    __shared__ f32x4 sums[ONE_WAVES][64];
    __shared__ float u[ONE_ROWS][16];
    __shared__ int rows[ADAPTER_TILE];
    TileView tile;
    if (!find_tile<true>(p, rows, tile)) return;
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const bool none = tile.adapter >= p.n;
    const int rank = none ? 0 : rank_of(p, tile.adapter);
    const float scale = none || p.scale == nullptr ? 1.0f : ldg_f32(p.scale + tile.adapter);
    const int n0 = blockIdx.y * RANGE + wave * 32;
    __syncthreads();
    const int row = rows[min(r16, tile.count - 1)];
    Eight<YF32> v;
    v.template load<true>(static_cast<const char *>(p.base) + (size_t)row * p.base_stride * (YF32 ? 4 : 2), n0 + kq * 8, p.N);
    if (rank > 0) {
        u32x4 bv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const char *at = static_cast<const char *>(p.b) + ((size_t)tile.adapter * p.N + min(n0 + (r16 >> 2) * 8 + j * 4 + (r16 & 3), p.N - 1)) * p.rank * L::SIZE;
            bv[j] = piece<L, true>(at, X::F32 ? kq * 4 : (kq & 1) * 8, rank, p.rank);
        }
        const char *xr = static_cast<const char *>(p.x) + (size_t)row * p.x_stride * L::SIZE;
        const char *ar = static_cast<const char *>(p.a) + ((size_t)tile.adapter * p.rank + min(r16, p.rank - 1)) * p.Kd * L::SIZE;
        const int lines = (p.Kd + L::VALUES - 1) / L::VALUES;
        constexpr int AHEAD = 4;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int l0 = wave; l0 < lines; l0 += ONE_WAVES * AHEAD) {
            u32x4 xv[AHEAD][2], av[AHEAD][2];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = min(l0 + i * ONE_WAVES, lines - 1) * L::VALUES + (h * 4 + kq) * (16 / L::SIZE);
                    xv[i][h] = piece<L, true>(xr, at, p.Kd, p.Kd);
                    av[i][h] = piece<L, true>(ar, at, p.Kd, p.Kd);
                }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (l0 + i * ONE_WAVES >= lines) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) acc = L::mac(av[i][h], xv[i][h], acc);
            }
        }
        sums[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
            f32x4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = sums[i][lane] + sums[i + 4][lane];
            const f32x4 sum = (q[0] + q[1]) + (q[2] + q[3]);
#pragma unroll
            for (int c = 0; c < 4; ++c) u[r16][kq * 4 + c] = sum[c];
            wave_lds_fence();
            float w[8];
            const int r0 = X::F32 ? kq * 4 : (kq & 1) * 8;
#pragma unroll
            for (int c = 0; c < (X::F32 ? 4 : 8); ++c) w[c] = r0 + c < rank ? u[r16][r0 + c] : 0.0f;
            put_u<L, YF32, 1>(w, 0, 0, lane, s);
        }
        __syncthreads();
        f32x4 d[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int part = 0; part < X::PARTS; ++part)
#pragma unroll
            for (int j = 0; j < 2; ++j) d[j] = L::mac(bv[j], s.v[part][0][0][lane], d[j]);
        v.add(scale, d[0], d[1]);
    }
    if (r16 < tile.count) v.template store<true>(static_cast<char *>(p.y) + (size_t)row * p.y_stride * (YF32 ? 4 : 2), n0 + kq * 8, p.N);
}

// 16 bytes at a time of every array
bool all_whole(const AdapterParams &p, int size, int ysize) {
    auto whole = [](const void *q, long long values, int bytes) { return aligned16(q) && values * bytes % 16 == 0; };
    return whole(p.x, p.x_stride, size) && whole(p.a, p.Kd, size) && whole(p.b, p.rank, size) && whole(p.base, p.base_stride, ysize) &&
           whole(p.y, p.y_stride, ysize) && p.N * ysize % 16 == 0;
}

template <typename L, bool FEW, int NR>
void launch_rank(const AdapterParams &p, bool y_f32, hipStream_t st) {
    auto whole = [](const void *q, long long values, int size) { return aligned16(q) && values * size % 16 == 0; };
    const bool wx = whole(p.x, p.x_stride, L::SIZE) && whole(p.a, p.Kd, L::SIZE), wb = whole(p.b, p.rank, L::SIZE);
    const int ysize = y_f32 ? 4 : 2;
    const bool wy = whole(p.base, p.base_stride, ysize) && whole(p.y, p.y_stride, ysize) && p.N * ysize % 16 == 0;
    const dim3 grid(p.max_tiles, p.splits, p.chunks), over(p.max_tiles, (p.N + RANGE - 1) / RANGE, p.chunks), block(WAVES * 64);
    if (wx) hipLaunchKernelGGL((adapter_shrink_kernel<L, true, FEW, NR>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((adapter_shrink_kernel<L, false, FEW, NR>), grid, block, 0, st, p);
    const dim3 wide(expand_waves(NR) * 64);
    auto expand = [&](auto kernel) { hipLaunchKernelGGL(kernel, over, wide, 0, st, p); };
    if (y_f32) {
        if (wy) wb ? expand(adapter_expand_kernel<L, true, true, true, FEW, NR>) : expand(adapter_expand_kernel<L, false, true, true, FEW, NR>);
        else wb ? expand(adapter_expand_kernel<L, true, true, false, FEW, NR>) : expand(adapter_expand_kernel<L, false, true, false, FEW, NR>);
    } else {
        if (wy) wb ? expand(adapter_expand_kernel<L, true, false, true, FEW, NR>) : expand(adapter_expand_kernel<L, false, false, true, FEW, NR>);
        else wb ? expand(adapter_expand_kernel<L, true, false, false, FEW, NR>) : expand(adapter_expand_kernel<L, false, false, false, FEW, NR>);
    }
}

template <typename L, bool FEW>
void launch_typed(const AdapterParams &p, bool y_f32, hipStream_t st) {
    if (p.width <= 16) launch_rank<L, FEW, 1>(p, y_f32, st);
    else if (p.width <= 32) launch_rank<L, FEW, 2>(p, y_f32, st);
    else if (p.width <= 64) launch_rank<L, FEW, 4>(p, y_f32, st);
    else launch_rank<L, FEW, 8>(p, y_f32, st);
}

// One launch | two, us: one row 4096 -> 4096 of rank 16 7.5 | 8.2, 16 rows of 16 adapters 8.4 | 9.9, one row 2048 -> 1408 of rank 8
// 4.6 | 7.5; beyond the limits: one row 8192 -> 4096 (256 KB of A) 11.8 | 9.1, 8 rows 4096 -> 14336 (448 workgroups) 12.9 | 9.4.
bool one_launch(const AdapterParams &p, bool f32, bool y_f32) {
    return p.rows <= ONE_MOST && p.rank <= 16 && (long long)p.max_tiles * ((p.N + RANGE - 1) / RANGE) <= ONE_GRID && (long long)p.rank * p.Kd * (f32 ? 4 : 2) <= ONE_BYTES && all_whole(p, f32 ? 4 : 2, y_f32 ? 4 : 2);
}

}  // namespace

// The launches are sized for the adapters in the arrays, not for those that the rows turn out to use: what is not used is workgroups that
// find no tile, and from about 256 adapters on fewer parts of the reduction.  2048 -> 4096, rank 16, in arrays of 6 / 64 / 512 / 1024 adapters, us: 8192
// rows of 6 adapters 46 45 57 70, 1024 rows of one 19 20 32 29, 128 rows of 6 13 13 18 22; up to 64 rows the arrays do not matter (9).
void plan_adapters(AdapterParams &p, bool f32) {
    p.chunks = (p.rows + ADAPTER_CHUNK - 1) / ADAPTER_CHUNK;
    const int rows = p.rows < ADAPTER_CHUNK ? p.rows : ADAPTER_CHUNK, keys = p.n + 1;
    p.max_tiles = rows / ADAPTER_TILE + (keys < rows ? keys : rows);
    p.width = p.rank <= 16 ? 16 : p.rank <= 32 ? 32 : p.rank <= 64 ? 64 : 128;
    p.u_rows = p.chunks > 1 ? (long long)p.chunks * ADAPTER_CHUNK : p.rows;
    // parts of the reduction: a workgroup a unit, and a line for each of a part's waves
    p.tiles_about = p.rows / ADAPTER_TILE + (p.n < p.rows ? p.n : p.rows);
    const int want = p.tiles_about > 0 ? (WANTED + p.tiles_about - 1) / p.tiles_about : 1;
    p.max_splits = ((p.Kd * (f32 ? 4 : 2) + 127) / 128 + WAVES - 1) / WAVES;
    p.max_splits = p.max_splits < MAX_SPLITS ? p.max_splits : MAX_SPLITS;
    p.splits = want < p.max_splits ? want : p.max_splits;
}

// splits * u_rows <= (WANTED / tiles + 1) * u_rows with tiles >= rows / 64 and, from 1024 rows on, u_rows < 2 * rows: a workspace for
// the largest batch serves the smaller ones
size_t adapter_u_rows(const AdapterParams &p) {
    const size_t all = (size_t)p.max_splits * p.u_rows, some = (size_t)p.u_rows + 2 * WANTED * ADAPTER_TILE;
    return all < some ? all : some;
}

int launch_adapters(const AdapterParams &p, bool f32, bool y_f32, hipStream_t st) {
    if (p.rows <= ADAPTER_TILE) {
        AdapterParams few = p;                               // a tile is all rows of an adapter
        few.max_tiles = p.n + (p.in_place ? 0 : 1) < p.rows ? p.n + (p.in_place ? 0 : 1) : p.rows;
        if (one_launch(few, f32, y_f32)) {
            const dim3 grid(few.max_tiles, (p.N + RANGE - 1) / RANGE), block(ONE_WAVES * 64);
            auto one = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, few); };
            if (f32) y_f32 ? one(adapter_one_kernel<F32Line, true>) : one(adapter_one_kernel<F32Line, false>);
            else y_f32 ? one(adapter_one_kernel<Bf16Line, true>) : one(adapter_one_kernel<Bf16Line, false>);
            return launch_status(__func__);
        }
        if (f32) launch_typed<F32Line, true>(few, y_f32, st);
        else launch_typed<Bf16Line, true>(few, y_f32, st);
        return launch_status(__func__);
    }
    const int threads = p.rows >= ADAPTER_CHUNK ? ADAPTER_CHUNK : (p.rows + 63) / 64 * 64;
    hipLaunchKernelGGL(adapter_group_kernel, dim3(p.chunks), dim3(threads), 0, st, p);
    if (f32) launch_typed<F32Line, false>(p, y_f32, st);
    else launch_typed<Bf16Line, false>(p, y_f32, st);
    return launch_status(__func__);
}

}  // namespace bm
