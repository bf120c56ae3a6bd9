// Low-rank adapters of many requests beside a shared projection:
//   y[t] = base[t] + scale[a] * B[a] (A[a] x[t]),   a = the adapter of row t
//
// Three launches: rows are grouped by adapter (chunks of 1024 rows, each on its own), u = A x of a tile of up to 64 rows of one
// adapter (the reduction cut into parts over the chip), then B u is added to base on the way to y.  A and B are read once for
// each such tile, x once, base and y once.  u is held in fp32.
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
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(ADAPTER_CHUNK) adapter_group_kernel(AdapterParams p) {
    constexpr int WAVES = ADAPTER_CHUNK / 64;
    __shared__ uint16_t count[WAVES][BM_MAX_ADAPTERS + 8];
    __shared__ int rows_before[BM_MAX_ADAPTERS + 8];
    __shared__ int wave_rows[WAVES], wave_tiles[WAVES];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, waves = blockDim.x >> 6, chunk = blockIdx.x;
    const int row = chunk * ADAPTER_CHUNK + tid, keys = p.n + 1;
    for (int k = tid; k < waves * (BM_MAX_ADAPTERS + 8); k += blockDim.x) (&count[0][0])[k] = 0;
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
        const int start = before_rows + r - total, tile0 = before_tiles + t - tiles;
        if (k < keys) rows_before[k] = start;
        for (int i = 0; i < tiles; ++i)
            p.tiles[(size_t)chunk * p.max_tiles + tile0 + i] =
                AdapterTile{k, start + i * ADAPTER_TILE, min(ADAPTER_TILE, total - i * ADAPTER_TILE), 0};
        __syncthreads();
    }
    if (key >= 0) p.order[(size_t)chunk * ADAPTER_CHUNK + rows_before[key] + count[wave][key] + rank] = row;
    if (tid == 0) p.n_tiles[chunk] = tiles_so_far;
}

// ---------------------------------------------------------------------------
// u = A x of a tile: the four waves take every fourth line of the workgroup's part of the reduction, their sums are added as
// (w0 + w2) + (w1 + w3).  Matrix rows are A's, columns the tile's rows: a lane ends with four neighbouring values of u.
// TS: blocks of 16 rows; NR: blocks of 16 ranks.
// ---------------------------------------------------------------------------
constexpr int WAVES = 4;
constexpr int WANTED = 512, MAX_SPLITS = 16;      // workgroups of the launch, parts of the reduction at most

template <typename L, bool WHOLE, int TS, int NR>
__device__ __forceinline__ void shrink_tile(const AdapterParams &p, const AdapterTile &tile, int chunk, int split, f32x4 (*sums)[64]) {
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const int lines = (p.Kd + L::VALUES - 1) / L::VALUES;
    const int begin = (int)((long long)split * lines / p.splits), end = (int)((long long)(split + 1) * lines / p.splits);
    const int blocks = (rank_of(p, tile.adapter) + 15) >> 4;                  // of ranks that count
    const char *xr[TS], *ar[NR];
#pragma unroll
    for (int i = 0; i < TS; ++i) {
        const int row = p.order[(size_t)chunk * ADAPTER_CHUNK + tile.start + min(i * 16 + r16, tile.count - 1)];
        xr[i] = static_cast<const char *>(p.x) + (size_t)row * p.x_stride * L::SIZE;
    }
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
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                if (j >= blocks) break;
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
    float *u = p.u + (split * (size_t)p.u_rows + (size_t)chunk * ADAPTER_CHUNK) * p.width;
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        if (j >= blocks) break;
#pragma unroll
        for (int i = 0; i < TS; ++i) {
            const f32x4 sum = acc[j][i] + sums[(NR + j) * TS + i][lane];
            if (i * 16 + r16 < tile.count)
                *(BM_GLOBAL f32x4 *)(u + (size_t)(tile.start + i * 16 + r16) * p.width + j * 16 + kq * 4) = sum;
        }
    }
}

template <typename L, bool WHOLE, int NR>
__global__ void __launch_bounds__(WAVES * 64) adapter_shrink_kernel(AdapterParams p) {
    __shared__ f32x4 sums[2 * NR * (ADAPTER_TILE / 16)][64];
    const int chunk = blockIdx.z;
    if ((int)blockIdx.x >= ldg_i32(p.n_tiles + chunk)) return;
    const AdapterTile tile = p.tiles[(size_t)chunk * p.max_tiles + blockIdx.x];
    if (tile.adapter >= p.n) return;
    if (tile.count <= 16) shrink_tile<L, WHOLE, 1, NR>(p, tile, chunk, blockIdx.y, sums);
    else shrink_tile<L, WHOLE, ADAPTER_TILE / 16, NR>(p, tile, chunk, blockIdx.y, sums);
}

// ---------------------------------------------------------------------------
// y = base + scale * B u of a tile and a range of columns.  Matrix rows are B's, columns the tile's rows.  Four matrix blocks cover
// 64 columns, their rows dealt so that a lane ends with eight neighbouring columns in each half: block j, row 4 q + v is
// column (j / 2) * 32 + q * 8 + (j % 2) * 4 + v.
// bf16: u goes to the matrix unit as the sum of two bf16 values, each the rest of those before it rounded (16 bits of u), of three
// (all 24) where y is fp32, which would show the difference: 1.6e-6 of an fp32 y with two, rank 128.  Up to 16 ranks the
// first two lie in one instruction's 32.
// ---------------------------------------------------------------------------
constexpr int RANGE = 256;               // columns of a workgroup, 64 a wave

// The values of u in the form of the matrix operand: [part][k block][row block][lane] 16 bytes
template <typename L, bool YF32, int NR>
struct Expanded {
    static constexpr bool F32 = L::SIZE == 4;
    static constexpr int KB = F32 ? NR : (NR + 1) / 2;       // blocks of 16 (fp32) or 32 ranks
    static constexpr int PARTS = F32 ? 1 : NR == 1 ? (YF32 ? 2 : 1) : (YF32 ? 3 : 2);
    u32x4 v[PARTS][KB][ADAPTER_TILE / 16][64];
};

// The bf16 values of a pair, and what they leave of it (an infinity leaves nothing)
__device__ __forceinline__ uint32_t take_bf16(float &a, float &b) {
    const uint32_t v = pack_bf16x2(a, b);
    const float x = __builtin_bit_cast(float, v << 16), y = __builtin_bit_cast(float, v & 0xffff0000u);
    a = fabsf(x) < __builtin_inff() ? a - x : 0.0f;
    b = fabsf(y) < __builtin_inff() ? b - y : 0.0f;
    return v;
}

template <typename L, bool YF32, int NR>
__device__ __forceinline__ void stage_u(const AdapterParams &p, const AdapterTile &tile, int chunk, int rank, Expanded<L, YF32, NR> &out) {
    using X = Expanded<L, YF32, NR>;
    const size_t step = (size_t)p.u_rows * p.width;
    const int blocks = (tile.count + 15) >> 4;
    // a thread makes one lane's piece of a k block: 8 ranks in bf16, 4 in fp32
    for (int at = threadIdx.x; at < X::KB * blocks * 64; at += WAVES * 64) {
        const int lane = at & 63, i = (at >> 6) % blocks, kb = (at >> 6) / blocks;
        const int kq = lane >> 4, row = min(i * 16 + (lane & 15), tile.count - 1);
        const int r0 = X::F32 ? kb * 16 + kq * 4 : NR == 1 ? (kq & 1) * 8 : kb * 32 + kq * 8;
        const float *u = p.u + ((size_t)chunk * ADAPTER_CHUNK + tile.start + row) * p.width + r0;
        float v[8];
#pragma unroll
        for (int h = 0; h < (X::F32 ? 1 : 2); ++h) {
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            if (r0 + 4 * h < rank) {                         // (blocks of 16 ranks behind the last one are not written)
                sum = *(const BM_GLOBAL f32x4 *)(u + 4 * h);
                for (int s = 1; s < p.splits; ++s) sum += *(const BM_GLOBAL f32x4 *)(u + s * step + 4 * h);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) v[4 * h + c] = r0 + 4 * h + c < rank ? sum[c] : 0.0f;
        }
        if constexpr (X::F32) {
            out.v[0][kb][i][lane] = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
        } else {
            constexpr int VALUES = NR == 1 ? X::PARTS + 1 : X::PARTS;
            u32x4 part[VALUES];
#pragma unroll
            for (int j = 0; j < VALUES; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) part[j][c] = take_bf16(v[2 * c], v[2 * c + 1]);
            if constexpr (NR == 1) {                         // ranks 0 to 15 twice: the first part, then the second
                out.v[0][0][i][lane] = kq < 2 ? part[0] : part[1];
                if constexpr (YF32) out.v[1][0][i][lane] = kq < 2 ? part[2] : u32x4{0, 0, 0, 0};
            } else {
#pragma unroll
                for (int j = 0; j < X::PARTS; ++j) out.v[j][kb][i][lane] = part[j];
            }
        }
    }
}

// N values of a row of y from column n on, as fp32
template <bool YF32, bool WHOLE, int N>
__device__ __forceinline__ void load_row(const void *row, int n, int end, float (&v)[N]) {
    if constexpr (WHOLE) {
        if (n < end) {
            if constexpr (YF32) {
#pragma unroll
                for (int i = 0; i < N; i += 4) {
                    const f32x4 q = *(const BM_GLOBAL f32x4 *)(static_cast<const float *>(row) + (n + i < end ? n + i : n));
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[i + c] = q[c];
                }
            } else {
                const u32x4 q = ldg128(static_cast<const uint16_t *>(row) + n);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = bf16_to_f32((uint16_t)(q[i / 2] >> 16 * (i % 2)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
            if (n + i < end) v[i] = YF32 ? ldg_f32(static_cast<const float *>(row) + n + i)
                                         : bf16_to_f32(*(const BM_GLOBAL uint16_t *)(static_cast<const uint16_t *>(row) + n + i));
        }
    }
}

template <bool YF32, bool WHOLE, int N>
__device__ __forceinline__ void store_row(void *row, int n, int end, const float (&v)[N]) {
    if constexpr (WHOLE) {
        if constexpr (YF32) {
#pragma unroll
            for (int i = 0; i < N; i += 4)
                if (n + i < end) *(BM_GLOBAL f32x4 *)(static_cast<float *>(row) + n + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
        } else if (n < end) {
            u32x4 q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            stg128(static_cast<uint16_t *>(row) + n, q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (n + i < end) {
                if (YF32) *(BM_GLOBAL float *)(static_cast<float *>(row) + n + i) = v[i];
                else stg16(static_cast<uint16_t *>(row) + n + i, f32_to_bf16(v[i]));
            }
    }
}

template <typename L, bool WHOLE, bool YF32, bool YWHOLE, int NR>
__global__ void __launch_bounds__(WAVES * 64) adapter_expand_kernel(AdapterParams p) {
    using X = Expanded<L, YF32, NR>;
    __shared__ X s;
    const int chunk = blockIdx.z;
    if ((int)blockIdx.x >= ldg_i32(p.n_tiles + chunk)) return;
    const AdapterTile tile = p.tiles[(size_t)chunk * p.max_tiles + blockIdx.x];
    const int lane = lane_id(), wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const bool none = tile.adapter >= p.n;                   // rows without an adapter: base goes to y
    const int rank = none ? 0 : rank_of(p, tile.adapter);
    const float scale = none || p.scale == nullptr ? 1.0f : ldg_f32(p.scale + tile.adapter);
    const int n0 = blockIdx.y * RANGE + wave * 64, blocks = (tile.count + 15) >> 4;
    const int ysize = YF32 ? 4 : 2;
    if (rank > 0) stage_u<L, YF32, NR>(p, tile, chunk, rank, s);
    u32x4 bv[X::KB][4];
    if (rank > 0 && n0 < p.N) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = n0 + (j / 2) * 32 + (r16 >> 2) * 8 + (j % 2) * 4 + (r16 & 3);
            const char *row = static_cast<const char *>(p.b) + ((size_t)tile.adapter * p.N + min(col, p.N - 1)) * p.rank * L::SIZE;
#pragma unroll
            for (int kb = 0; kb < X::KB; ++kb) {
                const int r0 = X::F32 ? kb * 16 + kq * 4 : NR == 1 ? (kq & 1) * 8 : kb * 32 + kq * 8;
                bv[kb][j] = piece<L, WHOLE>(row, r0, rank, p.rank);
            }
        }
    }
    __syncthreads();
    if (n0 >= p.N) return;
    for (int i = 0; i < blocks; ++i) {
        const bool live = i * 16 + r16 < tile.count;
        const int row = p.order[(size_t)chunk * ADAPTER_CHUNK + tile.start + min(i * 16 + r16, tile.count - 1)];
        const char *from = static_cast<const char *>(p.base) + (size_t)row * p.base_stride * ysize;
        float v[2][8];
#pragma unroll
        for (int h = 0; h < 2; ++h) load_row<YF32, YWHOLE>(from, n0 + h * 32 + kq * 8, p.N, v[h]);
        if (rank > 0) {
            f32x4 acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kb = 0; kb < X::KB; ++kb)
#pragma unroll
                for (int part = 0; part < X::PARTS; ++part) {
                    const u32x4 uv = s.v[part][kb][i][lane];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = L::mac(bv[kb][j], uv, acc[j]);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 8; ++c) v[h][c] = fmaf(scale, acc[2 * h + c / 4][c % 4], v[h][c]);
        }
        char *to = static_cast<char *>(p.y) + (size_t)row * p.y_stride * ysize;
        if (live)
#pragma unroll
            for (int h = 0; h < 2; ++h) store_row<YF32, YWHOLE>(to, n0 + h * 32 + kq * 8, p.N, v[h]);
    }
}

template <typename L, bool WHOLE, bool YF32, bool YWHOLE, int NR>
void launch_expand(const AdapterParams &p, hipStream_t st) {
    hipLaunchKernelGGL((adapter_expand_kernel<L, WHOLE, YF32, YWHOLE, NR>), dim3(p.max_tiles, (p.N + RANGE - 1) / RANGE, p.chunks), dim3(WAVES * 64), 0, st, p);
}

template <typename L, int NR>
void launch_rank(const AdapterParams &p, bool y_f32, hipStream_t st) {
    auto whole = [](const void *q, long long values, int size) { return aligned16(q) && values * size % 16 == 0; };
    const bool wx = whole(p.x, p.x_stride, L::SIZE) && whole(p.a, p.Kd, L::SIZE), wb = whole(p.b, p.rank, L::SIZE);
    const int ysize = y_f32 ? 4 : 2;
    const bool wy = whole(p.base, p.base_stride, ysize) && whole(p.y, p.y_stride, ysize) && p.N * ysize % 16 == 0;
    const dim3 grid(p.max_tiles, p.splits, p.chunks), block(WAVES * 64);
    if (wx) hipLaunchKernelGGL((adapter_shrink_kernel<L, true, NR>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((adapter_shrink_kernel<L, false, NR>), grid, block, 0, st, p);
    if (y_f32) {
        if (wy) wb ? launch_expand<L, true, true, true, NR>(p, st) : launch_expand<L, false, true, true, NR>(p, st);
        else wb ? launch_expand<L, true, true, false, NR>(p, st) : launch_expand<L, false, true, false, NR>(p, st);
    } else {
        if (wy) wb ? launch_expand<L, true, false, true, NR>(p, st) : launch_expand<L, false, false, true, NR>(p, st);
        else wb ? launch_expand<L, true, false, false, NR>(p, st) : launch_expand<L, false, false, false, NR>(p, st);
    }
}

template <typename L>
void launch_typed(const AdapterParams &p, bool y_f32, hipStream_t st) {
    if (p.width <= 16) launch_rank<L, 1>(p, y_f32, st);
    else if (p.width <= 32) launch_rank<L, 2>(p, y_f32, st);
    else if (p.width <= 64) launch_rank<L, 4>(p, y_f32, st);
    else launch_rank<L, 8>(p, y_f32, st);
}

}  // namespace

void plan_adapters(AdapterParams &p, bool f32) {
    p.chunks = (p.rows + ADAPTER_CHUNK - 1) / ADAPTER_CHUNK;
    const int rows = p.rows < ADAPTER_CHUNK ? p.rows : ADAPTER_CHUNK, keys = p.n + 1;
    p.max_tiles = rows / ADAPTER_TILE + (keys < rows ? keys : rows);
    p.width = p.rank <= 16 ? 16 : p.rank <= 32 ? 32 : p.rank <= 64 ? 64 : 128;
    p.u_rows = p.chunks > 1 ? (long long)p.chunks * ADAPTER_CHUNK : p.rows;
    // parts of the reduction: two workgroups a unit, and a line for each of a part's waves
    const long long tiles = (long long)p.rows / ADAPTER_TILE + (p.n < p.rows ? p.n : p.rows);
    const long long want = tiles > 0 ? (WANTED + tiles - 1) / tiles : 1;
    p.max_splits = ((p.Kd * (f32 ? 4 : 2) + 127) / 128 + WAVES - 1) / WAVES;
    p.max_splits = p.max_splits < MAX_SPLITS ? p.max_splits : MAX_SPLITS;
    p.splits = (int)(want < p.max_splits ? want : p.max_splits);
}

// splits * u_rows <= (WANTED / tiles + 1) * u_rows with tiles >= rows / 64 and, from 1024 rows on, u_rows < 2 * rows: a workspace for
// the largest batch serves the smaller ones
size_t adapter_u_rows(const AdapterParams &p) {
    const size_t all = (size_t)p.max_splits * p.u_rows, some = (size_t)p.u_rows + 2 * WANTED * ADAPTER_TILE;
    return all < some ? all : some;
}

int launch_adapters(const AdapterParams &p, bool f32, bool y_f32, hipStream_t st) {
    const int threads = p.rows >= ADAPTER_CHUNK ? ADAPTER_CHUNK : (p.rows + 63) / 64 * 64;
    hipLaunchKernelGGL(adapter_group_kernel, dim3(p.chunks), dim3(threads), 0, st, p);
    if (f32) launch_typed<F32Line>(p, y_f32, st);
    else launch_typed<Bf16Line>(p, y_f32, st);
    return launch_status(__func__);
}

}  // namespace bm
