// Low-rank adapters of many requests beside a shared projection: parameters and launchers (bm_adapters.hip).
#pragma once
#include "bm_kernels.h"

namespace bm {

constexpr int ADAPTER_CHUNK = 1024;      // rows that are grouped by adapter together
constexpr int MAX_ADAPTER_ROWS = 1 << 24, MAX_ADAPTER_WIDTH = 1 << 20;
constexpr int ADAPTER_TILE = 64;         // rows of one adapter that a workgroup takes

struct AdapterTile {
    int adapter;                  // n: rows without one
    int start, count;             // places in the chunk's order
    int unused;
};

struct AdapterParams {
    const void *x;                // [rows][Kd], x_stride values apart
    const int32_t *adapter;       // [rows]
    const void *a, *b;            // [n][rank][Kd], [n][N][rank]
    const int32_t *ranks;         // [n], or null: rank
    const float *scale;           // [n], or null: 1
    const void *base;             // [rows][N], base_stride values apart
    void *y;                      // [rows][N], y_stride values apart
    long long x_stride, base_stride, y_stride;
    int rows, Kd, N, n, rank;
    bool in_place;                // base is y: rows without an adapter stay as they are
    int chunks, max_tiles;        // chunks of rows, tiles of a chunk at most
    int tiles_about;              // of all chunks
    int max_splits;               // whatever the number of rows
    int splits;                   // parts of the reduction over Kd, added in order
    int width;                    // of a row of u: rank rounded up to 16, 32, 64 or 128
    int32_t *order;               // [chunks][ADAPTER_CHUNK] row at each place
    AdapterTile *tiles;           // [chunks][max_tiles], of no rows behind the last
    float *u;                     // [splits][u_rows][width]: a chunk's rows in its order, from row chunk * ADAPTER_CHUNK on
    long long u_rows;
};

// The launch for these sizes (rows, Kd, N, n and rank are set): chunks, max_tiles, tiles_about, splits, width and u_rows
void plan_adapters(AdapterParams &p, bool f32);
size_t adapter_u_rows(const AdapterParams &p);   // room for splits * u_rows, no less for more rows
int launch_adapters(const AdapterParams &p, bool f32, bool y_f32, hipStream_t st);

}  // namespace bm
