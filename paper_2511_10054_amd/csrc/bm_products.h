// Grouped products of 8-bit rows with 8-bit matrices: parameters and launchers (bm_products.hip).
#pragma once
#include "bm_quantize.h"

namespace bm {

constexpr int MAX_PRODUCT_KD = 32768;    // the scales of a weight block's row of blocks lie in LDS

struct ProductParams {
    const uint8_t *a;             // [a_rows][Kd] e4m3
    const float *a_scale;         // [a_rows][kb], kb = ceil(Kd / 128)
    const int32_t *row_map;       // output row -> row_map[row] / map_div, its row of a; null: itself
    int map_div;
    int a_rows;
    const uint8_t *b0, *b1, *sb0, *sb1;          // [E][N][Kd]; b1: the second matrix (up) or null; s..: groups from E on
    const float *bs0, *bs1, *sbs0, *sbs1;        // [E][ceil(N / 128)][kb]
    const int32_t *offsets;       // [n_groups + 1], or null: one group of all rows
    int E, n_groups;
    int rows;                     // bound of the offsets
    int N, Kd;
    void *c;                      // product: [rows][N] bf16 or fp32; swiglu: [rows][N] e4m3
    float *c_scale;               // swiglu: [rows][ceil(N / 128)]
    int c_f32;
};

bool product_grid_ok(long long rows, int N, int n_groups);    // the launch's grid stays within its limits

int launch_product(const ProductParams &p, hipStream_t st);   // c = a b0^T
int launch_swiglu(const ProductParams &p, hipStream_t st);    // c = e4m3(silu(a b0^T) * (a b1^T)) with scales

}  // namespace bm
