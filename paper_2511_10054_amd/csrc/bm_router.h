// Routing by scores, a balance bias and groups of experts: parameters and launchers (bm_router.hip).
#pragma once
#include "bm_kernels.h"

namespace bm {

constexpr int MAX_ROUTER_D = 1 << 20;
constexpr int MAX_ROUTER_GROUPS = 64;    // a lane of a wave for each

struct RouterParams {
    const void *x;                // [T][d]
    const void *w;                // [E][d]
    const float *bias;            // [E], added to the logits, or null
    const float *balance;         // [E], added to the scores for the choice alone, or null
    float *logits;                // [parts][T][E] scratch, without the bias
    int T, d, E, K;
    int n_groups, keep_groups, group_top;
    int per_group, lanes_per_group;      // set by the launch
    bool sigmoid, renorm;
    float scale;
    int32_t *ids;                 // [T][K]
    float *weights;               // [T][K]
};

size_t router_scratch_bytes(int T, int E);
int launch_route_scored(const RouterParams &p, bool f32, hipStream_t st);

}  // namespace bm
