// The accepted path of a verified tree, found by one wave.
#pragma once

#include "cache_state.h"

namespace rheo {

constexpr int kDepthMax = 15;                // accepted tokens of a step (rheo_create's limit)

// The nodes of the root and the `took` accepted tokens go to s_path; the error bit of a
// token that is no child of the node before it, or 0.  One search among the sequence's
// nodes a level.
__device__ __forceinline__ int walk_path(int lane, int n, const int32_t* parent, const int32_t* token,
                                         const int32_t* accepted, int took, int* s_path) {
    int node = 0;
    if (lane == 0) s_path[0] = 0;
    // the first 128 nodes in registers: a level is then no memory's latency
    int par[2], tok[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = min(64 * k + lane, n - 1);
        par[k] = 64 * k + lane < n ? parent[i] : -2;
        tok[k] = token[i];
    }
    const int want_lane = lane < took ? accepted[lane] : -1;
    for (int j = 0; j < took; ++j) {
        const int want = __shfl(want_lane, j);
        int found = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint64_t m = __ballot(par[k] == node && tok[k] == want && 64 * k + lane > node);
            if (m && !found) found = 64 * k + __builtin_ctzll(m);
        }
        // (children come behind their parents; only those count, in whatever
        // tree, so that the path rises as the moves need it)
        for (int i0 = max(node + 1, 128); i0 < n && !found; i0 += 64) {
            const int i = i0 + lane;
            const bool hit = i < n && parent[i] == node && token[i] == want;
            const uint64_t m = __ballot(hit);
            if (m) found = i0 + __builtin_ctzll(m);
        }
        if (!found) return CE_PATH;
        node = found;
        if (lane == 0) s_path[j + 1] = node;
    }
    return 0;
}

}  // namespace rheo
