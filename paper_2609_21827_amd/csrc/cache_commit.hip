// The accepted path of a verified tree and its cache entries (rheo_cache_commit).
#include "cache_state.h"

namespace rheo {

namespace {

constexpr int NTC = 256;
constexpr int kDepthMax = 15;                // accepted tokens of a step (rheo_create's limit)

}  // namespace

// Every block of a sequence walks the accepted path for itself (one search among
// the sequence's nodes a level), then moves its share of the layers' entries.
//
// Entry j of the path moves from len + path_j down to len + j.  path_j >= j
// and both rise with j (parents precede their children in pruned order), so
// the place j is read by no later entry: a thread that moves one 16-byte
// column of all entries, in rising j, never reads what it has written, and
// columns are independent.  Bytes moved are all there is; entries in their
// place already are left alone.  128 sequences, 32 layers, 4 entries on average
// (137 MB): 26 us, 5.2 TB/s; one sequence 4.5 us, the walk's latency.
__global__ __launch_bounds__(NTC) void k_cache_commit(CacheDev c, CommitArgs a, int split) {
    __shared__ int64_t s_src[kDepthMax + 1], s_dst[kDepthMax + 1];
    __shared__ int s_path[kDepthMax + 1];
    __shared__ int s_moves, s_len;
    const int b = blockIdx.x / split, part = blockIdx.x - b * split;
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) {
        const int len = a.lens[b], took = a.status && a.status[b] ? -1 : a.accept_len[b];
        const int32_t* parent = a.parent + (int64_t)b * a.n;
        const int32_t* token = a.token + (int64_t)b * a.n;
        int bad = 0;
        const int64_t room = (int64_t)c.width << c.page_shift;
        if (took > a.depth || took >= a.n) bad = CE_PATH;
        if (took >= 0 && (len < 0 || (int64_t)len + 1 + took > room)) bad |= CE_TABLE;
        bool good = took >= 0 && !bad;
        int node = 0;
        if (lane == 0) s_path[0] = 0;
        // the first 128 nodes in registers: a level is then no memory's latency
        int par[2], tok[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = min(64 * k + lane, a.n - 1);
            par[k] = 64 * k + lane < a.n ? parent[i] : -2;
            tok[k] = token[i];
        }
        if (good) {
            const int want_lane = lane < took ? a.accepted[(int64_t)b * a.depth + lane] : -1;
            for (int j = 0; j < took && good; ++j) {
                const int want = __shfl(want_lane, j);
                int found = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint64_t m = __ballot(par[k] == node && tok[k] == want &&
                                                64 * k + lane > node);
                    if (m && !found) found = 64 * k + __builtin_ctzll(m);
                }
                // (children come behind their parents; only those count, in whatever
                // tree, so that the path rises as the moves need it)
                for (int i0 = max(node + 1, 128); i0 < a.n && !found; i0 += 64) {
                    const int i = i0 + lane;
                    const bool hit = i < a.n && parent[i] == node && token[i] == want;
                    const uint64_t m = __ballot(hit);
                    if (m) found = i0 + __builtin_ctzll(m);
                }
                if (!found) {
                    bad |= CE_PATH;
                    good = false;
                } else {
                    node = found;
                    if (lane == 0) s_path[j + 1] = node;
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
        // the slots of each entry that moves, packed together in rising order
        bool moves = false;
        int64_t src = 0, dst = 0;
        if (good && lane >= 1 && lane <= took) {
            const int p = *(volatile int*)&s_path[lane];
            if ((int64_t)len + p >= room) {
                bad |= CE_TABLE;
            } else if (p != lane) {
                const int32_t* row = a.table + (int64_t)b * c.width;
                const int es = len + p, ed = len + lane;
                const int ps = row[es >> c.page_shift], pd = row[ed >> c.page_shift];
                const int in = (1 << c.page_shift) - 1;
                if ((unsigned)ps >= (unsigned)c.pages || (unsigned)pd >= (unsigned)c.pages) {
                    bad |= CE_PAGE;
                } else {
                    const int64_t bytes = (int64_t)c.K * c.D * 2;
                    src = ps * c.page_stride * 2 + (es & in) * bytes;
                    dst = pd * c.page_stride * 2 + (ed & in) * bytes;
                    moves = true;
                }
            }
        }
        bad |= (__any(bad & CE_PAGE) ? CE_PAGE : 0) | (__any(bad & CE_TABLE) ? CE_TABLE : 0);
        const uint64_t all = bad ? 0 : __ballot(moves);
        if (moves && !bad) {
            const int at = __builtin_popcountll(all & ((1ull << lane) - 1));
            s_src[at] = src;
            s_dst[at] = dst;
        }
        good = took >= 0 && !bad;
        if (lane == 0) {
            s_moves = __builtin_popcountll(all);
            s_len = good ? len + 1 + took : len;
            if (bad && part == 0) atomicOr(c.err, bad);
        }
        if (part == 0 && lane <= a.depth)
            a.path[(int64_t)b * (a.depth + 1) + lane] =
                good && lane <= took ? *(volatile int*)&s_path[lane] : -1;
    }
    __syncthreads();
    const int moves = s_moves;
    if (moves) {
        const int vecs = c.K * c.D / 8, total = c.layers * 2 * vecs;
        for (int f = part * NTC + tid; f < total; f += split * NTC) {
            const int layer = f / (2 * vecs), g = f - layer * 2 * vecs;
            char* base = (g < vecs ? a.k_cache : a.v_cache) + layer * c.layer_stride * 2 +
                         (int64_t)(g < vecs ? g : g - vecs) * 16;
            // four loads at a time (`moves` is the block's)
            for (int j0 = 0; j0 < moves; j0 += 4) {
                const int n = moves - j0;
                uint4 x0 = *(const uint4*)(base + s_src[j0]), x1 = x0, x2 = x0, x3 = x0;
                if (n > 1) x1 = *(const uint4*)(base + s_src[j0 + 1]);
                if (n > 2) x2 = *(const uint4*)(base + s_src[j0 + 2]);
                if (n > 3) x3 = *(const uint4*)(base + s_src[j0 + 3]);
                *(uint4*)(base + s_dst[j0]) = x0;
                if (n > 1) *(uint4*)(base + s_dst[j0 + 1]) = x1;
                if (n > 2) *(uint4*)(base + s_dst[j0 + 2]) = x2;
                if (n > 3) *(uint4*)(base + s_dst[j0 + 3]) = x3;
            }
        }
    }
    // new_lens may be lens itself: the sequence's last block writes it, when all
    // have read theirs.  (No data passes between the blocks, so the count needs no
    // fence; one, which writes the L2 back, took 100 us at 2048 blocks.)
    __syncthreads();
    if (tid == 0) {
        if (split == 1 || __hip_atomic_fetch_add(c.ticket + b, 1u, __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)split - 1) {
            if (split > 1) c.ticket[b] = 0;
            a.new_lens[b] = s_len;
        }
    }
}

hipError_t launch_cache_commit(const CacheDev& c, const CommitArgs& a, hipStream_t s) {
    const int total = c.layers * 2 * (c.K * c.D / 8);
    // one column a thread while that makes at most 2048 blocks in all
    int split = (total + NTC - 1) / NTC;
    if ((int64_t)split * c.B > 2048) split = 2048 / c.B;
    if (split < 1) split = 1;
    k_cache_commit<<<c.B * split, NTC, 0, s>>>(c, a, split);
    return hipGetLastError();
}

}  // namespace rheo
