// Block tables and slot maps from the lengths (rheo_cache_plan).
#include "cache_state.h"

namespace rheo {

namespace {

constexpr int NTP = 256;

struct Demand {
    int need, take, give;          // pages in all, to pop, to push
    bool fits;                     // valid, and its row of the table holds them
    bool valid;
};

__device__ __forceinline__ Demand demand_of(const CacheDev& c, const PlanArgs& a, int len, int count,
                                            int held) {
    Demand d;
    d.valid = len >= 0 && count >= 0 && count <= a.n && held >= 0 && held <= c.width;
    const int64_t need = ((int64_t)len + count + (1 << c.page_shift) - 1) >> c.page_shift;
    d.fits = d.valid && need <= c.width;
    d.need = d.fits ? (int)need : 0;
    d.take = d.fits ? max(d.need - held, 0) : 0;
    d.give = d.fits ? max(held - d.need, 0) : 0;
    return d;
}

__device__ __forceinline__ int clamp31(int64_t v) {
    return (int)(v < 0x7FFFFFFF ? v : 0x7FFFFFFF);
}
// Lacked pages may add up to 2^42, of which only sums below the pool's 2^31 are told
// apart: all others are more than there is.
__device__ __forceinline__ uint32_t clamp32(int64_t v) {
    return (uint32_t)(v < 0xFFFFFFFFll ? v : 0xFFFFFFFFll);
}
// A sequence's need (at most 2^30 pages) and whether it lacks some; kMisfit: out of range
// or too many.
constexpr uint32_t kMisfit = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t pack_need(const Demand& d) {
    return d.fits ? (uint32_t)d.need << 1 | (d.take > 0 ? 1u : 0u) : kMisfit;
}

}  // namespace

// Sums of the pages lacked and returned by all sequences before each, which
// every block takes over the whole batch for itself (three numbers a sequence,
// from the L2 after the first block), so that one launch does it all: no block
// waits for another.  A popped page that another sequence returns in this
// call is read from that sequence's row of the table, which nobody writes
// there.  What the sums are taken from (held, free_count) is written by
// the last block to finish, when all have read it.
//
// Latency is all there is (1 MB at 1024 sequences of 81 rows): the sums are one
// round of loads and one exchange, and a block's rows are worked on all at once: 18 us
// there (10 without rows), 4 us for one sequence.
__global__ __launch_bounds__(NTP) void k_cache_plan(CacheDev c, PlanArgs a) {
    // [B + 1] pages lacked by all before, [B + 1] returned; [B] pages needed (pack_need)
    extern __shared__ int s_sum[];
    __shared__ int64_t s_wave[2][NTP / 64];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = c.B;
    uint32_t* const s_take = (uint32_t*)s_sum;
    int* const s_give = s_sum + B + 1;
    uint32_t* const s_need = (uint32_t*)s_give + B + 1;
    // consecutive sequences a thread, then the threads' sums
    const int per = (B + NTP - 1) / NTP, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    const int have0 = *a.free_count;
    int64_t take = 0, give = 0;
    bool bad = false;
    for (int b = b0; b < b1; b += 4) {
        int len[4], count[4], held[4];       // (the last sequence's again past the end)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = min(b + k, b1 - 1);
            len[k] = a.lens[i];
            count[k] = a.count ? a.count[i] : a.n;
            held[k] = a.held[i];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (b + k >= b1) break;
            const Demand d = demand_of(c, a, len[k], count[k], held[k]);
            s_take[b + k] = clamp32(take);   // (relative to the thread's first)
            s_give[b + k] = clamp31(give);
            s_need[b + k] = pack_need(d);
            take += d.take;
            give += d.give;
            bad |= !d.valid;
        }
    }
    int64_t ti = take, gi = give;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t t = __shfl_up(ti, o), g = __shfl_up(gi, o);
        if (lane >= o) { ti += t; gi += g; }
    }
    if (lane == 63) { s_wave[0][wave] = ti; s_wave[1][wave] = gi; }
    __syncthreads();
    int64_t tb = ti - take, gb = gi - give, takes = 0, gives = 0;
    for (int w = 0; w < NTP / 64; ++w) {
        if (w < wave) { tb += s_wave[0][w]; gb += s_wave[1][w]; }
        takes += s_wave[0][w];
        gives += s_wave[1][w];
    }
    for (int b = b0; b < b1; ++b) {
        s_take[b] = clamp32(tb + s_take[b]);
        s_give[b] = clamp31(gb + s_give[b]);
    }
    if (tid == 0) {
        s_take[B] = clamp32(takes);
        s_give[B] = clamp31(gives);
    }
    const int have = min(max(have0, 0), c.pages);
    bad |= have != have0 || have + gives > c.pages;
    const int64_t room = have + gives;
    __syncthreads();
    if (blockIdx.x == 0 && bad) atomicOr(c.err, CE_PLAN);
    auto fits = [&](int b) { return s_need[b] != kMisfit; };
    auto lacks = [&](int b) { return fits(b) && (s_need[b] & 1u); };
    auto need_of = [&](int b) { return fits(b) ? (int)(s_need[b] >> 1) : 0; };
    auto served = [&](int b) {
        return fits(b) && (!lacks(b) || (int64_t)s_take[b + 1] <= room);
    };
    // of a served sequence
    auto took_of = [&](int b) { return (int)(s_take[b + 1] - s_take[b]); };

    // page number v of the stack after the pushes
    auto stack_page = [&](int64_t v) -> int {
        int page;
        if (v < have) {
            page = a.free_list[v];
        } else {
            // the (room - 1 - v)-th returned page: the last sequence that fewer are
            // returned before (those that return none share their sum with the next)
            const int r = clamp31(room - 1 - v);
            int lo = 0, hi = B - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_give[mid] <= r) lo = mid; else hi = mid - 1;
            }
            // (held out of range as a whole: sums that the index does not follow)
            const int64_t at = (int64_t)need_of(lo) + r - s_give[lo];
            page = a.table[(int64_t)lo * c.width + (at < 0 ? 0 : at < c.width ? at : c.width - 1)];
        }
        if ((unsigned)page >= (unsigned)c.pages) {
            atomicOr(c.err, CE_PLAN);
            page = 0;
        }
        return page;
    };

    // the block's sequences: blockIdx.x and every gridDim.x-th after it, their new
    // pages (16 threads each) and their rows all at once
    const int mine = (B - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
    for (int k = tid / 16; k < mine; k += NTP / 16) {
        const int b = blockIdx.x + k * gridDim.x;
        if (!served(b) || !lacks(b)) continue;
        const int took = took_of(b), held = need_of(b) - took;
        for (int p = tid % 16; p < took; p += 16)
            a.table[(int64_t)b * c.width + held + p] = stack_page(room - 1 - s_take[b] - p);
    }
    const int rows = mine * a.n;               // (at most 2^30)
    for (int f = tid; f < rows; f += NTP) {
        const int k = f / a.n, i = f - k * a.n;
        const int b = blockIdx.x + k * gridDim.x;
        const int64_t at = (int64_t)b * a.n + i;
        const int len = a.lens[b], count = a.count ? a.count[b] : a.n;
        const int depth = a.depth ? a.depth[at] : i;
        int64_t slot = -1;
        int pos = -1;
        if (served(b) && i < count) {
            const int held = need_of(b) - took_of(b);                    // (or more)
            const int e = len + i, p = e >> c.page_shift;
            const int page = p < held ? a.table[(int64_t)b * c.width + p]
                                      : stack_page(room - 1 - s_take[b] - (p - held));
            if ((unsigned)page >= (unsigned)c.pages) {
                atomicOr(c.err, CE_PAGE);
            } else {
                slot = ((int64_t)page << c.page_shift) + (e & ((1 << c.page_shift) - 1));
                pos = len + depth;
            }
        }
        a.slots[at] = slot;
        a.positions[at] = pos;
    }
    for (int k = tid; k < mine; k += NTP) {
        const int b = blockIdx.x + k * gridDim.x;
        a.status[b] = served(b) ? 0 : fits(b) ? 1 : 2;
    }

    // every read of this block is done (no data passes to the last block, so the
    // count needs no fence)
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0)
            s_last = __hip_atomic_fetch_add(c.ticket + B, 1u, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
        __syncthreads();
        if (!s_last) return;
        if (tid == 0) c.ticket[B] = 0;
    }
    // pages popped: up to the last sequence that got any
    int used = 0;
    for (int b = b0; b < b1; ++b) {
        if (!served(b)) continue;
        if (lacks(b)) used = (int)s_take[b + 1];
        a.held[b] = need_of(b);
    }
    for (int o = 32; o; o >>= 1) used = max(used, __shfl_xor(used, o));
    if (lane == 0) s_wave[0][wave] = used;
    __syncthreads();
    for (int w = 0; w < NTP / 64; ++w) used = max(used, (int)s_wave[0][w]);
    const int64_t left = room - used;
    // returned pages that were not popped again: only if fewer are left than
    // pushed, so that no block of this launch read the places written here
    for (int64_t v = have + tid; v < left && v < c.pages; v += NTP) a.free_list[v] = stack_page(v);
    if (tid == 0) *a.free_count = (int)min(left, (int64_t)c.pages);
}

hipError_t launch_cache_plan(const CacheDev& c, const PlanArgs& a, hipStream_t s) {
    const int blocks = c.B < 256 ? c.B : 256;
    k_cache_plan<<<blocks, NTP, sizeof(int) * (3 * (size_t)c.B + 2), s>>>(c, a);
    return hipGetLastError();
}

}  // namespace rheo
