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

__device__ __forceinline__ Demand demand_of(const CacheDev& c, const PlanArgs& a, int b) {
    const int len = a.lens[b], held = a.held[b];
    const int count = a.count ? a.count[b] : a.n;
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

}  // namespace

// Sums of the pages lacked and returned by all sequences before each, which
// every block takes over the whole batch for itself (three numbers a sequence,
// from the L2 after the first block), so that one launch does it all: no block
// waits for another.  A popped page that another sequence returns in this
// call is read from that sequence's row of the table, which nobody writes
// there.  What the sums are taken from (held, free_count) is written by
// the last block to finish, when all have read it.
__global__ __launch_bounds__(NTP) void k_cache_plan(CacheDev c, PlanArgs a) {
    extern __shared__ int s_sum[];           // [B] pages lacked before, [B] returned before
    __shared__ int64_t s_wave[2][NTP / 64];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int* s_take = s_sum;
    int* s_give = s_sum + c.B;
    // consecutive sequences a thread, then the threads' sums
    const int per = (c.B + NTP - 1) / NTP, b0 = min(tid * per, c.B), b1 = min(b0 + per, c.B);
    int64_t take = 0, give = 0;
    bool bad = false;
    for (int b = b0; b < b1; ++b) {
        const Demand d = demand_of(c, a, b);
        s_take[b] = clamp31(take);           // (relative to the thread's first)
        s_give[b] = clamp31(give);
        take += d.take;
        give += d.give;
        bad |= !d.valid;
    }
    int64_t ti = take, gi = give;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t t = __shfl_up(ti, o), g = __shfl_up(gi, o);
        if (lane >= o) { ti += t; gi += g; }
    }
    if (lane == 63) { s_wave[0][wave] = ti; s_wave[1][wave] = gi; }
    __syncthreads();
    int64_t tb = ti - take, gb = gi - give, gives = 0;
    for (int w = 0; w < NTP / 64; ++w) {
        if (w < wave) { tb += s_wave[0][w]; gb += s_wave[1][w]; }
        gives += s_wave[1][w];
    }
    for (int b = b0; b < b1; ++b) {
        s_take[b] = clamp31(tb + s_take[b]);
        s_give[b] = clamp31(gb + s_give[b]);
    }
    const int have0 = *a.free_count;
    const int have = min(max(have0, 0), c.pages);
    bad |= have != have0 || have + gives > c.pages;
    const int64_t room = have + gives;
    __syncthreads();
    if (blockIdx.x == 0 && bad) atomicOr(c.err, CE_PLAN);

    // page number v of the stack after the pushes
    auto stack_page = [&](int64_t v) -> int {
        int page;
        if (v < have) {
            page = a.free_list[v];
        } else {
            // the (room - 1 - v)-th returned page: the sequence it is of, then its place
            const int r = (int)(room - 1 - v);
            int lo = 0, hi = c.B - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (s_give[mid] <= r) lo = mid; else hi = mid - 1;
            }
            // (sequences that return nothing share their sum with the next)
            const Demand d = demand_of(c, a, lo);
            page = a.table[(int64_t)lo * c.width + min(d.need + r - s_give[lo], c.width - 1)];
        }
        if ((unsigned)page >= (unsigned)c.pages) {
            atomicOr(c.err, CE_PLAN);
            page = 0;
        }
        return page;
    };

    for (int b = blockIdx.x; b < c.B; b += gridDim.x) {
        const Demand d = demand_of(c, a, b);
        const int held = a.held[b], before = s_take[b];
        const bool served = d.fits && (d.take == 0 || (int64_t)before + d.take <= room);
        int32_t* row = a.table + (int64_t)b * c.width;
        const int64_t top = room - 1 - before + held;    // (place p's page: stack_page(top - p))
        if (served && d.take)
            for (int p = held + tid; p < d.need; p += NTP) row[p] = stack_page(top - p);
        const int len = a.lens[b];
        const int count = !served ? 0 : a.count ? a.count[b] : a.n;
        for (int i = tid; i < a.n; i += NTP) {
            int64_t slot = -1;
            int pos = -1;
            if (i < count) {
                const int e = len + i, p = e >> c.page_shift;
                int page = p < held ? row[p] : stack_page(top - p);
                if ((unsigned)page >= (unsigned)c.pages) {
                    atomicOr(c.err, CE_PAGE);
                } else {
                    slot = ((int64_t)page << c.page_shift) + (e & ((1 << c.page_shift) - 1));
                    pos = len + (a.depth ? a.depth[(int64_t)b * a.n + i] : i);
                }
            }
            a.slots[(int64_t)b * a.n + i] = slot;
            a.positions[(int64_t)b * a.n + i] = pos;
        }
        if (tid == 0) a.status[b] = served ? 0 : d.fits ? 1 : 2;
    }

    // every read of this block is done
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0) {
            __threadfence();
            s_last = atomicAdd(c.ticket + c.B, 1u) == gridDim.x - 1;
        }
        __syncthreads();
        if (!s_last) return;
        if (tid == 0) c.ticket[c.B] = 0;
    }
    int64_t used = 0;
    for (int b = b0; b < b1; ++b) {
        const Demand d = demand_of(c, a, b);
        if (d.fits && d.take && (int64_t)s_take[b] + d.take <= room) used += d.take;
    }
    for (int o = 32; o; o >>= 1) used += __shfl_xor(used, o);
    __syncthreads();
    if (lane == 0) s_wave[0][wave] = used;
    __syncthreads();
    used = 0;
    for (int w = 0; w < NTP / 64; ++w) used += s_wave[0][w];
    const int64_t left = room - used;
    // returned pages that were not popped again: only if fewer are left than
    // pushed, so that no block of this launch read the places written here
    for (int64_t v = have + tid; v < left && v < c.pages; v += NTP) a.free_list[v] = stack_page(v);
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const Demand d = demand_of(c, a, b);
        if (d.fits && (d.take == 0 || (int64_t)s_take[b] + d.take <= room)) a.held[b] = d.need;
    }
    if (tid == 0) *a.free_count = (int)min(left, (int64_t)c.pages);
}

hipError_t launch_cache_plan(const CacheDev& c, const PlanArgs& a, hipStream_t s) {
    const int blocks = c.B < 256 ? c.B : 256;
    k_cache_plan<<<blocks, NTP, 2 * sizeof(int) * (size_t)c.B, s>>>(c, a);
    return hipGetLastError();
}

}  // namespace rheo
