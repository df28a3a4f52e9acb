// Rows into and out of 4-bit pages (rheo_packed_append, rheo_packed_read,
// rheo_packed_commit).
#include "commit_walk.h"
#include "packed_format.h"

namespace rheo {

namespace {

constexpr int NTP = 256;

// One row's keys or values are K heads of 4 nb parts of eight elements; part f of them.
struct Part {
    int head, block, quarter;      // of the block
    int d;                         // its first element
};
__device__ __forceinline__ Part part_of(int f, int nb) {
    Part u;
    u.head = f / (4 * nb);
    const int r = f - u.head * 4 * nb;
    u.block = r >> 2;
    u.quarter = r & 3;
    u.d = 8 * r;
    return u;
}

// Where a part's codes and its block's exponent lie, in bytes from the page's start.
__device__ __forceinline__ int64_t codes_at(const PackedDev& p, const Part& u, int entry) {
    return u.head * p.head + ((int64_t)entry * p.nb + u.block) * 16 + u.quarter * 4;
}
__device__ __forceinline__ int64_t exponent_at(const CacheDev& c, const PackedDev& p, const Part& u,
                                               int entry) {
    return u.head * p.head + ((int64_t)(16 * p.nb + u.block) << c.page_shift) + entry;
}

// The page and the entry in it of a slot; false (and a flag) for one out of range.
__device__ __forceinline__ bool place_of(const CacheDev& c, const PackedDev& p, int64_t slot,
                                         int64_t* page, int* entry) {
    if (slot >= (int64_t)c.pages << c.page_shift) {
        atomicOr(c.err, CE_SLOT);
        return false;
    }
    *page = (slot >> c.page_shift) * p.page_stride;
    *entry = (int)slot & ((1 << c.page_shift) - 1);
    return true;
}

template <typename T>
__device__ __forceinline__ bool store_part(const CacheDev& c, const PackedDev& p, const Part& u,
                                           uint8_t* page, int entry, uint4 x) {
    uint32_t codes, scale;
    const bool bad = pack_block<T>(x, &codes, &scale);
    *(uint32_t*)(page + codes_at(p, u, entry)) = codes;
    if (u.quarter == 0) page[exponent_at(c, p, u, entry)] = (uint8_t)scale;
    return bad;
}

}  // namespace

// Rows into pages, or (READ) out of them.  Four lanes hold a block of 32 elements, 16 bytes
// each: the largest magnitude passes between them, each writes a word of codes, the first
// the exponent.  A workgroup takes ROWS rows at a time, head after head, so that what
// it writes of a head's page (or reads) is 16 entries next to each other where their slots are:
// 1 KB of codes instead of 64 bytes here and there, which the chip's eight L2 would each
// write a part of.  Bound by memory: 12064 rows of 40 heads of 80, 204 MB, 58 us into pages (79
// row by row; a copy's rate 41; 180 MB fetched for the rows' 154, 52 written for 49), and 37 out of
// them again, in part from the memory's cache (59).

template <typename T, int NB, int ROWS, bool READ>
__global__ __launch_bounds__(NTP) void k_packed_rows(CacheDev c, PackedDev p, rheo_packed_rows r,
                                                     int split, int heads) {
    constexpr int PARTS = 4 * NB;
    __shared__ int64_t s_page[ROWS];        // bytes of the row's page from the pool's start, or -1
    __shared__ int s_entry[ROWS];
    const int64_t rows = (int64_t)c.B * r.n;
    const int layer = blockIdx.y, tid = threadIdx.x;
    T* const k = (T*)r.k + layer * r.layer_stride;
    T* const v = (T*)r.v + layer * r.layer_stride;
    uint8_t* const kp = p.k + layer * p.layer_stride;
    uint8_t* const vp = p.v + layer * p.layer_stride;
    bool bad = false;
    // (`heads` of them from h0 on, the workgroup's of `split` next to each other)
    const int h0 = blockIdx.x % split * heads, end = min(heads, c.K - h0) * ROWS * PARTS;
    const int64_t step = (int64_t)(gridDim.x / split) * ROWS;
    for (int64_t r0 = (int64_t)(blockIdx.x / split) * ROWS; r0 < rows; r0 += step) {
        __syncthreads();
        if (tid < ROWS) {
            const int64_t slot = r0 + tid < rows ? r.slots[r0 + tid] : -1;
            int64_t page = 0;
            int entry = 0;
            const bool there = slot >= 0 && place_of(c, p, slot, &page, &entry);
            s_page[tid] = there ? page : -1;
            s_entry[tid] = entry;
        }
        __syncthreads();
        // (a multiple of four: a block's lanes are all here or none)
        for (int f0 = tid; f0 < end; f0 += 2 * NTP) {
            // two parts at a time, all their loads first
            Part u[2];
            int64_t page[2], at[2];
            int entry[2];
            uint4 x[2], y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int f = f0 + j * NTP, g = f / PARTS, i = g % ROWS, q = f % PARTS;
                page[j] = f < end ? s_page[i] : -1;
                entry[j] = s_entry[i];
                u[j] = Part{h0 + g / ROWS, q >> 2, q & 3, 8 * q};
                at[j] = (r0 + i) * r.row_stride + u[j].head * c.D + u[j].d;
                x[j] = y[j] = make_uint4(0, 0, 0, 0);
                if (page[j] < 0) continue;
                if constexpr (!READ) {
                    if (u[j].d < c.D) {
                        x[j] = *(const uint4*)(k + at[j]);
                        y[j] = *(const uint4*)(v + at[j]);
                    }
                } else {
                    const int64_t codes = page[j] + codes_at(p, u[j], entry[j]);
                    const int64_t exps = page[j] + exponent_at(c, p, u[j], entry[j]);
                    x[j].x = *(const uint32_t*)(kp + codes);
                    y[j].x = *(const uint32_t*)(vp + codes);
                    x[j].y = kp[exps];
                    y[j].y = vp[exps];
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (page[j] < 0) continue;
                if constexpr (!READ) {
                    bad |= store_part<T>(c, p, u[j], kp + page[j], entry[j], x[j]);
                    bad |= store_part<T>(c, p, u[j], vp + page[j], entry[j], y[j]);
                } else if (u[j].d < c.D) {
                    // (every code's value is exact in T)
                    const float f = scale_of(x[j].y), g = scale_of(y[j].y);
                    *(uint4*)(k + at[j]) = make_uint4(pair_of<T, 0>(x[j].x, f), pair_of<T, 1>(x[j].x, f),
                                                      pair_of<T, 2>(x[j].x, f), pair_of<T, 3>(x[j].x, f));
                    *(uint4*)(v + at[j]) = make_uint4(pair_of<T, 0>(y[j].x, g), pair_of<T, 1>(y[j].x, g),
                                                      pair_of<T, 2>(y[j].x, g), pair_of<T, 3>(y[j].x, g));
                }
            }
        }
    }
    if (!READ && __any(bad) && (tid & 63) == 0) atomicOr(c.err, CE_VALUE);
}

// Every block of a sequence walks the accepted path for itself, then rounds its share of
// the layers' rows into the pages, a part of all the path's rows a thread.  Rows and pages are
// different memory, so the order is free.  The sequence's last block writes the length, which
// may be lens itself.  Bound by memory, after the walk: 128 sequences, 32 layers, 5 entries on
// average (108 MB; 86 fetched, 28 written for 23) 34 us (a copy's rate 22); one sequence 5, the
// walk's latency.  (The path's rows of a head by neighbouring threads: 39 to 51 us.)
template <typename T>
__global__ __launch_bounds__(NTP) void k_packed_commit(CacheDev c, PackedDev p,
                                                       rheo_packed_commit_args a, int split) {
    __shared__ int64_t s_page[kDepthMax + 1];
    __shared__ int s_path[kDepthMax + 1], s_entry[kDepthMax + 1];
    __shared__ int s_moves, s_len;
    const int b = blockIdx.x / split, part = blockIdx.x - b * split;
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) {
        const int len = a.lens[b], took = a.status && a.status[b] ? -1 : a.accept_len[b];
        const int64_t room = (int64_t)c.width << c.page_shift;
        int bad = 0;
        if (took > a.depth || took >= a.n) bad = CE_PATH;
        if (took >= 0 && (len < 0 || (int64_t)len + 1 + took > room)) bad |= CE_TABLE;
        if (took >= 0 && !bad)
            bad = walk_path(lane, a.n, a.parent + (int64_t)b * a.n, a.token + (int64_t)b * a.n,
                            a.accepted + (int64_t)b * a.depth, took, s_path);
        if (took >= 0 && !bad && lane <= took) {
            const int e = len + lane, page = a.table[(int64_t)b * c.width + (e >> c.page_shift)];
            if ((unsigned)page >= (unsigned)c.pages) bad = CE_PAGE;
            s_page[lane] = page * p.page_stride;
            s_entry[lane] = e & ((1 << c.page_shift) - 1);
        }
        bad |= __any(bad & CE_PAGE) ? CE_PAGE : 0;
        const bool good = took >= 0 && !bad;
        __builtin_amdgcn_wave_barrier();
        if (lane == 0) {
            s_moves = good ? took + 1 : 0;
            s_len = good ? len + 1 + took : len;
            if (bad && part == 0) atomicOr(c.err, bad);
        }
        if (part == 0 && lane <= a.depth)
            a.path[(int64_t)b * (a.depth + 1) + lane] =
                good && lane <= took ? *(volatile int*)&s_path[lane] : -1;
    }
    __syncthreads();
    const int moves = s_moves;
    bool wrong = false;
    if (moves) {
        const int parts = c.K * 4 * p.nb, total = c.layers * 2 * parts;
        for (int f = part * NTP + tid; f < total; f += split * NTP) {
            const int layer = f / (2 * parts), g = f - layer * 2 * parts;
            const bool keys = g < parts;
            const Part u = part_of(keys ? g : g - parts, p.nb);
            const T* x = (const T*)(keys ? a.k : a.v) + layer * a.layer_stride +
                         (int64_t)b * a.n * a.row_stride + u.head * c.D + u.d;
            uint8_t* pages = (keys ? p.k : p.v) + layer * p.layer_stride;
            const bool in = u.d < c.D;
            // four rows at a time (`moves` is the block's)
            for (int j0 = 0; j0 < moves; j0 += 4) {
                uint4 y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    y[j] = make_uint4(0, 0, 0, 0);
                    if (in && j0 + j < moves) y[j] = *(const uint4*)(x + s_path[j0 + j] * a.row_stride);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j0 + j < moves)
                        wrong |= store_part<T>(c, p, u, pages + s_page[j0 + j], s_entry[j0 + j], y[j]);
            }
        }
    }
    if (__any(wrong) && lane == 0) atomicOr(c.err, CE_VALUE);
    __syncthreads();
    if (tid == 0) {
        if (split == 1 || __hip_atomic_fetch_add(c.ticket + b, 1u, __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)split - 1) {
            if (split > 1) c.ticket[b] = 0;
            a.new_lens[b] = s_len;
        }
    }
}

namespace {

// f(a constant: the blocks of 32 elements of a head, 1 to 8)
template <typename F>
hipError_t by_blocks(int nb, F f) {
    switch (nb) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 3: f(std::integral_constant<int, 3>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 5: f(std::integral_constant<int, 5>()); break;
    case 6: f(std::integral_constant<int, 6>()); break;
    case 7: f(std::integral_constant<int, 7>()); break;
    default: f(std::integral_constant<int, 8>());
    }
    return hipGetLastError();
}

template <typename T, bool READ>
hipError_t start_rows(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r, hipStream_t s) {
    return by_blocks(p.nb, [&](auto nb) {
        // a sequence's few rows are next to no others: one at a time (one row of 8 heads 2.7 us,
        // as one of 16 5.4)
        const int rows = r.n < 8 ? 1 : 16;
        const int64_t groups = ((int64_t)c.B * r.n + rows - 1) / rows;
        // some four parts a thread: more workgroups, where rows are few, than one for all heads
        const int most_heads = 4 * NTP / (rows * 4 * nb), heads = most_heads < 1 ? 1 : most_heads;
        const int split = (c.K + heads - 1) / heads;
        int64_t most = (1 << 22) / ((int64_t)r.layers * split);   // (fewer than 2^32 threads)
        if (most < 1) most = 1;
        const dim3 grid((int)(groups < most ? groups : most) * split, r.layers);
        if (rows == 1) k_packed_rows<T, nb, 1, READ><<<grid, NTP, 0, s>>>(c, p, r, split, heads);
        else k_packed_rows<T, nb, 16, READ><<<grid, NTP, 0, s>>>(c, p, r, split, heads);
    });
}

}  // namespace

hipError_t launch_packed_append(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                                hipStream_t s) {
    return c.dtype == RHEO_BF16 ? start_rows<__bf16, false>(c, p, r, s)
                                : start_rows<_Float16, false>(c, p, r, s);
}

hipError_t launch_packed_read(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                              hipStream_t s) {
    return c.dtype == RHEO_BF16 ? start_rows<__bf16, true>(c, p, r, s)
                                : start_rows<_Float16, true>(c, p, r, s);
}

hipError_t launch_packed_commit(const CacheDev& c, const PackedDev& p,
                                const rheo_packed_commit_args& a, hipStream_t s) {
    const int total = c.layers * 2 * (c.K * 4 * p.nb);
    // one part a thread while that makes at most 2048 blocks in all
    int split = (total + NTP - 1) / NTP;
    if ((int64_t)split * c.B > 2048) split = 2048 / c.B;
    if (split < 1) split = 1;
    if (c.dtype == RHEO_BF16) k_packed_commit<__bf16><<<c.B * split, NTP, 0, s>>>(c, p, a, split);
    else k_packed_commit<_Float16><<<c.B * split, NTP, 0, s>>>(c, p, a, split);
    return hipGetLastError();
}

}  // namespace rheo
