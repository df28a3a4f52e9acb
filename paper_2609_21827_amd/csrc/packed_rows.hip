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

// Four lanes hold a block of 32 elements, 16 bytes each: the largest magnitude passes
// between them, each writes a word of codes, the first the exponent.  A block of threads
// takes `each` rows at a time, some 4096 elements or a row.  Bound by memory.
template <typename T>
__global__ __launch_bounds__(NTP) void k_packed_append(CacheDev c, PackedDev p, rheo_packed_rows r,
                                                       int each) {
    const int parts = c.K * 4 * p.nb;
    const int64_t rows = (int64_t)c.B * r.n;
    const int layer = blockIdx.y;
    const T* const k = (const T*)r.k + layer * r.layer_stride;
    const T* const v = (const T*)r.v + layer * r.layer_stride;
    uint8_t* const kp = p.k + layer * p.layer_stride;
    uint8_t* const vp = p.v + layer * p.layer_stride;
    bool bad = false;
    for (int64_t r0 = (int64_t)blockIdx.x * each; r0 < rows; r0 += (int64_t)gridDim.x * each) {
        const int here = (int)min((int64_t)each, rows - r0);
        for (int f = threadIdx.x; f < here * parts; f += NTP) {
            const int i = f / parts;
            const int64_t row = r0 + i, slot = r.slots[row];
            if (slot < 0) continue;
            int64_t page;
            int entry;
            if (!place_of(c, p, slot, &page, &entry)) continue;
            const Part u = part_of(f - i * parts, p.nb);
            const int64_t at = row * r.row_stride + u.head * c.D + u.d;
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (u.d < c.D) {
                x = *(const uint4*)(k + at);
                y = *(const uint4*)(v + at);
            }
            bad |= store_part<T>(c, p, u, kp + page, entry, x);
            bad |= store_part<T>(c, p, u, vp + page, entry, y);
        }
    }
    if (__any(bad) && (threadIdx.x & 63) == 0) atomicOr(c.err, CE_VALUE);
}

// The same turned round.  Every code's value is exact in T.
template <typename T>
__global__ __launch_bounds__(NTP) void k_packed_read(CacheDev c, PackedDev p, rheo_packed_rows r,
                                                     int each) {
    const int parts = c.K * 4 * p.nb;
    const int64_t rows = (int64_t)c.B * r.n;
    const int layer = blockIdx.y;
    T* const k = (T*)r.k + layer * r.layer_stride;
    T* const v = (T*)r.v + layer * r.layer_stride;
    const uint8_t* const kp = p.k + layer * p.layer_stride;
    const uint8_t* const vp = p.v + layer * p.layer_stride;
    for (int64_t r0 = (int64_t)blockIdx.x * each; r0 < rows; r0 += (int64_t)gridDim.x * each) {
        const int here = (int)min((int64_t)each, rows - r0);
        for (int f = threadIdx.x; f < here * parts; f += NTP) {
            const int i = f / parts;
            const int64_t row = r0 + i, slot = r.slots[row];
            if (slot < 0) continue;
            int64_t page;
            int entry;
            if (!place_of(c, p, slot, &page, &entry)) continue;
            const Part u = part_of(f - i * parts, p.nb);
            if (u.d >= c.D) continue;
            const int64_t codes = page + codes_at(p, u, entry);
            const int64_t at_scale = page + exponent_at(c, p, u, entry);
            const int64_t at = row * r.row_stride + u.head * c.D + u.d;
            const uint32_t x = *(const uint32_t*)(kp + codes), y = *(const uint32_t*)(vp + codes);
            const float f_x = scale_of(kp[at_scale]), f_y = scale_of(vp[at_scale]);
            *(uint4*)(k + at) = make_uint4(pair_of<T, 0>(x, f_x), pair_of<T, 1>(x, f_x),
                                           pair_of<T, 2>(x, f_x), pair_of<T, 3>(x, f_x));
            *(uint4*)(v + at) = make_uint4(pair_of<T, 0>(y, f_y), pair_of<T, 1>(y, f_y),
                                           pair_of<T, 2>(y, f_y), pair_of<T, 3>(y, f_y));
        }
    }
}

// Every block of a sequence walks the accepted path for itself, then rounds its share of
// the layers' rows into the pages.  Rows and pages are different memory, so the order is
// free.  The sequence's last block writes the length, which may be lens itself.
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

// Rows that a block takes at a time, and blocks.
struct Cut {
    int each, blocks;
};
Cut cut_rows(const CacheDev& c, const PackedDev& p, int64_t rows, int layers) {
    const int parts = c.K * 4 * p.nb;
    const int each = parts < 512 ? 512 / parts : 1;
    const int64_t blocks = (rows + each - 1) / each;
    const int most = 65536 / layers;         // (a launch has less than 2^32 threads)
    return {each, (int)(blocks < most ? blocks : most)};
}

}  // namespace

hipError_t launch_packed_append(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                                hipStream_t s) {
    const Cut t = cut_rows(c, p, (int64_t)c.B * r.n, r.layers);
    const dim3 grid(t.blocks, r.layers);
    if (c.dtype == RHEO_BF16) k_packed_append<__bf16><<<grid, NTP, 0, s>>>(c, p, r, t.each);
    else k_packed_append<_Float16><<<grid, NTP, 0, s>>>(c, p, r, t.each);
    return hipGetLastError();
}

hipError_t launch_packed_read(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                              hipStream_t s) {
    const Cut t = cut_rows(c, p, (int64_t)c.B * r.n, r.layers);
    const dim3 grid(t.blocks, r.layers);
    if (c.dtype == RHEO_BF16) k_packed_read<__bf16><<<grid, NTP, 0, s>>>(c, p, r, t.each);
    else k_packed_read<_Float16><<<grid, NTP, 0, s>>>(c, p, r, t.each);
    return hipGetLastError();
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
