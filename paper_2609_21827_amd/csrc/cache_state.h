// Device state of a cache handle and the launches of its operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rheo.h"

namespace rheo {

// bits of the handle's sticky error flag (rheo_cache_error)
enum CacheError { CE_PLAN = 1, CE_SLOT = 2, CE_POSITION = 4, CE_PAGE = 8, CE_PATH = 16,
                  CE_TABLE = 32, CE_VALUE = 64 };

// most rows of a rheo_cache_write: a wave each, and a launch has less than 2^32 threads
constexpr int64_t kWriteRows = ((int64_t)1 << 26) - 4;

struct CacheDev {
    int B, H, K, D;                // sequences, query heads, key/value heads, head size
    int page_shift, pages, width, layers;
    int dtype;
    int64_t page_stride, layer_stride;
    int32_t* err;
    uint32_t* ticket;              // [B + 1] arrivals, 0 between launches: a sequence's, the plan's
    float* part;                   // attention: partial results (see attention.hip)
    int slots;                     // attention: compute units of the device
};

struct PlanArgs {
    int n;
    const int32_t *lens, *count, *depth;
    int32_t *held, *table, *free_list, *free_count;
    int64_t* slots;
    int32_t *positions, *status;
};

struct CommitArgs {
    int n, depth;
    const int32_t *parent, *token, *accepted, *accept_len, *lens, *table;
    const int32_t* status;         // or NULL
    char *k_cache, *v_cache;
    int32_t *path, *new_lens;
};

// The 4-bit pages as the kernels take them.
struct PackedDev {
    uint8_t *k, *v;
    int64_t page_stride, layer_stride, head;   // bytes between pages, layers, a page's heads
    int nb;                        // blocks of 32 elements of a head
};

hipError_t launch_packed_append(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                                hipStream_t s);
hipError_t launch_packed_read(const CacheDev& c, const PackedDev& p, const rheo_packed_rows& r,
                              hipStream_t s);
hipError_t launch_packed_commit(const CacheDev& c, const PackedDev& p,
                                const rheo_packed_commit_args& a, hipStream_t s);
hipError_t launch_packed_attention(const CacheDev& c, const PackedDev& p,
                                   const rheo_packed_attention_args& a, hipStream_t s);
// floats of partial results that launch_packed_attention may write
size_t packed_workspace(const CacheDev& c);

hipError_t launch_cache_plan(const CacheDev& c, const PlanArgs& a, hipStream_t s);
hipError_t launch_cache_write(const CacheDev& c, const rheo_write_args& a, hipStream_t s);
hipError_t launch_tree_attention(const CacheDev& c, const rheo_attention_args& a, hipStream_t s);
hipError_t launch_cache_commit(const CacheDev& c, const CommitArgs& a, hipStream_t s);
// once for the current device, before the first launch
hipError_t prepare_attention(const CacheDev& c);
hipError_t prepare_packed(const CacheDev& c);
// floats of partial results that launch_tree_attention may write
size_t attention_workspace(const CacheDev& c);

}  // namespace rheo
