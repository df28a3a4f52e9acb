// Host side of the cache and scoring calls of include/rheo.h: validation,
// workspaces and kernel launches.
#include <cmath>
#include <new>

#include "api_common.h"
#include "cache_state.h"
#include "rheo.h"
#include "score_state.h"

using namespace rheo;

struct rheo_cache {
    CacheDev dev;
    int device = 0;
};

struct rheo_scorer {
    ScoreDev dev;
    int device = 0;
};

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;   // rows of one call
// entries of one scoring call: a block of 256 threads each, less than 2^32 in all
constexpr int64_t kMaxEntries = ((int64_t)1 << 24) - 1;

int zeroed(void** p, size_t bytes) {
    hipError_t e = hipMalloc(p, bytes);
    if (e != hipSuccess) {
        *p = nullptr;
        return fail(RHEO_ENOMEM, "hipMalloc(%zu): %s", bytes, hipGetErrorString(e));
    }
    e = hipMemset(*p, 0, bytes);
    return e == hipSuccess ? RHEO_OK : hip_fail(e, "initialising a workspace");
}

int check_words(const void* p, size_t size, const char* name) {
    if (!p) return fail(RHEO_EINVAL, "%s is NULL", name);
    if ((uintptr_t)p % size) return fail(RHEO_EINVAL, "%s is not %zu-byte aligned", name, size);
    return RHEO_OK;
}

int check_stride(int64_t stride, int64_t least, const char* name) {
    if (stride < least)
        return fail(RHEO_EINVAL, "%s must be >= %lld", name, (long long)least);
    if (stride % 8) return fail(RHEO_EINVAL, "%s must be a multiple of 16 bytes", name);
    // (kMaxRows rows of it stay within 64 bits)
    if (stride > ((int64_t)1 << 31)) return fail(RHEO_EINVAL, "%s is too large", name);
    return RHEO_OK;
}

int check_rows(const CacheDev& d, int32_t n, int least, int64_t most = kMaxRows) {
    if (n < least || (int64_t)d.B * n > most)
        return fail(RHEO_EINVAL, "n must be in [%d, %lld]", least, (long long)(most / d.B));
    return RHEO_OK;
}

bool overlap(const void* p, size_t np, const void* q, size_t nq) {
    return (const char*)p < (const char*)q + nq && (const char*)q < (const char*)p + np;
}

int launched(hipError_t e, const char* what) { return e == hipSuccess ? RHEO_OK : hip_fail(e, what); }

void free_cache(rheo_cache* c) {
    if (c->dev.err) (void)hipFree(c->dev.err);
    if (c->dev.ticket) (void)hipFree(c->dev.ticket);
    if (c->dev.part) (void)hipFree(c->dev.part);
    delete c;
}

}  // namespace

extern "C" {

int rheo_cache_create(const rheo_cache_config* cfg, rheo_cache** out) {
    if (!cfg || !out) return fail(RHEO_EINVAL, "NULL argument");
    const rheo_cache_config& g = *cfg;
    if (g.batch < 1 || g.batch > 4096) return fail(RHEO_EINVAL, "batch must be in [1, 4096]");
    if (g.kv_heads < 1) return fail(RHEO_EINVAL, "kv_heads must be >= 1");
    if (g.heads < 1 || g.heads > 1024 || g.heads % g.kv_heads)
        return fail(RHEO_EINVAL, "heads must be a multiple of kv_heads in [1, 1024]");
    if (g.head_dim < 8 || g.head_dim > 256 || g.head_dim % 8)
        return fail(RHEO_EINVAL, "head_dim must be a multiple of 8 in [8, 256]");
    if (g.page_size < 1 || g.page_size > 4096 || (g.page_size & (g.page_size - 1)))
        return fail(RHEO_EINVAL, "page_size must be a power of two in [1, 4096]");
    if (g.pages < 1) return fail(RHEO_EINVAL, "pages must be >= 1");
    if (g.table_width < 1 || (int64_t)g.table_width * g.page_size > (1 << 30))
        return fail(RHEO_EINVAL, "table_width must be >= 1 and a row's entries at most 2^30");
    if (g.layers < 1 || g.layers > 1024) return fail(RHEO_EINVAL, "layers must be in [1, 1024]");
    if (g.dtype != RHEO_BF16 && g.dtype != RHEO_F16) return fail(RHEO_EINVAL, "unknown dtype");
    const int64_t page = (int64_t)g.page_size * g.kv_heads * g.head_dim;
    const int64_t page_stride = g.page_stride ? g.page_stride : page;
    if (page_stride < page || page_stride % 8 || page_stride > ((int64_t)1 << 40))
        return fail(RHEO_EINVAL, "page_stride must hold a page and be a multiple of 16 bytes");
    // (byte offsets of a pool's entries stay within 64 bits)
    if (page_stride > ((int64_t)1 << 48) / g.pages)
        return fail(RHEO_EINVAL, "pages * page_stride must be at most 2^48");
    // (the last page need not be followed by a gap)
    const int64_t layer = (g.pages - 1) * page_stride + page;
    const int64_t layer_stride = g.layer_stride ? g.layer_stride : g.pages * page_stride;
    if (g.layers > 1 && (layer_stride < layer || layer_stride % 8 ||
                         layer_stride > ((int64_t)1 << 48)))
        return fail(RHEO_EINVAL, "layer_stride must hold a layer and be a multiple of 16 bytes");

    rheo_cache* c = new (std::nothrow) rheo_cache();
    if (!c) return fail(RHEO_ENOMEM, "out of host memory");
    CacheDev& d = c->dev;
    d = CacheDev{};
    d.B = g.batch; d.H = g.heads; d.K = g.kv_heads; d.D = g.head_dim;
    d.page_shift = __builtin_ctz((unsigned)g.page_size);
    d.pages = g.pages; d.width = g.table_width; d.layers = g.layers; d.dtype = g.dtype;
    d.page_stride = page_stride; d.layer_stride = layer_stride;
    hipError_t e = hipGetDevice(&c->device);
    if (e == hipSuccess)
        e = hipDeviceGetAttribute(&d.slots, hipDeviceAttributeMultiprocessorCount, c->device);
    int rc = e == hipSuccess ? RHEO_OK : hip_fail(e, "hipGetDevice");
    if (rc == RHEO_OK) rc = zeroed((void**)&d.err, sizeof(int32_t));
    if (rc == RHEO_OK) rc = zeroed((void**)&d.ticket, (d.B + 1) * sizeof(uint32_t));
    if (rc == RHEO_OK) rc = zeroed((void**)&d.part, attention_workspace(d) * sizeof(float));
    if (rc == RHEO_OK && (e = prepare_attention(d)) != hipSuccess)
        rc = hip_fail(e, "tree attention set-up");
    if (rc == RHEO_OK && (e = hipDeviceSynchronize()) != hipSuccess)
        rc = hip_fail(e, "initialising a workspace");
    if (rc != RHEO_OK) {
        free_cache(c);
        return rc;
    }
    *out = c;
    return RHEO_OK;
}

int rheo_cache_destroy(rheo_cache* c) {
    if (!c) return RHEO_OK;
    OnDevice on(c->device);
    (void)hipDeviceSynchronize();
    free_cache(c);
    return RHEO_OK;
}

int rheo_cache_error(rheo_cache* c, int32_t* host_flag) {
    if (!c || !host_flag) return fail(RHEO_EINVAL, "NULL argument");
    OnDevice on(c->device);
    hipError_t e = on.error();
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e == hipSuccess) e = hipMemcpy(host_flag, c->dev.err, sizeof(int32_t), hipMemcpyDeviceToHost);
    return launched(e, "reading the device error flag");
}

int rheo_cache_plan(rheo_cache* c, int32_t n, const int32_t* lens, const int32_t* count,
                    const int32_t* depth, int32_t* held, int32_t* table, int32_t* free_list,
                    int32_t* free_count, int64_t* slots, int32_t* positions, int32_t* status,
                    void* stream) {
    if (!c) return fail(RHEO_EINVAL, "NULL cache");
    int rc = check_rows(c->dev, n, 0);
    if (rc == RHEO_OK) rc = check_words(lens, 4, "lens");
    if (rc == RHEO_OK) rc = check_words(held, 4, "held");
    if (rc == RHEO_OK) rc = check_words(table, 4, "table");
    if (rc == RHEO_OK) rc = check_words(free_list, 4, "free_list");
    if (rc == RHEO_OK) rc = check_words(free_count, 4, "free_count");
    if (rc == RHEO_OK) rc = check_words(status, 4, "status");
    if (rc == RHEO_OK && n) rc = check_words(slots, 8, "slots");
    if (rc == RHEO_OK && n) rc = check_words(positions, 4, "positions");
    if (rc == RHEO_OK && count) rc = check_words(count, 4, "count");
    if (rc == RHEO_OK && depth) rc = check_words(depth, 4, "depth");
    if (rc) return rc;
    OnDevice on(c->device);
    if (on.error() != hipSuccess) return hip_fail(on.error(), "hipSetDevice");
    const PlanArgs a{n, lens, count, depth, held, table, free_list, free_count, slots, positions,
                     status};
    return launched(launch_cache_plan(c->dev, a, (hipStream_t)stream), "cache plan launch");
}

int rheo_cache_write(rheo_cache* c, const rheo_write_args* args, void* stream) {
    if (!c || !args) return fail(RHEO_EINVAL, "NULL argument");
    const rheo_write_args& a = *args;
    const CacheDev& d = c->dev;
    int rc = check_rows(d, a.n, 0, kWriteRows);
    if (rc) return rc;
    if (a.rot_dim < 0 || a.rot_dim > d.D || a.rot_dim % 2)
        return fail(RHEO_EINVAL, "rot_dim must be even and in [0, head_dim]");
    if (a.interleaved != 0 && a.interleaved != 1)
        return fail(RHEO_EINVAL, "interleaved must be 0 or 1");
    if (!(a.eps >= 0.0f) || !std::isfinite(a.eps)) return fail(RHEO_EINVAL, "eps must be >= 0");
    if (a.n == 0) return RHEO_OK;            // (empty arrays may have no address)
    if (!a.q != !a.q_out) return fail(RHEO_EINVAL, "q and q_out: both or none");
    if (a.q) {
        if ((rc = check_ptr(a.q, "q")) || (rc = check_ptr(a.q_out, "q_out"))) return rc;
        if ((rc = check_stride(a.q_stride, (int64_t)d.H * d.D, "q_stride"))) return rc;
        if ((rc = check_stride(a.q_out_stride, (int64_t)d.H * d.D, "q_out_stride"))) return rc;
        if (a.q == a.q_out && a.q_stride != a.q_out_stride)
            return fail(RHEO_EINVAL, "q_out may be q itself only with q's stride");
    }
    if ((rc = check_ptr(a.k, "k")) || (rc = check_ptr(a.v, "v"))) return rc;
    if ((rc = check_stride(a.k_stride, (int64_t)d.K * d.D, "k_stride"))) return rc;
    if ((rc = check_stride(a.v_stride, (int64_t)d.K * d.D, "v_stride"))) return rc;
    if ((rc = check_words(a.slots, 8, "slots"))) return rc;
    if (a.rot_dim) {
        if ((rc = check_words(a.positions, 4, "positions"))) return rc;
        if ((rc = check_words(a.rotation, 4, "rotation"))) return rc;
        if (a.max_position < 1) return fail(RHEO_EINVAL, "max_position must be >= 1");
    }
    if (a.q_weight && (rc = check_ptr(a.q_weight, "q_weight"))) return rc;
    if (a.k_weight && (rc = check_ptr(a.k_weight, "k_weight"))) return rc;
    if ((rc = check_ptr(a.k_cache, "k_cache")) || (rc = check_ptr(a.v_cache, "v_cache"))) return rc;
    OnDevice on(c->device);
    if (on.error() != hipSuccess) return hip_fail(on.error(), "hipSetDevice");
    return launched(launch_cache_write(d, a, (hipStream_t)stream), "cache write launch");
}

int rheo_tree_attention(rheo_cache* c, const rheo_attention_args* args, void* stream) {
    if (!c || !args) return fail(RHEO_EINVAL, "NULL argument");
    const rheo_attention_args& a = *args;
    const CacheDev& d = c->dev;
    int rc = check_rows(d, a.n, 0);
    if (rc) return rc;
    if ((int64_t)a.n * d.H > kMaxRows) return fail(RHEO_EINVAL, "n * heads must be <= 2^30");
    // (a tail of 2^24 entries: its masks' rows stay within 32 bits of each other)
    if (a.tail < 0 || a.tail > (1 << 24)) return fail(RHEO_EINVAL, "tail must be in [0, 2^24]");
    if (!a.mask && a.tail < a.n) return fail(RHEO_EINVAL, "tail must be >= n without a mask");
    // (8 / scale, the slack of the kernel's reference, and scale log2(e) stay finite)
    if (!(a.scale >= 0x1p-100f && a.scale <= 0x1p100f))
        return fail(RHEO_EINVAL, "scale must be in [2^-100, 2^100]");
    if (a.n == 0) return RHEO_OK;            // (empty arrays may have no address)
    if ((rc = check_ptr(a.q, "q")) || (rc = check_ptr(a.out, "out"))) return rc;
    if ((rc = check_stride(a.q_stride, (int64_t)d.H * d.D, "q_stride"))) return rc;
    if ((rc = check_stride(a.out_stride, (int64_t)d.H * d.D, "out_stride"))) return rc;
    if (a.q == a.out) return fail(RHEO_EINVAL, "out must not be q");
    if ((rc = check_ptr(a.k_cache, "k_cache")) || (rc = check_ptr(a.v_cache, "v_cache"))) return rc;
    if ((rc = check_words(a.table, 4, "table")) || (rc = check_words(a.lens, 4, "lens"))) return rc;
    if (a.count && (rc = check_words(a.count, 4, "count"))) return rc;
    if (a.lse && (rc = check_words(a.lse, 4, "lse"))) return rc;
    if (a.status && (rc = check_words(a.status, 4, "status"))) return rc;
    OnDevice on(c->device);
    if (on.error() != hipSuccess) return hip_fail(on.error(), "hipSetDevice");
    return launched(launch_tree_attention(d, a, (hipStream_t)stream), "tree attention launch");
}

int rheo_cache_commit(rheo_cache* c, int32_t n, int32_t depth, const int32_t* parent,
                      const int32_t* token, const int32_t* accepted, const int32_t* accept_len,
                      const int32_t* lens, const int32_t* table, void* k_cache, void* v_cache,
                      int32_t* path, int32_t* new_lens, void* stream) {
    return rheo_cache_commit_served(c, n, depth, parent, token, accepted, accept_len, lens, table,
                                    nullptr, k_cache, v_cache, path, new_lens, stream);
}

int rheo_cache_commit_served(rheo_cache* c, int32_t n, int32_t depth, const int32_t* parent,
                             const int32_t* token, const int32_t* accepted,
                             const int32_t* accept_len, const int32_t* lens, const int32_t* table,
                             const int32_t* status, void* k_cache, void* v_cache, int32_t* path,
                             int32_t* new_lens, void* stream) {
    if (!c) return fail(RHEO_EINVAL, "NULL cache");
    const CacheDev& d = c->dev;
    int rc = check_rows(d, n, 1);
    if (rc) return rc;
    if (depth < 1 || depth > 15) return fail(RHEO_EINVAL, "depth must be in [1, 15]");
    if ((rc = check_words(parent, 4, "parent")) || (rc = check_words(token, 4, "token")) ||
        (rc = check_words(accepted, 4, "accepted")) ||
        (rc = check_words(accept_len, 4, "accept_len")) || (rc = check_words(lens, 4, "lens")) ||
        (rc = check_words(table, 4, "table")) || (rc = check_ptr(k_cache, "k_cache")) ||
        (rc = check_ptr(v_cache, "v_cache")) || (rc = check_words(path, 4, "path")) ||
        (rc = check_words(new_lens, 4, "new_lens")))
        return rc;
    if (status && (rc = check_words(status, 4, "status"))) return rc;
    if (new_lens != lens && overlap(new_lens, 4 * (size_t)d.B, lens, 4 * (size_t)d.B))
        return fail(RHEO_EINVAL, "new_lens overlaps lens");
    OnDevice on(c->device);
    if (on.error() != hipSuccess) return hip_fail(on.error(), "hipSetDevice");
    const CommitArgs a{n, depth, parent, token, accepted, accept_len, lens, table, status,
                       (char*)k_cache, (char*)v_cache, path, new_lens};
    return launched(launch_cache_commit(d, a, (hipStream_t)stream), "cache commit launch");
}

int rheo_scorer_create(int32_t vocab, int32_t dtype, int64_t row_stride, rheo_scorer** out) {
    if (!out) return fail(RHEO_EINVAL, "NULL argument");
    if (vocab < 2 || vocab > (1 << 24)) return fail(RHEO_EINVAL, "vocab must be in [2, 2^24]");
    if (dtype != RHEO_F32 && dtype != RHEO_BF16 && dtype != RHEO_F16)
        return fail(RHEO_EINVAL, "unknown dtype");
    if (row_stride < vocab || row_stride > ((int64_t)1 << 32))
        return fail(RHEO_EINVAL, "row_stride must be >= vocab (and at most 2^32)");
    if (row_stride * (dtype == RHEO_F32 ? 4 : 2) % 16)
        return fail(RHEO_EINVAL, "row_stride must be a multiple of 16 bytes");
    rheo_scorer* s = new (std::nothrow) rheo_scorer();
    if (!s) return fail(RHEO_ENOMEM, "out of host memory");
    s->dev = ScoreDev{vocab, dtype, row_stride, nullptr};
    hipError_t e = hipGetDevice(&s->device);
    int rc = e == hipSuccess ? RHEO_OK : hip_fail(e, "hipGetDevice");
    if (rc == RHEO_OK) rc = zeroed((void**)&s->dev.work, score_workspace());
    // (the fill must not land in a first call's results on another stream)
    if (rc == RHEO_OK && (e = hipDeviceSynchronize()) != hipSuccess)
        rc = hip_fail(e, "initialising a workspace");
    if (rc != RHEO_OK) {
        if (s->dev.work) (void)hipFree(s->dev.work);
        delete s;
        return rc;
    }
    *out = s;
    return RHEO_OK;
}

int rheo_scorer_destroy(rheo_scorer* s) {
    if (!s) return RHEO_OK;
    OnDevice on(s->device);
    (void)hipDeviceSynchronize();
    (void)hipFree(s->dev.work);
    delete s;
    return RHEO_OK;
}

int rheo_token_logprobs(rheo_scorer* s, const void* logits, int32_t B, int32_t n,
                        const int32_t* path, const int32_t* token, int32_t m, int32_t top,
                        float T, float* logprob, float* entropy, int32_t* rank,
                        int32_t* top_token, float* top_logprob, void* stream) {
    if (!s) return fail(RHEO_EINVAL, "NULL scorer");
    if (B < 0 || n < 0 || m < 0 || (int64_t)B * n > kMaxRows || (int64_t)B * m > kMaxEntries)
        return fail(RHEO_EINVAL, "B, n and m must be >= 0, B * n <= 2^30 and B * m < 2^24");
    if (!path && m > n) return fail(RHEO_EINVAL, "m must be <= n without a path");
    if (top < 0 || top > 32 || top > s->dev.V)
        return fail(RHEO_EINVAL, "top must be in [0, min(32, vocab)]");
    if (!(T > 0.0f) || !std::isfinite(T) || !std::isfinite((float)(1.4426950408889634 / T)))
        return fail(RHEO_EINVAL, "temperature must be finite, > 0 and not too small");
    if ((int64_t)B * m == 0 || n == 0) return RHEO_OK;
    int rc;
    if ((rc = check_ptr(logits, "logits")) || (rc = check_words(token, 4, "token")) ||
        (rc = check_words(logprob, 4, "logprob")))
        return rc;
    if ((path && (rc = check_words(path, 4, "path"))) ||
        (entropy && (rc = check_words(entropy, 4, "entropy"))) ||
        (rank && (rc = check_words(rank, 4, "rank"))))
        return rc;
    if (top && ((rc = check_words(top_token, 4, "top_token")) ||
                (rc = check_words(top_logprob, 4, "top_logprob"))))
        return rc;
    OnDevice on(s->device);
    if (on.error() != hipSuccess) return hip_fail(on.error(), "hipSetDevice");
    const LogprobArgs a{(const char*)logits, B, n, m, top, path, token,
                        (float)(1.4426950408889634 / (double)T), T, logprob, entropy, rank,
                        top_token, top_logprob};
    return launched(launch_token_logprobs(s->dev, a, (hipStream_t)stream), "token logprobs launch");
}

}  // extern "C"
