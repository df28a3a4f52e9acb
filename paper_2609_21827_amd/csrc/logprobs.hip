// Log probabilities of given tokens, entropy, rank and the top of their rows
// (rheo_token_logprobs).
#include <type_traits>

#include "half_types.h"
#include "rheo.h"
#include "rheo_device.h"
#include "score_state.h"

namespace rheo {

namespace {

constexpr int NTL = 512;                  // threads of a block
constexpr int NWL = NTL / 64;
constexpr int EPT = 16;                   // elements a thread holds of a chunk
constexpr int CHUNK = NTL * EPT;          // 8192 elements
constexpr int TOP = 32;                   // most alternatives
constexpr int LIST = 1024;                // most candidates of a chunk
constexpr int PARTS = 2048;               // most segments of a launch that splits rows
constexpr float kLn2 = 0.69314718055994531f;

// What a row, or a part of it, comes to: the largest logit, and with t = (l -
// max) log2(e) / T the sums of 2^t and t 2^t; the number of tokens before the
// given one.
struct Stat {
    float m, s, st;
    int before;
};

// A segment's result as it is joined: its best keys in falling order, 0 past
// them.
struct Part {
    Stat stat;
    uint64_t key[TOP];
};

template <int DT>
using Elem = typename std::conditional<DT == RHEO_F32, float,
             typename std::conditional<DT == RHEO_BF16, __bf16, _Float16>::type>::type;

// The 16-byte vector at element e of a row as floats; past V -inf, which adds
// nothing to a sum and orders behind every token by its id.
template <int DT>
__device__ __forceinline__ void load_vec(const char* row, int64_t e, int V, float* x) {
    constexpr int VEC = DT == RHEO_F32 ? 4 : 8;
    if (e + VEC <= V) {
        const uint4 w = *(const uint4*)(row + e * sizeof(Elem<DT>));
        if constexpr (DT == RHEO_F32) {
            x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y);
            x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
        } else {
            unpack8<Elem<DT>>(w, x);
        }
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k)
            x[k] = e + k < V ? (float)((const Elem<DT>*)row)[e + k] : -INFINITY;
    }
}

// Sums relative to a larger maximum: with d = (m - ref) kT <= 0, 2^t becomes
// 2^t 2^d and t 2^t becomes (t + d) 2^t 2^d.  Nothing counted yet (m = -inf):
// both sums are 0.
__device__ __forceinline__ void rebase(Stat& a, float m, float kT) {
    if (!(a.m < m)) return;
    const float d = a.m == -INFINITY ? 0.0f : (a.m - m) * kT;
    const float e = __builtin_amdgcn_exp2f(d);
    a.st = e > 0.0f ? __fmaf_rn(a.s, d, a.st) * e : 0.0f;
    a.s *= e;
    a.m = m;
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float kT) {
    const float m = fmaxf(a.m, b.m);
    rebase(a, m, kT);
    rebase(b, m, kT);
    return Stat{m, a.s + b.s, a.st + b.st, a.before + b.before};
}

__device__ __forceinline__ Stat wave_join(Stat v, float kT) {
    for (int o = 32; o; o >>= 1)
        v = join(v, Stat{__shfl_xor(v.m, o), __shfl_xor(v.s, o), __shfl_xor(v.st, o),
                         __shfl_xor(v.before, o)}, kT);
    return v;
}

// The k-th largest of a wave's 64 values (1 <= k <= 64): bit by bit from the
// top, set where k values are at least that large.
__device__ __forceinline__ uint32_t wave_kth(uint32_t v, int k) {
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t u = t | (1u << bit);
        if (__builtin_popcountll(__ballot(v >= u)) >= k) t = u;
    }
    return t;
}

__device__ __forceinline__ int block_count(int v, int* sh) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < NWL; ++w) sum += sh[w];
    return sum;
}

// An entry's outputs, by one wave; `best` in falling order, lane i's key i.
__device__ __forceinline__ void put_outputs(const LogprobArgs& a, int entry, const Stat& st,
                                            float lt, uint64_t best) {
    const int lane = threadIdx.x & 63;
    const float ln_z = logf(st.s);
    if (lane == 0) {
        a.logprob[entry] = (lt - st.m) / a.T - ln_z;
        if (a.entropy) a.entropy[entry] = ln_z - st.st / st.s * kLn2;
        if (a.rank) a.rank[entry] = st.before;
    }
    if (lane < a.top) {
        const int64_t o = (int64_t)entry * a.top + lane;
        a.top_token[o] = key_id(best);
        a.top_logprob[o] = (key_value(best) - st.m) / a.T - ln_z;
    }
}

}  // namespace

// One block takes a segment of one entry's row, chunk by chunk, every element
// once from memory into a register: running maximum and sums a thread, the
// tokens before the given one, and the best `top` keys so far in LDS (a key:
// logit descending, id ascending, as one 64-bit number).
//
// Candidates of a chunk are the elements above a bound: the worst of the best
// so far, or until there are `top` of them the largest of the waves' top-th
// largest thread maxima (at least `top` elements of the chunk are that large).
// They are ranked by counting.  Where more than LIST pass the bound (ties, rows
// that rise), the chunk's top-th largest key is found bit by bit over the
// registers: at most `top` are that large.
template <int DT>
__global__ __launch_bounds__(NTL) void k_row_stats(ScoreDev c, LogprobArgs a, int segs,
                                                   int seg_chunks) {
    __shared__ uint64_t s_list[LIST + TOP], s_best[TOP];
    __shared__ Stat s_stat[NWL];
    __shared__ int s_sum[NWL], s_cnt;
    __shared__ uint32_t s_bound[NWL];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int entry = blockIdx.x / segs, seg = blockIdx.x - entry * segs;
    const int b = entry / a.m;
    const int line = a.path ? a.path[entry] : entry - b * a.m;
    const int token = a.token[entry];
    if ((unsigned)line >= (unsigned)a.n || (unsigned)token >= (unsigned)c.V) return;
    constexpr int VEC = 16 / (int)sizeof(Elem<DT>), NV = EPT / VEC;
    const char* row = a.logits + ((int64_t)b * a.n + line) * c.stride * sizeof(Elem<DT>);
    const int V = c.V, top = a.top;
    const float kT = a.kT;
    const float lt = (float)((const Elem<DT>*)row)[token];
    const uint64_t own = logit_key(lt, (uint32_t)token);
    const int first = seg * seg_chunks * CHUNK;
    const int end = min(V, first + seg_chunks * CHUNK);

    Stat st = {-INFINITY, 0.0f, 0.0f, 0};
    int best = 0;                          // keys in s_best
    for (int c0 = first; c0 < end; c0 += CHUNK) {
        float x[EPT];
#pragma unroll
        for (int v = 0; v < NV; ++v) load_vec<DT>(row, c0 + (v * NTL + tid) * VEC, V, x + v * VEC);
        auto id_of = [&](int k) { return c0 + ((k / VEC) * NTL + tid) * VEC + k % VEC; };

        float m = x[0];
#pragma unroll
        for (int k = 1; k < EPT; ++k) m = fmaxf(m, x[k]);
        rebase(st, m, kT);
        const float ref = st.m == -INFINITY ? 0.0f : st.m;
#pragma unroll
        for (int k = 0; k < EPT; ++k) {
            // (2^-150 is 0 in fp32, so a masked token's t adds 0 and not NaN)
            const float t = fmaxf((x[k] - ref) * kT, -150.0f);
            const float e = __builtin_amdgcn_exp2f(t);
            st.s += e;
            st.st = __fmaf_rn(t, e, st.st);
            st.before += logit_key(x[k], (uint32_t)id_of(k)) > own && id_of(k) < V;
        }
        if (top == 0) continue;

        // the bound: codes at least `code` pass, and keys above `over`
        uint64_t over = 0;
        uint32_t code = 0;
        const int left = min(V - c0, CHUNK);             // elements of the chunk
        if (best == top) {
            over = s_best[top - 1];
            code = (uint32_t)(over >> 32);
        } else {
            const uint32_t kth = wave_kth(ord32(m), top);
            if (lane == 0) s_bound[wave] = kth;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NWL; ++w) code = max(code, s_bound[w]);
        }
        int mine = 0;
        const float low = unord32(code);                 // (no NaN: a logit's code, or 0)
        if (code == 0 || m >= low) {
#pragma unroll
            for (int k = 0; k < EPT; ++k)
                mine += id_of(k) < V && ord32(x[k]) >= code && logit_key(x[k], id_of(k)) > over;
        }
        int total = block_count(mine, s_sum);
        if (total > LIST) {
            // the top-th largest key above `over`; 64 bits of it, since keys differ
            const int k_th = min(top, left);
            uint64_t t = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t u = t | (1ull << bit);
                int cnt = 0;
#pragma unroll
                for (int k = 0; k < EPT; ++k)
                    cnt += id_of(k) < V && logit_key(x[k], id_of(k)) >= u;
                if (block_count(cnt, s_sum) >= k_th) t = u;
            }
            over = max(over, t - 1);
            code = (uint32_t)(t >> 32);
            mine = 0;
#pragma unroll
            for (int k = 0; k < EPT; ++k) mine += id_of(k) < V && logit_key(x[k], id_of(k)) > over;
            total = block_count(mine, s_sum);
        }
        if (total == 0) continue;
        // the candidates behind the best so far, in any order
        if (tid == 0) s_cnt = best;
        if (tid < best) s_list[tid] = s_best[tid];
        __syncthreads();
        if (mine) {
            int at = atomicAdd(&s_cnt, mine);
#pragma unroll
            for (int k = 0; k < EPT; ++k) {
                const uint64_t key = logit_key(x[k], id_of(k));
                if (id_of(k) < V && ord32(x[k]) >= code && key > over) s_list[at++] = key;
            }
        }
        __syncthreads();
        const int all = best + total;
        for (int i = tid; i < all; i += NTL) {
            const uint64_t key = s_list[i];
            int rank = 0;
            for (int j = 0; j < all; ++j) rank += s_list[j] > key;
            if (rank < top) s_best[rank] = key;
        }
        best = min(all, top);
        __syncthreads();
    }

    st = wave_join(st, kT);
    if (lane == 0) s_stat[wave] = st;
    __syncthreads();
    if (wave) return;
    st = lane < NWL ? s_stat[lane] : Stat{-INFINITY, 0.0f, 0.0f, 0};
    st = wave_join(st, kT);
    const uint64_t key = lane < best ? s_best[lane] : 0;
    if (segs == 1) {
        put_outputs(a, entry, st, lt, key);
    } else {
        Part* p = (Part*)c.work + blockIdx.x;
        if (lane == 0) p->stat = st;
        if (lane < top) p->key[lane] = key;
    }
}

// The segments of an entry joined, one wave each: lane i keeps the head of
// segment i's keys; `top` times the largest head is taken.
template <int DT>
__global__ __launch_bounds__(64) void k_row_join(ScoreDev c, LogprobArgs a, int segs) {
    const int lane = threadIdx.x, entry = blockIdx.x, b = entry / a.m;
    const int line = a.path ? a.path[entry] : entry - b * a.m;
    const int token = a.token[entry];
    if ((unsigned)line >= (unsigned)a.n || (unsigned)token >= (unsigned)c.V) return;
    const char* row = a.logits + ((int64_t)b * a.n + line) * c.stride * sizeof(Elem<DT>);
    const float lt = (float)((const Elem<DT>*)row)[token];
    const Part* p = (const Part*)c.work + (int64_t)entry * segs + lane;
    const bool has = lane < segs;
    const Stat st = wave_join(has ? p->stat : Stat{-INFINITY, 0.0f, 0.0f, 0}, a.kT);
    uint64_t head = has && a.top ? p->key[0] : 0, best = 0;
    int at = 0;
    for (int i = 0; i < a.top; ++i) {
        uint64_t m = head;
        for (int o = 32; o; o >>= 1) {
            const uint64_t u = __shfl_xor(m, o);
            m = u > m ? u : m;
        }
        if (lane == i) best = m;
        if (head == m && m) head = ++at < a.top ? p->key[at] : 0;
    }
    put_outputs(a, entry, st, lt, best);
}

namespace {

template <int DT>
hipError_t start(const ScoreDev& c, const LogprobArgs& a, hipStream_t s) {
    const int entries = a.B * a.m, chunks = (c.V + CHUNK - 1) / CHUNK;
    // Rows are split while their segments are few enough to need each other's
    // compute units, into at most 64 (a lane each in the join)
    int segs = PARTS / entries;
    segs = segs < 1 ? 1 : segs > 64 ? 64 : segs;
    if (segs > chunks) segs = chunks;
    const int seg_chunks = (chunks + segs - 1) / segs;
    segs = (chunks + seg_chunks - 1) / seg_chunks;
    k_row_stats<DT><<<entries * segs, NTL, 0, s>>>(c, a, segs, seg_chunks);
    if (segs > 1) k_row_join<DT><<<entries, 64, 0, s>>>(c, a, segs);
    return hipGetLastError();
}

}  // namespace

size_t score_workspace() { return PARTS * sizeof(Part); }

hipError_t launch_token_logprobs(const ScoreDev& c, const LogprobArgs& a, hipStream_t s) {
    if (c.dtype == RHEO_F32) return start<RHEO_F32>(c, a, s);
    if (c.dtype == RHEO_BF16) return start<RHEO_BF16>(c, a, s);
    return start<RHEO_F16>(c, a, s);
}

}  // namespace rheo
