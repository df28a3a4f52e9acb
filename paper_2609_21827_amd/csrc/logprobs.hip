// Log probabilities of given tokens, entropy, rank and the top of their rows
// (rheo_token_logprobs).
#include <type_traits>

#include "half_types.h"
#include "rheo.h"
#include "rheo_device.h"
#include "score_state.h"

namespace rheo {

namespace {

constexpr int NTL = 256;                  // threads of a block
constexpr int NWL = NTL / 64;
constexpr int EPT = 16;                   // elements a thread holds of a chunk
constexpr int CHUNK = NTL * EPT;          // 4096 elements
constexpr int TOP = 32;                   // most alternatives
constexpr int LIST = 1024;                // most candidates of a chunk
constexpr int PARTS = 2400;               // most segments of a launch that splits rows
constexpr float kLn2 = 0.69314718055994531f;

// What a row, or a part of it, comes to: the largest logit, and with t = (l -
// max) log2(e) / T the sums of 2^t and t 2^t; the number of tokens before the
// given one.  (t as one fused l kT - max kT would save an instruction of twelve,
// but the maximum's own t would not be 0, nor a sure token's log probability.)
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

// The 16-byte vector at element e of a row; past V -inf, which adds nothing to
// a sum and orders behind every token by its id.
template <int DT>
__device__ __forceinline__ uint4 load_vec(const char* row, int64_t e, int V) {
    constexpr int VEC = DT == RHEO_F32 ? 4 : 8;
    if (e + VEC <= V) return *(const uint4*)(row + e * sizeof(Elem<DT>));
    uint32_t w[4];
    if constexpr (DT == RHEO_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = e + k < V ? ((const uint32_t*)row)[e + k] : 0xFF800000u;
    } else {
        constexpr uint32_t low = DT == RHEO_BF16 ? 0xFF80u : 0xFC00u;
        const uint16_t* h = (const uint16_t*)row;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            w[k] = (e + 2 * k < V ? h[e + 2 * k] : low) |
                   (e + 2 * k + 1 < V ? h[e + 2 * k + 1] : low) << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT>
__device__ __forceinline__ void unpack_vec(const uint4& v, float* x) {
    if constexpr (DT == RHEO_F32) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    } else {
        unpack8<Elem<DT>>(v, x);
    }
}

// Sums relative to a larger maximum: with d = (m - m') kT <= 0, 2^t becomes 2^t 2^d
// and t 2^t becomes (t + d) 2^t 2^d.  Nothing counted yet (m = -inf): both are 0.
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

// A lower bound of the k-th largest of a wave's 64 values (1 <= k <= 64): its
// upper 16 bits, from the top, each set where k values are at least that large.
__device__ __forceinline__ uint32_t wave_kth(uint32_t v, int k) {
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
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
// once from memory into a register, the next chunk on its way: running maximum
// and sums a thread, the tokens before the given one, and a list in LDS of the
// keys that may be among the best `top` (a key: logit descending, id ascending,
// as one 64-bit number).
//
// The list takes every element above a bound and is ranked, by counting, after
// the first chunk, when it has twice `top` and 16, and at the end; the worst of the
// best is then the bound.  The
// first bound comes from the first chunk's thread maxima: with NWL waves, at least
// `top` of its elements are as large as the least of the waves' ceil(top /
// NWL)-th largest (of a chunk that leaves waves empty, as the largest of the
// waves' top-th largest).  A chunk that overflows the list (ties, rows that
// rise) is looked at again with its top-th largest key, found bit by bit over
// the registers: at most `top` are that large.
//
// 640 rows of 151936 bf16 (194 MB, 41 us at the copy's rate): 45 us without
// alternatives, 77 with 20, most of the difference in the first chunks' bounds and
// ranks.  Half of a wave's time is waits there, a fifth issue.
//
template <int DT>
__global__ __launch_bounds__(NTL) void k_row_stats(ScoreDev c, LogprobArgs a, int segs,
                                                   int seg_chunks) {
    __shared__ uint64_t s_list[LIST], s_best[TOP];
    __shared__ Stat s_stat[NWL];
    __shared__ int s_sum[NWL], s_cnt[3];
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
    const int first = seg * seg_chunks * CHUNK;
    const int end = min(V, first + seg_chunks * CHUNK);
    uint4 next[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) next[v] = load_vec<DT>(row, first + (v * NTL + tid) * VEC, V);
    const float lt = (float)((const Elem<DT>*)row)[token];
    if (tid < 3) s_cnt[tid] = 0;
    __syncthreads();

    Stat st = {-INFINITY, 0.0f, 0.0f, 0};
    int before = 0;                        // of the wave
    int listed = 0;                        // keys in s_list
    uint64_t over = 0;                     // keys above it go in,
    float low = 0.0f;                      // of logits at least that large
    // the best of the list, sorted, at its front; `over` and `low` after them
    auto rank = [&]() {
        for (int i = tid; i < listed; i += NTL) {
            const uint64_t key = s_list[i];
            int r = 0;
#pragma unroll 8
            for (int j = 0; j < listed; ++j) r += s_list[j] > key;
            if (r < top) s_best[r] = key;
        }
        listed = min(listed, top);
        __syncthreads();
        if (tid < listed) s_list[tid] = s_best[tid];
        if (listed == top) {
            over = s_best[top - 1];
            low = key_value(over);
        }
        __syncthreads();
    };
    // keys that a chunk adds are counted in one of three places, so that one barrier a
    // chunk is enough: a place is cleared between the barriers after its last use
    int turn = 0;
    for (int c0 = first; c0 < end; c0 += CHUNK) {
        float x[EPT];
#pragma unroll
        for (int v = 0; v < NV; ++v) unpack_vec<DT>(next[v], x + v * VEC);
        if (c0 + CHUNK < end)
#pragma unroll
            for (int v = 0; v < NV; ++v)
                next[v] = load_vec<DT>(row, c0 + CHUNK + (v * NTL + tid) * VEC, V);
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
        }
        // tokens before the given one, a wave's by ballot: a tie goes before it where
        // its id is lower
        if (c0 + CHUNK <= token) {
#pragma unroll
            for (int k = 0; k < EPT; ++k) before += __builtin_popcountll(__ballot(x[k] >= lt));
        } else if (c0 > token) {
#pragma unroll
            for (int k = 0; k < EPT; ++k) before += __builtin_popcountll(__ballot(x[k] > lt));
        } else {
#pragma unroll
            for (int k = 0; k < EPT; ++k)
                before += __builtin_popcountll(
                    __ballot((x[k] > lt) | ((x[k] == lt) & (id_of(k) < token))));
        }
        if (top == 0) continue;

        if (c0 == first) {
            const bool full = min(V - c0, CHUNK) >= NTL * VEC;
            const uint32_t kth = wave_kth(ord32(m), full ? (top + NWL - 1) / NWL : top);
            if (lane == 0) s_bound[wave] = kth;
            __syncthreads();
            uint32_t code = s_bound[0];
#pragma unroll
            for (int w = 1; w < NWL; ++w)
                code = full ? min(code, s_bound[w]) : max(code, s_bound[w]);
            // (no NaN: the code is at least that of -inf, cut to its upper half)
            low = code <= 0x007FFFFFu ? -INFINITY : unord32(code);
        }
        auto list = [&](int k) {
            const uint64_t key = logit_key(x[k], (uint32_t)id_of(k));
            if (key > over && id_of(k) < V) {
                const int at = listed + atomicAdd(&s_cnt[turn], 1);
                if (at < LIST) s_list[at] = key;
            }
        };
        // (few threads have one: a branch an element, skipped by whole waves)
        if (m >= low)
#pragma unroll
            for (int k = 0; k < EPT; ++k)
                if (x[k] >= low) list(k);
        if (tid == 0) s_cnt[turn == 2 ? 0 : turn + 1] = 0;
        __syncthreads();
        const int total = listed + s_cnt[turn];
        turn = turn == 2 ? 0 : turn + 1;
        if (total <= LIST) {
            listed = total;
            if (c0 == first || total > 2 * top + 16) rank();
            continue;
        }
        // this chunk's keys are not all in: without them, then its best alone
        rank();
        const int k_th = min(top, min(V - c0, CHUNK));
        uint64_t t = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t u = t | (1ull << bit);
            int cnt = 0;
#pragma unroll
            for (int k = 0; k < EPT; ++k)
                cnt += id_of(k) < V && logit_key(x[k], (uint32_t)id_of(k)) >= u;
            if (block_count(cnt, s_sum) >= k_th) t = u;
        }
        if (t - 1 > over) over = t - 1;
        low = fmaxf(low, key_value(t));
#pragma unroll
        for (int k = 0; k < EPT; ++k)
            if (x[k] >= low) list(k);
        __syncthreads();
        listed += s_cnt[turn];
        __syncthreads();
        if (tid == 0) s_cnt[turn] = 0;
        rank();                            // (with a barrier before the place's next use)
    }
    if (top) rank();
    const int best = listed;

    st = wave_join(st, kT);
    st.before = before;
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
    const int wide = segs > 1 ? 1 << (31 - __builtin_clz(segs - 1)) : 0;    // lanes that compare
    for (int i = 0; i < a.top; ++i) {
        uint64_t m = head;
        for (int o = wide; o; o >>= 1) {
            const uint64_t u = __shfl_xor(m, o);
            m = u > m ? u : m;
        }
        m = lane_u64(m, 0);
        if (lane == i) best = m;
        if (head == m && m) head = ++at < a.top ? p->key[at] : 0;
    }
    put_outputs(a, entry, st, lt, best);
}

namespace {

template <int DT>
hipError_t start(const ScoreDev& c, const LogprobArgs& a, hipStream_t s) {
    const int entries = a.B * a.m, chunks = (c.V + CHUNK - 1) / CHUNK;
    // Rows are split while all segments stay below PARTS, eight or nine blocks a
    // compute unit (of which five are resident: 96 registers, 106 for fp32), into at
    // most 64 (a lane each in the join).  Splitting costs a
    // first chunk's selection a segment and the join: 640 rows of 151936, 20
    // alternatives, 79 us in one to three parts each and 85 in six; but 1152 entries of
    // which half are left out 95 us whole and 80 in halves, since whole they leave
    // most of the chip's waves unused.
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
