// Attention over 4-bit pages and a 16-bit tail (rheo_packed_attention).
//
// o_i = sum_j p_ij v_j with p = softmax_j(scale q_i.k_j), in one pass over the entries
// with a running maximum and sum, for the g = heads / kv_heads query heads of a key head
// and a sequence's rows together, as rheo_tree_attention does it.  What differs is where
// the operands come from: a wave reads codes, 17 bytes for 32 elements, and makes the matrix
// cores' operands of them in its registers (the values are exact in 16 bits), with nothing
// passing through LDS and no wave waiting for another before an item's end.
//
// Products are transposed, S^T = K Q^T and O^T = V^T P^T, as 16x16x32 tiles; a wave
// takes 32 entries at a time, two blocks u of 16, and 16 MQ rows.  Lane 16 g + n holds
//   of K: entry n of each block, elements 8 NB g + 8 s + (0..7) at step s (Q alike), so
//         that its 4 NB bytes of codes lie together;
//   of V: elements 2 NB n + (0..2 NB - 1) of the entries 4 g + (0..3) of both blocks;
//         column n of tile t is element 2 NB n + t, and a tile's operand is the entries'
//         words of two elements taken apart and joined by pairs of entries;
//   of S^T: row n, entries 4 g + (0..3) of each block: with the second product's inner
//         index 8 g + j <-> entry (j < 4 ? 4 g + j of block 0 : 4 g + j - 4 of block 1) its
//         probabilities are the right operand as they stand;
//   of O^T: row n, elements 8 NB g + (0..8 NB - 1), next to each other.
//
// Work is one line of tiles over all (sequence, key head, block of rows), cut evenly over
// the workgroups; items that are cut leave partial results, which k_packed_join adds up.
// With a window an item's tiles are those of the first entries that stay visible and those
// from the first row's window on.
#include <type_traits>

#include "packed_format.h"
#include "softmax_ref.h"

namespace rheo {

namespace {

// A launch's shape: NB blocks of 32 head elements; a wave has MQ tiles of 16 rows, WR waves
// of a workgroup's four have different rows, the others share the entries; RES workgroups
// to a compute unit.
template <int NB_, int MQ_, int WR_, int RES_>
struct PShape {
    static constexpr int NB = NB_, MQ = MQ_, WR = WR_, RES = RES_, WT = 4 / WR;
    static constexpr int DP = 32 * NB, OT = 2 * NB;
    static constexpr int ROWS = 16 * MQ * WR, KT = 32 * WT;    // of an item, of a tile
    // a partial result: O^T as the lanes hold it, maximum and sum of each row, a flag
    static constexpr int PART = ROWS * DP + 2 * ROWS + 64;
    static constexpr int LDS = WT > 1 ? (4 - WR) * MQ * 8 * NB * 64 * 4 : 0;
    static constexpr bool DEAL = WR == 4;                      // see deal_items
};
constexpr int NT = 256, NW = 4;

struct AttnArgs {
    CacheDev c;
    PackedDev p;
    rheo_packed_attention_args a;
    int g;                         // query heads of a key head
    int* desc;                     // [groups][8]: what k_packed_join adds up
    int groups;                    // most stretches (workgroups)
    int whole;                     // whole items may be given out (see deal_items)
};

// A sequence's part of the line.
struct Seq {
    int len, rows, tail, nrb;      // entries in pages, rows there, tail's, row blocks
};

template <typename S>
__device__ __forceinline__ Seq seq_of(const AttnArgs& p, int b) {
    Seq s;
    const int64_t room = (int64_t)p.c.width << p.c.page_shift;
    s.len = p.a.lens[b];
    int count = p.a.count ? p.a.count[b] : p.a.n;
    if (p.a.status && p.a.status[b]) count = 0;      // not served: no row of it is there
    s.rows = min(max(count, 0), p.a.n);
    if (count != s.rows) atomicOr(p.c.err, CE_PLAN);
    s.tail = max(p.a.tail - (p.a.n - s.rows), 0);
    if (s.len < 0 || s.len > room) {
        if (s.rows) atomicOr(p.c.err, CE_TABLE);
        s.len = (int)min((int64_t)max(s.len, 0), room);
    }
    s.nrb = (s.rows * p.g + S::ROWS - 1) / S::ROWS;
    return s;
}

// What a row block attends, as a whole: entries lo to hi, and those before `sinks`; and
// its tiles.  Tiles of the pages come first, `pages` of them, then the tail's.  Of these
// the block takes the first `head` and those from `from` on, `count` in all (one at
// least).
struct Span {
    int lo, hi, pages, head, from, count;
    __device__ __forceinline__ int tile(int k) const { return k < head ? k : k - head + from; }
};

template <typename S>
__device__ __forceinline__ Span span_of(const AttnArgs& p, const Seq& s, int rb) {
    const rheo_packed_attention_args& a = p.a;
    Span x;
    x.hi = s.len + s.tail - 1;
    x.lo = 0;
    int first = s.len;                               // position of the first row
    if (!a.mask) {
        first = s.len + a.tail - a.n + rb * S::ROWS / p.g;
        const int last = min(((rb + 1) * S::ROWS - 1) / p.g, s.rows - 1);
        x.hi = min(x.hi, s.len + a.tail - a.n + last);
    }
    if (a.window) x.lo = max(first - a.window + 1, 0);
    x.pages = (s.len + S::KT - 1) / S::KT;
    const auto tile_of = [&](int e) {
        return e < s.len ? e / S::KT : x.pages + (e - s.len) / S::KT;
    };
    const int end = tile_of(max(x.hi, 0));
    x.from = x.hi < x.lo ? end : tile_of(x.lo);
    x.head = a.window && a.sinks && x.hi >= 0 ? min(tile_of(min(a.sinks - 1, x.hi)) + 1, x.from) : 0;
    x.count = x.head + end - x.from + 1;
    return x;
}

// Tiles of all row blocks of a sequence, for one key head.
template <typename S>
__device__ __forceinline__ int64_t tiles_of_head(const AttnArgs& p, const Seq& s) {
    if (p.a.mask) return s.nrb ? (int64_t)s.nrb * span_of<S>(p, s, 0).count : 0;
    int64_t t = 0;
    for (int rb = 0; rb < s.nrb; ++rb) t += span_of<S>(p, s, rb).count;
    return t;
}

// What is the same in all lanes, said so: it then takes scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
__device__ __forceinline__ Seq uniform(const Seq& s) {
    return Seq{uniform(s.len), uniform(s.rows), uniform(s.tail), uniform(s.nrb)};
}
__device__ __forceinline__ Span uniform(const Span& s) {
    return Span{uniform(s.lo),   uniform(s.hi),   uniform(s.pages),
                uniform(s.head), uniform(s.from), uniform(s.count)};
}

// Stretch w of the line: tiles [t0, t1) of it, the sequence that t0 is in and the tiles
// before that sequence.  All threads of the block call it.
struct Stretch {
    int64_t total, t0, t1, before;
    int groups, seq;
};

__device__ __forceinline__ int64_t stretch_start(int64_t total, int groups, int w) {
    return total * w / groups;
}

template <typename S>
__device__ Stretch find_stretch(const AttnArgs& p, int w) {
    __shared__ int64_t s_wave[NW], s_before;
    __shared__ int s_seq;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = p.c.B;
    const int per = (B + NT - 1) / NT, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += p.c.K * tiles_of_head<S>(p, seq_of<S>(p, b));
    int64_t incl = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int64_t excl = incl - mine, total = 0;
    for (int v = 0; v < NW; ++v) {
        if (v < wave) excl += s_wave[v];
        total += s_wave[v];
    }
    total = uniform64(total);
    Stretch r;
    r.total = total;
    r.groups = (int)(total < p.groups ? total : p.groups);
    r.seq = 0;
    r.before = 0;
    if (w >= r.groups) {
        r.t0 = r.t1 = 0;
        return r;
    }
    r.t0 = stretch_start(total, r.groups, w);
    r.t1 = stretch_start(total, r.groups, w + 1);
    if (r.t0 >= excl && r.t0 < excl + mine) {
        int64_t t = excl;
        for (int b = b0; b < b1; ++b) {
            const int64_t k = p.c.K * tiles_of_head<S>(p, seq_of<S>(p, b));
            if (r.t0 < t + k) {
                s_seq = b;
                s_before = t;
                break;
            }
            t += k;
        }
    }
    __syncthreads();
    r.seq = uniform(s_seq);
    r.before = uniform64(s_before);
    return r;
}

// Whole items dealt out instead of stretches, where that is nearly as even: the sequences
// sorted by length, their items given to the workgroups in order, there and back (the
// longest with the shortest).  A cut of 256 rows costs their partial results' way out and
// back.  All threads call it; at most kDealt sequences, an item a key head each.
constexpr int kDealt = 256;

__device__ __forceinline__ int dealt_item(int round, int w, int groups) {
    return round * groups + (round & 1 ? groups - 1 - w : w);
}

template <typename S>
__device__ bool deal_items(const AttnArgs& p, int64_t total, int* s_order) {
    __shared__ int s_tiles[kDealt], s_most[NW];
    const int tid = threadIdx.x, B = p.c.B, K = p.c.K, items = B * K;
    __syncthreads();
    for (int b = tid; b < B; b += NT) {
        const Seq s = seq_of<S>(p, b);
        s_tiles[b] = s.nrb ? span_of<S>(p, s, 0).count : 0;
    }
    __syncthreads();
    for (int b = tid; b < B; b += NT) {
        const int mine = s_tiles[b];
        int rank = 0;
        for (int o = 0; o < B; ++o) rank += s_tiles[o] > mine || (s_tiles[o] == mine && o < b);
        s_order[rank] = b;
    }
    __syncthreads();
    int most = 0;
    for (int w = tid; w < p.groups; w += NT) {
        int sum = 0;
        for (int r = 0; r * p.groups < items; ++r) {
            const int i = dealt_item(r, w, p.groups);
            if (i < items) sum += s_tiles[s_order[i / K]];
        }
        most = max(most, sum);
    }
    for (int o = 32; o; o >>= 1) most = max(most, __shfl_xor(most, o));
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
    for (int w = 0; w < NW; ++w) most = max(most, s_most[w]);
    const int64_t mean = total / p.groups;
    return most <= mean + mean / 16 + 8;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
    typedef typename Pack<T>::v8 v8;
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
}

// A row's maximum or sum over the four lanes that hold it.
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// Both elements of a word 0 where they are infinite or NaN.
template <typename T>
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    constexpr uint32_t E = Pack<T>::kExp;
    return ((w & E) == E ? 0 : w & 0xFFFFu) | ((w & E << 16) == E << 16 ? 0 : w & 0xFFFF0000u);
}

// A wave's codes of 32 entries, as loaded.
template <int NB>
struct Raw {
    static constexpr bool P2 = (NB & (NB - 1)) == 0;
    static constexpr int VW = NB <= 4 ? 1 : 2;       // words of an entry's V a lane
    static constexpr int SB = P2 ? 1 : 2;            // blocks that these lie in
    static constexpr int KS = P2 ? (NB + 3) / 4 : NB;      // exponents of K a lane
    uint32_t k[2][NB], ks[2][KS], v[8][VW], vs[2][SB];
};

// The blocks of a lane's elements of K at step s, and of its pair p of V.
template <int NB>
__device__ __forceinline__ int k_block(int g, int s) { return (NB * g + s) >> 2; }
template <int NB>
__device__ __forceinline__ int v_block(int n, int p) { return (NB * n + p) >> 4; }

template <typename S>
struct Rows {
    u32x4 q[S::MQ][S::NB];
    f32x4 o[S::MQ][S::OT];
    float m[S::MQ], l[S::MQ];      // the exponents' reference, a score; the lane's sum
    int lo[S::MQ], hi[S::MQ];      // entries that the lane's row attends (and sinks)
};

// One step: scores of 32 entries from K's operands (`key(u, s)`), softmax, O += P V with V's
// words (`val(j, p)`: pair p of entry j % 4 of block j / 4).  `seen(mq, u, r)`: whether the
// lane's row attends entry 4 g + r of block u; asked if `masked`.
template <typename T, typename S, typename Key, typename Val, typename Seen>
__device__ __forceinline__ void step(Rows<S>& x, float to2, float slack, bool masked, Key key, Val val,
                                     Seen seen) {
    f32x4 sc[S::MQ][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int mq = 0; mq < S::MQ; ++mq) sc[mq][u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < S::NB; ++s) {
            const u32x4 k = key(u, s);
#pragma unroll
            for (int mq = 0; mq < S::MQ; ++mq) sc[mq][u] = mfma<T>(k, x.q[mq][s], sc[mq][u]);
        }
    }
    if (masked) {
#pragma unroll
        for (int mq = 0; mq < S::MQ; ++mq)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[mq][u][r] = seen(mq, u, r) ? sc[mq][u][r] : -INFINITY;
    }
    // The exponents' reference follows a row's own maximum by steps (kSlack), so that O is
    // rescaled once or twice an item.
    float mx[S::MQ];
    bool up = false;
#pragma unroll
    for (int mq = 0; mq < S::MQ; ++mq) {
        mx[mq] = fmaxf(fmaxf(fmaxf(sc[mq][0][0], sc[mq][0][1]), fmaxf(sc[mq][0][2], sc[mq][0][3])),
                       fmaxf(fmaxf(sc[mq][1][0], sc[mq][1][1]), fmaxf(sc[mq][1][2], sc[mq][1][3])));
        up |= mx[mq] > x.m[mq] + slack;
    }
    if (__any(up)) {
#pragma unroll
        for (int mq = 0; mq < S::MQ; ++mq) {
            const float m = row_max(mx[mq]);
            const bool mine = m > x.m[mq] + slack;
            const float f = mine ? __builtin_amdgcn_exp2f((x.m[mq] * to2 - kRise<T>) - ref_of<T>(m, to2))
                                 : 1.0f;
            x.l[mq] *= f;
#pragma unroll
            for (int t = 0; t < S::OT; ++t) x.o[mq][t] *= f;
            x.m[mq] = mine ? m : x.m[mq];
        }
    }
    // The sum takes the probabilities unrounded, the second product in 16 bits, what the
    // matrix cores take.
    u32x4 pt[S::MQ];
#pragma unroll
    for (int mq = 0; mq < S::MQ; ++mq) {
        const float ref = ref_of<T>(x.m[mq], to2);
        float e[8], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[mq][i >> 2][i & 3], to2, -ref));
            sum += e[i];
        }
        x.l[mq] += sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) pt[mq][i] = pack2<T>(e[2 * i], e[2 * i + 1]);
    }
#pragma unroll
    for (int p = 0; p < S::NB; ++p) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = val(j, p);
        u32x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
            hi[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
        }
#pragma unroll
        for (int mq = 0; mq < S::MQ; ++mq) {
            x.o[mq][2 * p] = mfma<T>(lo, pt[mq], x.o[mq][2 * p]);
            x.o[mq][2 * p + 1] = mfma<T>(hi, pt[mq], x.o[mq][2 * p + 1]);
        }
    }
}

// The infinite and NaN values of the tail, which the products left out, added to the
// elements d0 .. d0 + n - 1 of a finished row that attends them.  Their probabilities are
// not 0, so the values themselves decide.  Rare and slow.
template <typename T>
__device__ __forceinline__ void add_unfinite(const AttnArgs& p, int b, int hk, const Seq& sq, int qi,
                                             T* out, int d0, int n) {
    const rheo_packed_attention_args& a = p.a;
    const int64_t qrow = (int64_t)b * a.n + qi;
    const int reach = sq.len + a.tail - a.n + qi;
#pragma unroll 1
    for (int j = 0; j < sq.tail; ++j) {
        const int e = sq.len + j;
        const bool seen = a.mask ? a.mask[qrow * a.tail + j] != 0
                                 : e <= reach && (!a.window || e > reach - a.window || e < a.sinks);
        if (!seen) continue;
        const T* v = (const T*)a.v_tail + ((int64_t)b * a.tail + j) * a.tail_stride + hk * p.c.D;
#pragma unroll 1
        for (int d = d0; d < min(d0 + n, p.c.D); ++d) {
            const float x = (float)v[d];
            if (!(fabsf(x) < INFINITY)) out[d] = (T)((float)out[d] + x);
        }
    }
}

// 8 NB elements of a row, 8 NB g on, from the order of the lanes' O^T: 2 NB r + t at [t][r].
template <typename T, int NB, typename Get>
__device__ __forceinline__ void store_row(T* out, int g, int D, float inv, Get get) {
#pragma unroll
    for (int c = 0; c < NB; ++c) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = get((8 * c + i) % (2 * NB), (8 * c + i) / (2 * NB)) * inv;
        const int d = 8 * NB * g + 8 * c;
        if (d < D) *(uint4*)(out + d) = pack8<T>(f);
    }
}

}  // namespace

template <typename T, typename S>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(S::RES, S::RES))) void
k_packed_attention(AttnArgs p) {
    constexpr int NB = S::NB, MQ = S::MQ;
    extern __shared__ __align__(16) char s_lds[];
    __shared__ float s_ml[S::WT > 1 ? NW * MQ * 16 * 2 : 2];
    __shared__ int s_order[S::DEAL ? kDealt : 1];    // sequences, the longest first
    const int tid = threadIdx.x, lane = tid & 63, n16 = lane & 15, g4 = lane >> 4;
    const int wave = uniform(tid >> 6), wr = wave % S::WR, wt = wave / S::WR;
    const CacheDev& c = p.c;
    const rheo_packed_attention_args& a = p.a;
    const int w = blockIdx.x, D = c.D;
    const float to2 = a.scale * kLog2e;              // scores to exponents of 2
    const float slack = kSlack<T> / to2;
    const int in_page = (1 << c.page_shift) - 1;
    const int scales = 16 * NB << c.page_shift;      // where a head's page has its exponents
    // the lane's offsets from an entry block's first codes and exponents
    const int k_at = n16 * 16 * NB + 4 * NB * g4, v_at = 4 * g4 * 16 * NB + NB * n16;

    Stretch st = find_stretch<S>(p, w);
    bool dealt = false;
    if constexpr (S::DEAL)
        if (p.whole && st.groups == p.groups)
            dealt = uniform(deal_items<S>(p, st.total, s_order)) != 0;
    if (tid == 0) p.desc[8 * w] = 0;
    if (!dealt && st.t0 >= st.t1) return;
    // the item at hand: sequence, key head, row block, its tile to begin with; the
    // tiles left of the stretch, or the round of the deal
    int b = 0, hk = 0, rb = 0, tile = 0, round = 0;
    int64_t left = 0;
    Seq sq;
    auto next_dealt = [&]() {
        for (; S::DEAL && round * p.groups < c.B * c.K; ++round) {
            const int i = dealt_item(round, w, p.groups);
            if (i >= c.B * c.K) continue;
            b = uniform(s_order[i / c.K]);
            hk = i % c.K;
            sq = uniform(seq_of<S>(p, b));
            if (sq.nrb) {
                left = span_of<S>(p, sq, 0).count;
                ++round;
                return true;
            }
        }
        return false;
    };
    if (dealt) {
        if (!next_dealt()) return;
    } else {
        b = st.seq;
        sq = uniform(seq_of<S>(p, b));
        int64_t rel = st.t0 - st.before;
        const int64_t per_head = tiles_of_head<S>(p, sq);
        hk = uniform((int)(rel / per_head));
        rel -= hk * per_head;
        for (int n; rel >= (n = span_of<S>(p, sq, rb).count); ++rb) rel -= n;
        rb = uniform(rb);
        tile = uniform((int)rel);
        left = st.t1 - st.t0;
        // the join of the first item, by the first cut inside it
        const int64_t begins = st.t0 - tile, ends = begins + span_of<S>(p, sq, rb).count;
        if (tid == 0 && tile > 0 && stretch_start(st.total, st.groups, w - 1) <= begins) {
            int* d = p.desc + 8 * w;
            int n = 2;
            while (stretch_start(st.total, st.groups, w + n - 1) < ends) ++n;
            d[0] = n;                                // partial results
            d[1] = 2 * (w - 1) + (stretch_start(st.total, st.groups, w - 1) < begins ? 1 : 0);
            d[2] = b;
            d[3] = hk;
            d[4] = rb;
        }
    }

    for (bool first = true; left > 0; first = false) {
        const Span span = uniform(span_of<S>(p, sq, rb));
        const int end_tile = (int)min((int64_t)span.count, tile + left);
        // (of the pages; then the tail's)
        const int end_pages = min(end_tile, span.from < span.pages ? span.pages - span.from + span.head
                                                                   : min(span.head, span.pages));
        const int32_t* row_table = a.table + (int64_t)b * c.width;
        const uint8_t* const k_head = p.p.k + hk * p.p.head;
        const uint8_t* const v_head = p.p.v + hk * p.p.head;

        Rows<S> x;
        int lo_most = 0, hi_least = 0x7FFFFFFF;
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq) {
            const int r = rb * S::ROWS + (wr * MQ + mq) * 16 + n16;
            const bool live = r < sq.rows * p.g;
            const int qi = live ? r / p.g : 0, qh = hk * p.g + (live ? r - qi * p.g : 0);
            const int64_t qrow = (int64_t)b * a.n + qi;
            const T* q = (const T*)a.q + qrow * a.q_stride + (int64_t)qh * D;
#pragma unroll
            for (int s = 0; s < NB; ++s) {
                const int d = 8 * NB * g4 + 8 * s;
                x.q[mq][s] = u32x4{0, 0, 0, 0};
                if (live && d < D) x.q[mq][s] = *(const u32x4*)(q + d);
            }
            int at = sq.len + a.tail - a.n + qi;     // the row's position
            if (a.mask) at = a.window && a.positions ? max(a.positions[qrow], sq.len) : sq.len;
            x.hi[mq] = a.mask ? sq.len - 1 : at;
            x.lo[mq] = a.window ? at - a.window + 1 : 0;
            if (live) {
                lo_most = max(lo_most, x.lo[mq]);
                hi_least = min(hi_least, x.hi[mq]);
            }
        }
        for (int o = 1; o < 16; o <<= 1) {
            lo_most = max(lo_most, __shfl_xor(lo_most, o));
            hi_least = min(hi_least, __shfl_xor(hi_least, o));
        }
        lo_most = uniform(lo_most);
        hi_least = uniform(min(hi_least, sq.len - 1));
        const int sinks = a.window ? a.sinks : 0;

        // The wave's 32 entries of a tile of the pages begin at e0; of two blocks of 16
        // those are read that some row attends
        const auto begins = [&](int k) { return span.tile(k) * S::KT + 32 * wt; };
        const auto wanted = [&](int e) {
            return e < sq.len && e <= span.hi && (e + 15 >= span.lo || e < sinks);
        };
        struct Two { int a, b; };
        const auto fetch_pages = [&](int k) {
            Two t{-1, -1};
            if (k < end_pages) {
                const int e0 = begins(k);
                const bool n0 = wanted(e0), n1 = wanted(e0 + 16);
                if (n0 | n1) {
                    t.a = row_table[(n0 ? e0 : e0 + 16) >> c.page_shift];
                    t.b = row_table[(n1 ? e0 + 16 : e0) >> c.page_shift];
                }
            }
            return t;
        };
        const auto page_of = [&](int page) {
            page = uniform(page);
            if ((unsigned)page >= (unsigned)c.pages) {
                if (lane == 0) atomicOr(c.err, CE_PAGE);
                page = 0;
            }
            return page * p.p.page_stride;
        };
        Raw<NB> raw;
        const auto fetch = [&](int k, const Two& t) {
            const int e0 = begins(k);
            if (!(wanted(e0) | wanted(e0 + 16))) return;
            const int64_t page[2] = {page_of(t.a), page_of(t.b)};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i0 = (e0 + 16 * u) & in_page;
                const uint8_t* kc = k_head + page[u] + (int64_t)i0 * (16 * NB);
                const uint8_t* vc = v_head + page[u] + (int64_t)i0 * (16 * NB);
                const uint8_t* kx = k_head + page[u] + scales + i0;
                const uint8_t* vx = v_head + page[u] + scales + i0;
                __builtin_memcpy(raw.k[u], __builtin_assume_aligned(kc + k_at, 4), 4 * NB);
#pragma unroll
                for (int s = 0; s < Raw<NB>::KS; ++s)
                    raw.ks[u][s] = kx[(k_block<NB>(g4, Raw<NB>::P2 ? 4 * s : s) << c.page_shift) + n16];
                // (a lane's NB bytes at any place: the whole words' last may be the next
                // entry's, or of the exponents behind the last)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    __builtin_memcpy(raw.v[4 * u + j], vc + v_at + j * 16 * NB, 4 * Raw<NB>::VW);
#pragma unroll
                for (int s = 0; s < Raw<NB>::SB; ++s)
                    raw.vs[u][s] = *(const uint32_t*)(
                        vx + (v_block<NB>(n16, s * (NB - 1)) << c.page_shift) + 4 * g4);
            }
        };

        bool careful = false;
        for (;;) {                                   // again where the tail is not finite
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq) {
#pragma unroll
                for (int t = 0; t < S::OT; ++t) x.o[mq][t] = f32x4{0, 0, 0, 0};
                x.m[mq] = -INFINITY;
                x.l[mq] = 0.0f;
            }
            Two pages = fetch_pages(tile);
            if (tile < end_pages) fetch(tile, pages);
            pages = fetch_pages(tile + 1);
#pragma unroll 1
            for (int k = tile; k < end_pages; ++k) {
                const int e0 = begins(k);
                const bool now = wanted(e0) | wanted(e0 + 16);
                const bool masked = !(e0 + 31 <= hi_least && (e0 >= lo_most || e0 + 31 < sinks));
                if (!now) {
                    if (k + 1 < end_pages) fetch(k + 1, pages);
                    pages = fetch_pages(k + 2);
                    continue;
                }
                if (masked) {
                    // what nobody attends is any bytes: its exponents 0, so that its
                    // values are finite
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        uint32_t keep = 0;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int e = e0 + 16 * u + 4 * g4 + r;
                            const bool in = e < sq.len && e <= span.hi && (e >= span.lo || e < sinks);
                            keep |= in ? 0xFFu << (8 * r) : 0;
                        }
#pragma unroll
                        for (int s = 0; s < Raw<NB>::SB; ++s) raw.vs[u][s] &= keep;
                    }
                }
                const Raw<NB> now_raw = raw;
                if (k + 1 < end_pages) fetch(k + 1, pages);
                pages = fetch_pages(k + 2);
                step<T, S>(
                    x, to2, slack, masked,
                    [&](int u, int s) {
                        const uint32_t cw = now_raw.k[u][s];
                        const float f = scale_of(now_raw.ks[u][Raw<NB>::P2 ? s / 4 : s]);
                        return u32x4{pair_of<T, 0>(cw, f), pair_of<T, 1>(cw, f), pair_of<T, 2>(cw, f),
                                     pair_of<T, 3>(cw, f)};
                    },
                    [&](int j, int q) {
                        uint32_t sw = now_raw.vs[j >> 2][0];
                        if constexpr (!Raw<NB>::P2)
                            if (v_block<NB>(n16, q) != v_block<NB>(n16, 0))
                                sw = now_raw.vs[j >> 2][Raw<NB>::SB - 1];
                        const float f = j % 4 == 0   ? scale_at<0>(sw)
                                        : j % 4 == 1 ? scale_at<1>(sw)
                                        : j % 4 == 2 ? scale_at<2>(sw)
                                                     : scale_at<3>(sw);
                        const uint32_t cw = now_raw.v[j][q / 4];
                        return q % 4 == 0   ? pair_of<T, 0>(cw, f)
                               : q % 4 == 1 ? pair_of<T, 1>(cw, f)
                               : q % 4 == 2 ? pair_of<T, 2>(cw, f)
                                            : pair_of<T, 3>(cw, f);
                    },
                    [&](int mq, int u, int r) {
                        const int e = e0 + 16 * u + 4 * g4 + r;
                        return e < sq.len && e <= x.hi[mq] && (e >= x.lo[mq] || e < sinks);
                    });
            }
#pragma unroll 1
            for (int k = max(tile, end_pages); k < end_tile; ++k) {
                const int j0 = (span.tile(k) - span.pages) * S::KT + 32 * wt;
                if (j0 >= sq.tail) continue;
                const int64_t row0 = (int64_t)b * a.tail;
                const T* const kt = (const T*)a.k_tail + hk * D;
                const T* const vt = (const T*)a.v_tail + hk * D;
                u32x4 ko[2][NB];
                uint32_t vo[8][NB];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int j = min(j0 + 16 * u + n16, sq.tail - 1);
                    const T* row = kt + (row0 + j) * a.tail_stride;
#pragma unroll
                    for (int s = 0; s < NB; ++s) {
                        const int d = 8 * NB * g4 + 8 * s;
                        ko[u][s] = *(const u32x4*)(row + min(d, D - 8));
                        if (d >= D) ko[u][s] = u32x4{0, 0, 0, 0};
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int at = j0 + 16 * (j >> 2) + 4 * g4 + (j & 3);
                    const T* row = vt + (row0 + min(at, sq.tail - 1)) * a.tail_stride;
#pragma unroll
                    for (int q = 0; q < NB; ++q) {
                        // (pairs past the head are columns that no one stores)
                        vo[j][q] = *(const uint32_t*)(row + min(2 * NB * n16 + 2 * q, D - 2));
                        if (at >= sq.tail) vo[j][q] = 0;
                        if (careful) vo[j][q] = finite_pair<T>(vo[j][q]);
                    }
                }
                const uint8_t* mrow[MQ];
#pragma unroll
                for (int mq = 0; mq < MQ; ++mq) {
                    const int r = rb * S::ROWS + (wr * MQ + mq) * 16 + n16;
                    mrow[mq] = a.mask + ((int64_t)b * a.n + min(r / p.g, sq.rows - 1)) * a.tail;
                }
                step<T, S>(
                    x, to2, slack, true, [&](int u, int s) { return ko[u][s]; },
                    [&](int j, int q) { return vo[j][q]; },
                    [&](int mq, int u, int r) {
                        const int j = j0 + 16 * u + 4 * g4 + r, e = sq.len + j;
                        if (a.mask) return j < sq.tail && mrow[mq][min(j, sq.tail - 1)] != 0;
                        return j < sq.tail && e <= x.hi[mq] && (e >= x.lo[mq] || e < sinks);
                    });
            }
            if (careful) break;
            // A value that is infinite or NaN has left none of its sums finite, a row's that
            // does not attend it (0 times it is NaN) neither: then once more without them.
            float z = 0.0f;
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq)
#pragma unroll
                for (int t = 0; t < S::OT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z = __fmaf_rn(x.o[mq][t][r], 0.0f, z);
            careful = __syncthreads_or(!(z == 0.0f) && end_tile > end_pages) != 0;
            if (!careful) break;
        }

        // the waves of a row block put together
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq) x.l[mq] = row_sum(x.l[mq]);
        if constexpr (S::WT > 1) {
            __syncthreads();                         // (the last item's have been read)
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq)
                if (g4 == 0) {
                    s_ml[((wave * MQ + mq) * 16 + n16) * 2] = x.m[mq];
                    s_ml[((wave * MQ + mq) * 16 + n16) * 2 + 1] = x.l[mq];
                }
            __syncthreads();
            float* out = (float*)s_lds;
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq) {
                float m = -INFINITY, l = 0.0f;
#pragma unroll
                for (int k = 0; k < S::WT; ++k)
                    m = fmaxf(m, s_ml[(((k * S::WR + wr) * MQ + mq) * 16 + n16) * 2]);
                const float ref = ref_of<T>(m, to2);
#pragma unroll
                for (int k = 0; k < S::WT; ++k) {
                    const float* ml = s_ml + (((k * S::WR + wr) * MQ + mq) * 16 + n16) * 2;
                    l += ml[1] * __builtin_amdgcn_exp2f((ml[0] * to2 - kRise<T>) - ref);
                }
                const float f = __builtin_amdgcn_exp2f((x.m[mq] * to2 - kRise<T>) - ref);
#pragma unroll
                for (int t = 0; t < S::OT; ++t) {
                    x.o[mq][t] *= f;
                    if (wt > 0)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            out[((((wave - S::WR) * MQ + mq) * S::OT + t) * 4 + r) * 64 + lane] =
                                x.o[mq][t][r];
                }
                x.m[mq] = m;
                x.l[mq] = l;
            }
            __syncthreads();
            if (wt == 0)
#pragma unroll 1
                for (int k = 1; k < S::WT; ++k)
#pragma unroll
                    for (int mq = 0; mq < MQ; ++mq)
#pragma unroll
                        for (int t = 0; t < S::OT; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                x.o[mq][t][r] +=
                                    out[(((((k - 1) * S::WR + wr) * MQ + mq) * S::OT + t) * 4 + r) * 64 +
                                        lane];
        }
        if (wt == 0) {
            const bool whole = tile == 0 && end_tile == span.count;
            float* part = c.part + (int64_t)(2 * w + (first ? 0 : 1)) * S::PART;
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq) {
                const int rt = wr * MQ + mq, r = rb * S::ROWS + rt * 16 + n16;
                if (whole) {
                    if (r < sq.rows * p.g) {
                        const int qi = r / p.g, qh = hk * p.g + r - qi * p.g;
                        const int64_t qrow = (int64_t)b * a.n + qi;
                        const float inv = x.l[mq] == 0.0f ? 0.0f : 1.0f / x.l[mq];
                        T* o = (T*)a.out + qrow * a.out_stride + (int64_t)qh * D;
                        store_row<T, NB>(o, g4, D, inv, [&](int t, int i) { return x.o[mq][t][i]; });
                        if (a.lse && g4 == 0) a.lse[qrow * c.H + qh] = lse_of<T>(x.m[mq], x.l[mq], a.scale);
                        if (careful) add_unfinite<T>(p, b, hk, sq, qi, o, 8 * NB * g4, 8 * NB);
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < S::OT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            part[((rt * S::OT + t) * 4 + i) * 64 + lane] = x.o[mq][t][i];
                    if (g4 == 0) {
                        float* ml = part + S::ROWS * S::DP + (rt * 16 + n16) * 2;
                        ml[0] = x.m[mq];
                        ml[1] = x.l[mq];
                    }
                }
            }
            if (!whole && tid == 0) ((int*)part)[S::PART - 1] = careful;
        }
        // the next item
        left -= end_tile - tile;
        tile = 0;
        if (dealt) {
            if (!next_dealt()) break;
        } else if (++rb == sq.nrb) {
            rb = 0;
            if (++hk == c.K) {
                hk = 0;
                if (left > 0) {
                    do { sq = uniform(seq_of<S>(p, ++b)); } while (sq.nrb == 0);
                }
            }
        }
    }
}

// The partial results of one cut item added up: block y of a launch has the item that
// stretch y describes, block x its 16 rows.  The four waves share the partial results and
// are added up in LDS.
template <typename T, typename S>
__global__ __launch_bounds__(NT) void k_packed_join(AttnArgs p) {
    constexpr int NB = S::NB, E = 8 * NB;
    extern __shared__ __align__(16) char s_lds[];
    float* const s_o = (float*)s_lds;                // [NW][E][64]
    __shared__ float s_m[NW][16], s_l[NW][16];
    __shared__ int s_flag[NW];
    const int* desc = p.desc + 8 * blockIdx.y;
    const int n = desc[0];
    if (n == 0) return;
    const int slot0 = desc[1], b = desc[2], hk = desc[3], rb = desc[4];
    const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
    const int wave = uniform(threadIdx.x >> 6), rt = blockIdx.x;
    const rheo_packed_attention_args& a = p.a;
    const CacheDev& c = p.c;
    const Seq sq = seq_of<S>(p, b);
    const int rows = sq.rows * p.g;
    if (rb * S::ROWS + rt * 16 >= rows) return;
    const float to2 = a.scale * kLog2e;
    // (slot0 is the first stretch's, maybe its second; the others' first)
    const int w0 = slot0 >> 1, ml = S::ROWS * S::DP + (rt * 16 + n16) * 2, oi = rt * E * 64 + lane;
    float m = -INFINITY, l = 0.0f, o[E];
    int bad = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
#pragma unroll 1
    for (int k = wave; k < n; k += NW) {
        const float* q = c.part + (int64_t)(k ? 2 * (w0 + k) : slot0) * S::PART;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = q[oi + 64 * e];
        const float mk = q[ml], lk = q[ml + 1];
        bad |= ((const int*)q)[S::PART - 1];
        const float top = fmaxf(m, mk), ref = ref_of<T>(top, to2);
        const float f = __builtin_amdgcn_exp2f((m * to2 - kRise<T>) - ref);
        const float h = __builtin_amdgcn_exp2f((mk * to2 - kRise<T>) - ref);
        m = top;
        l = __fmaf_rn(lk, h, l * f);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = __fmaf_rn(y[e], h, o[e] * f);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[(wave * E + e) * 64 + lane] = o[e];
    if (g4 == 0) {
        s_m[wave][n16] = m;
        s_l[wave][n16] = l;
    }
    if (lane == 0) s_flag[wave] = bad;
    __syncthreads();
    if (wave) return;
    m = -INFINITY;
    for (int k = 0; k < NW; ++k) m = fmaxf(m, s_m[k][n16]);
    const float ref = ref_of<T>(m, to2);
    l = 0.0f;
    bad = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    for (int k = 0; k < NW; ++k) {
        const float f = __builtin_amdgcn_exp2f((s_m[k][n16] * to2 - kRise<T>) - ref);
        l = __fmaf_rn(s_l[k][n16], f, l);
        bad |= s_flag[k];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = __fmaf_rn(s_o[(k * E + e) * 64 + lane], f, o[e]);
    }
    const int r = rb * S::ROWS + rt * 16 + n16;
    if (r >= rows) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int qi = r / p.g, qh = hk * p.g + r - qi * p.g;
    const int64_t qrow = (int64_t)b * a.n + qi;
    T* out = (T*)a.out + qrow * a.out_stride + (int64_t)qh * c.D;
    store_row<T, NB>(out, g4, c.D, inv, [&](int t, int i) { return o[4 * t + i]; });
    if (a.lse && g4 == 0) a.lse[qrow * c.H + qh] = lse_of<T>(m, l, a.scale);
    if (bad) add_unfinite<T>(p, b, hk, sq, qi, out, 8 * NB * g4, 8 * NB);
}

namespace {

// Shapes for up to 16, 32, 64, 128 and more rows of an item.
template <int NB>
struct Shapes {
    static constexpr bool W = NB > 4;
    typedef PShape<NB, 1, 1, 2> R1;
    typedef PShape<NB, 2, 1, W ? 1 : 2> R2;
    typedef PShape<NB, W ? 2 : 4, W ? 2 : 1, 1> R4;
    typedef PShape<NB, W ? 2 : 4, W ? 4 : 2, 1> R8;
    typedef PShape<NB, W ? 2 : 4, 4, 1> R16;
};

template <typename S>
size_t part_floats(int units) {
    return (size_t)units * S::RES * 2 * S::PART;
}

template <int NB>
size_t workspace(int units) {
    typedef Shapes<NB> H;
    const size_t n[5] = {part_floats<typename H::R1>(units), part_floats<typename H::R2>(units),
                         part_floats<typename H::R4>(units), part_floats<typename H::R8>(units),
                         part_floats<typename H::R16>(units)};
    size_t most = 0;
    for (size_t x : n) most = x > most ? x : most;
    return most;
}

template <typename T, typename S>
hipError_t start(AttnArgs p, hipStream_t s) {
    p.groups = p.c.slots * S::RES;
    // (fewer items than workgroups: the cuts are what fills them)
    p.whole = (int64_t)p.a.n * p.g <= S::ROWS && p.c.B <= kDealt &&
              (int64_t)p.c.B * p.c.K >= p.groups;
    k_packed_attention<T, S><<<p.groups, NT, S::LDS, s>>>(p);
    k_packed_join<T, S><<<dim3(S::ROWS / 16, p.groups), NT, NW * 8 * S::NB * 64 * 4, s>>>(p);
    return hipGetLastError();
}

template <typename T, int NB>
hipError_t start_rows(const AttnArgs& p, hipStream_t s) {
    typedef Shapes<NB> H;
    const int64_t rows = (int64_t)p.a.n * p.g;
    if (rows <= 16) return start<T, typename H::R1>(p, s);
    if (rows <= 32) return start<T, typename H::R2>(p, s);
    if (rows <= 64) return start<T, typename H::R4>(p, s);
    if (rows <= 128) return start<T, typename H::R8>(p, s);
    return start<T, typename H::R16>(p, s);
}

template <typename T, typename S>
hipError_t allow_lds() {
    hipError_t e = hipSuccess;
    if (S::LDS > 64 * 1024)
        e = hipFuncSetAttribute((const void*)k_packed_attention<T, S>,
                                hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    return e;
}

template <typename T, int NB>
hipError_t prepare_rows() {
    typedef Shapes<NB> H;
    hipError_t e = allow_lds<T, typename H::R1>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R2>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R4>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R8>();
    return e == hipSuccess ? allow_lds<T, typename H::R16>() : e;
}

}  // namespace

// f(a constant: the blocks of 32 elements of a head, 1 to 8)
template <typename F>
auto by_blocks(int nb, F f) {
    switch (nb) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    case 4: return f(std::integral_constant<int, 4>());
    case 5: return f(std::integral_constant<int, 5>());
    case 6: return f(std::integral_constant<int, 6>());
    case 7: return f(std::integral_constant<int, 7>());
    default: return f(std::integral_constant<int, 8>());
    }
}

hipError_t prepare_packed(const CacheDev& c) {
    return by_blocks((c.D + 31) / 32, [&](auto nb) {
        return c.dtype == RHEO_BF16 ? prepare_rows<__bf16, nb>() : prepare_rows<_Float16, nb>();
    });
}

size_t packed_workspace(const CacheDev& c) {
    return by_blocks((c.D + 31) / 32, [&](auto nb) { return workspace<nb>(c.slots); }) +
           (size_t)c.slots * 2 * 8;          // and the descriptions of the joins
}

hipError_t launch_packed_attention(const CacheDev& c, const PackedDev& d,
                                   const rheo_packed_attention_args& a, hipStream_t s) {
    AttnArgs p{};
    p.c = c;
    p.p = d;
    p.a = a;
    p.g = c.H / c.K;
    p.desc = (int*)(c.part + packed_workspace(c) - (size_t)c.slots * 2 * 8);
    return by_blocks(d.nb, [&](auto nb) {
        return c.dtype == RHEO_BF16 ? start_rows<__bf16, nb>(p, s) : start_rows<_Float16, nb>(p, s);
    });
}

}  // namespace rheo
