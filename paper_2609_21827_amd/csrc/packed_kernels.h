// Attention over 4-bit pages and a 16-bit tail (rheo_packed_attention).
//
// o_i = sum_j p_ij v_j with p = softmax_j(scale q_i.k_j), in one pass over the entries
// with a running maximum and sum, for the g = heads / kv_heads query heads of a key head
// and a sequence's rows together, as rheo_tree_attention does it.  What differs is where
// the operands come from: codes, 17 bytes for 32 elements, whose values (exact in 16 bits) the
// matrix cores take.  gfx950 makes a word of two of them from a byte in one instruction.
//
// Products are transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane's scores are all one
// row's and its probabilities are the second product's right operand as they stand.  Up to 16 rows
// each wave makes its operands in registers (own_tiles), 16x16x32; more rows take them
// from LDS, where all waves put them (shared_tiles), 32x32x16.
//
// Work is one line of tiles over all (sequence, key head, block of rows), cut evenly over
// the workgroups; items that are cut leave partial results, which k_packed_join adds up.
// With a window an item's tiles are those of the first entries that stay visible and those
// from the first row's window on.
//
// What bounds it.  Few rows, memory: 128 single tokens over 2000 to 8191 entries (4 key heads
// of 128, fp16, 358 MB) 93 us where a copy's rate would take 72; what is over is the line, the
// items' beginnings one after another, and some workgroups' slower memory.  Up to 256 rows,
// issuing instructions: 64 trees of 244 rows over 1000 to 4096 entries (8 key heads, 0.27 GB,
// 176 GFLOP) 210 to 215 us by box, 818 to 838 TFLOP/s, where a large product's would take 152.
// A SIMD's two waves have 2160 cycles of products a tile of 64 entries and 490 vector
// operations, each 4.6 cycles (measured beside products: 6 + 4.6 n a product of 16.9); one
// wave's chain alone is some 3150 cycles, and the tile takes 4900.  No gain came from one of
// the two waves half a tile later (211 to 237 us), from their priorities, from loads two tiles
// ahead, or from a chunk's scores one chunk ahead (registers spill: 1624 us).  Scores by the
// matrix cores' own 4-bit operands (K as it is, q in two parts of 8 bits) are no faster, and
// off by 2^-16 of the sum of |q k|.
#pragma once

#include <type_traits>

#include "packed_format.h"
#include "packed_heads.h"
#include "softmax_ref.h"

namespace rheo {

namespace {

// A launch's shape: NB blocks of 32 head elements, a workgroup of NW waves, RES of them to a
// compute unit.  SHARED: the waves have 32 rows each and make a tile's operands together, in
// LDS (shared_tiles), 64 entries of it.  Else all have the same 16 rows and every fourth 32
// entries (own_tiles).
template <int NB_, bool SHARED_, int NW_, int RES_>
struct PShape {
    static constexpr bool SHARED = SHARED_;
    static constexpr int NB = NB_, NW = NW_, RES = RES_;
    static constexpr int DP = 32 * NB, NT = 64 * NW;
    static constexpr int WAVES = (RES * NW + 3) / 4;           // a SIMD
    static constexpr int RL = SHARED ? 32 : 16;                // rows of a wave: n of a lane
    static constexpr int EL = RL * DP / 64;                    // elements of one that a lane holds
    static constexpr int EC = EL / NB;                         // ... in a chunk of them
    static constexpr int ROWS = RL * (SHARED ? NW : 1);         // of an item
    static constexpr int KT = SHARED ? 64 : 32 * NW;          // entries of a tile
    static constexpr int ROWB = 2 * DP + 32;                   // see shared_tiles
    static constexpr int STAGE = KT * (2 * DP + ROWB);
    // An item's beginning and end (its lengths, rows and first pages one after another, its
    // results) take as long as some tiles: the line counts as many more for each.  (128
    // single tokens, 4 key heads, over 2000 to 8000 entries: the last workgroup ends at
    // 111 us with none, the mean at 83.)
    static constexpr int SETUP = SHARED ? 4 : 5;
    // a partial result: O^T as the lanes hold it, maximum and sum of each row, a flag
    static constexpr int PART = ROWS * DP + 2 * ROWS + 64;
    static constexpr int RING = NW == 8 ? 3 : 2;             // see shared_tiles
    static constexpr int LDS = SHARED ? RING * STAGE : (NW - 1) * EL * 64 * 4;
    // Element e of a lane's EL, of the lanes' group g (see the mappings above)
    __device__ __forceinline__ static int element(int g, int e) {
        return SHARED ? 32 * (e / 16) + 8 * (e % 16 / 4) + 4 * g + e % 4
                      : 2 * NB * (4 * g + e % 4) + e / 4;
    }
};

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
    int length;                    // on the line: `count` and `setup` before them
    __device__ __forceinline__ int tile(int k) const { return k < head ? k : k - head + from; }
};

// The first entry in the window of a row at position `at`.  Positions and windows may be as
// large as 2^31 - 1, and a row without entries stands before the first: neither wraps
// (entries are fewer than 2^30 + 2^24, and sums of one with a tile stay in 32 bits).
__device__ __forceinline__ int window_begin(int at, int window) {
    return min(max(at, 0) - window + 1, 0x7FFF0000);
}

template <typename S>
__device__ __forceinline__ Span span_of(const AttnArgs& p, const Seq& s, int rb, int setup = 0) {
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
    if (a.window) x.lo = max(window_begin(first, a.window), 0);
    x.pages = (s.len + S::KT - 1) / S::KT;
    const auto tile_of = [&](int e) {
        return e < s.len ? e / S::KT : x.pages + (e - s.len) / S::KT;
    };
    const int end = tile_of(max(x.hi, 0));
    x.from = x.hi < x.lo ? end : tile_of(x.lo);
    x.head = a.window && a.sinks && x.hi >= 0 ? min(tile_of(min(a.sinks - 1, x.hi)) + 1, x.from) : 0;
    x.count = x.head + end - x.from + 1;
    x.length = x.count + setup;
    return x;
}

// The line's part of a sequence and one key head: all its row blocks.
template <typename S>
__device__ __forceinline__ int64_t length_of_head(const AttnArgs& p, const Seq& s, int setup) {
    if (p.a.mask) return s.nrb ? (int64_t)s.nrb * span_of<S>(p, s, 0, setup).length : 0;
    int64_t t = 0;
    for (int rb = 0; rb < s.nrb; ++rb) t += span_of<S>(p, s, rb, setup).length;
    return t;
}

// Addresses in global memory, said so: loads that may be of LDS as well would wait for both.
template <typename T>
using Global = const __attribute__((address_space(1))) T*;
template <typename T>
__device__ __forceinline__ Global<T> global(const void* q) { return (Global<T>)(const T*)q; }
template <typename T, int A>
__device__ __forceinline__ T load(Global<uint8_t> q) {
    struct __attribute__((packed, aligned(A))) Word { T v; };
    return ((const __attribute__((address_space(1))) Word*)q)->v;
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
    return Span{uniform(s.lo),   uniform(s.hi),    uniform(s.pages), uniform(s.head),
                uniform(s.from), uniform(s.count), uniform(s.length)};
}

// Stretch w of the line: tiles [t0, t1) of it, the sequence that t0 is in and the tiles
// before that sequence.  All threads of the block call it.
struct Stretch {
    int64_t total, t0, t1, before;
    int groups, seq, setup;        // (setup: see SETUP; what an item's length has of it)
    Seq of;                        // that sequence's
};

// a / b of numbers that are seldom past 32 bits (a 64-bit division is some hundred
// instructions, one after another)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    if (((uint64_t)a | (uint64_t)b) >> 32) return a / b;
    return (uint32_t)a / (uint32_t)b;
}

__device__ __forceinline__ int64_t stretch_start(int64_t total, int groups, int w) {
    return quotient(total * w, groups);
}
// the stretch that place t of the line is in
__device__ __forceinline__ int stretch_of(int64_t total, int groups, int64_t t) {
    return (int)quotient((t + 1) * groups - 1, total);
}

template <typename S>
__device__ Stretch find_stretch(const AttnArgs& p, int w) {
    __shared__ int64_t s_wave[S::NW], s_items[S::NW], s_before;
    __shared__ int s_seq;
    __shared__ Seq s_of;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = p.c.B;
    const int per = (B + S::NT - 1) / S::NT, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    int64_t mine = 0, items = 0;             // tiles and items of the thread's sequences
    for (int b = b0; b < b1; ++b) {
        const Seq s = seq_of<S>(p, b);
        mine += p.c.K * length_of_head<S>(p, s, 0);
        items += (int64_t)p.c.K * s.nrb;
    }
    int64_t incl = mine, incl_items = items;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t u = __shfl_up(incl, o), v = __shfl_up(incl_items, o);
        if (lane >= o) {
            incl += u;
            incl_items += v;
        }
    }
    if (lane == 63) {
        s_wave[wave] = incl;
        s_items[wave] = incl_items;
    }
    __syncthreads();
    int64_t excl = incl - mine, total = 0, excl_items = incl_items - items, all_items = 0;
    for (int v = 0; v < S::NW; ++v) {
        if (v < wave) {
            excl += s_wave[v];
            excl_items += s_items[v];
        }
        total += s_wave[v];
        all_items += s_items[v];
    }
    Stretch r;
    // (where every tile can have a workgroup, each begins one item at most)
    r.setup = uniform(total > p.groups ? S::SETUP : 0);
    total = uniform64(total + r.setup * all_items);
    excl += r.setup * excl_items;
    mine += r.setup * items;
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
            const Seq s = seq_of<S>(p, b);
            const int64_t k = p.c.K * length_of_head<S>(p, s, r.setup);
            if (r.t0 < t + k) {
                s_seq = b;
                s_of = s;
                s_before = t;
                break;
            }
            t += k;
        }
    }
    __syncthreads();
    r.seq = uniform(s_seq);
    r.of = uniform(s_of);
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
__device__ bool deal_items(const AttnArgs& p, int64_t total, int setup, int* s_order) {
    __shared__ int s_tiles[kDealt], s_most[S::NW];
    const int tid = threadIdx.x, B = p.c.B, K = p.c.K, items = B * K;
    __syncthreads();
    for (int b = tid; b < B; b += S::NT) {
        const Seq s = seq_of<S>(p, b);
        s_tiles[b] = s.nrb ? span_of<S>(p, s, 0, setup).length : 0;
    }
    __syncthreads();
    for (int b = tid; b < B; b += S::NT) {
        const int mine = s_tiles[b];
        int rank = 0;
        for (int o = 0; o < B; ++o) rank += s_tiles[o] > mine || (s_tiles[o] == mine && o < b);
        s_order[rank] = b;
    }
    __syncthreads();
    int most = 0;
    for (int w = tid; w < p.groups; w += S::NT) {
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
    for (int w = 0; w < S::NW; ++w) most = max(most, s_most[w]);
    const int64_t mean = total / p.groups;
    return most <= mean + mean / 16 + 8;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lds_s4;

template <typename T>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, const f32x16& c) {
    typedef typename Pack<T>::v8 v8;
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
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

// Both elements of a word 0 where they are infinite or NaN.
template <typename T>
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    constexpr uint32_t E = Pack<T>::kExp;
    return ((w & E) == E ? 0 : w & 0xFFFFu) | ((w & E << 16) == E << 16 ? 0 : w & 0xFFFF0000u);
}

// The blocks of a lane's elements of K at step s, and of its pair p of V.
template <int NB>
__device__ __forceinline__ int k_block(int g, int s) { return (NB * g + s) >> 2; }
template <int NB>
__device__ __forceinline__ int v_block(int n, int p) { return (NB * n + p) >> 4; }

// What a wave holds of an item: lane RL g + n has row n's.
template <typename S>
struct Rows {
    typedef std::conditional_t<S::SHARED, f32x16, f32x4> Part;
    static constexpr int QS = S::SHARED ? 2 * S::NB : S::NB, VL = S::SHARED ? 16 : 4;
    u32x4 q[QS];
    Part o[S::EL / VL];
    float m, l;                    // the exponents' reference, a score; the lane's sum
    int lo, hi;                    // entries that the row attends (and sinks)
    uint32_t mask;                 // its row of the mask
    __device__ __forceinline__ float at(int e) const { return o[e / VL][e % VL]; }
};

// The exponents' reference follows a row's own maximum by steps (kSlack), so that O is
// rescaled once or twice an item.  `mx`: the largest of the lane's scores.
template <typename T, typename S>
__device__ __forceinline__ void follow(Rows<S>& x, float mx, float to2, float slack) {
    if (!__any(mx > x.m + slack)) return;
    float m = mx;
#pragma unroll
    for (int o = S::RL; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    const bool mine = m > x.m + slack;
    const float f = mine ? __builtin_amdgcn_exp2f((x.m * to2 - kRise<T>) - ref_of<T>(m, to2)) : 1.0f;
    x.l *= f;
#pragma unroll
    for (int t = 0; t < S::EL / Rows<S>::VL; ++t) x.o[t] *= f;
    x.m = mine ? m : x.m;
}

// Eight scores of a lane to probabilities.  The sum takes them unrounded, the second product
// in 16 bits, what the matrix cores take.  That is a choice, rheo_tree_attention's: the rounding
// is off by nearly as much again as the output's (trees over 4096 entries, bf16: 2.3e-3 of the
// norm against 64 bits, 1.7e-3 by the output's alone), and a second product with what it left
// over would lengthen a loop that is bound by issuing instructions.
template <typename T>
__device__ __forceinline__ u32x4 weights(const f32x4 (&sc)[2], float m, float to2, float* l) {
    const float ref = ref_of<T>(m, to2);
    float e[8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[i >> 2][i & 3], to2, -ref));
        sum += e[i];
    }
    *l += sum;
    u32x4 pt;
#pragma unroll
    for (int i = 0; i < 4; ++i) pt[i] = pack2<T>(e[2 * i], e[2 * i + 1]);
    return pt;
}

// The operands of two tiles of V from the words w of eight entries.
__device__ __forceinline__ void by_entries(const uint32_t (&w)[8], u32x4* lo, u32x4* hi) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        (*lo)[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
        (*hi)[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
    }
}

// The infinite and NaN values of the tail, which the products left out, added to a lane's
// elements of chunk c of a finished row that attends them.  Their probabilities are not 0, so
// the values themselves decide.  Rare and slow.
template <typename T, typename S>
__device__ __forceinline__ void add_unfinite(const AttnArgs& p, int b, int hk, const Seq& sq, int qi,
                                             T* out, int g, int c) {
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
        for (int i = 0; i < S::EC; ++i) {
            const int d = S::element(g, c * S::EC + i);
            if (d >= p.c.D) continue;
            const float x = (float)v[d];
            if (!(fabsf(x) < INFINITY)) out[d] = (T)((float)out[d] + x);
        }
    }
}

// A lane's chunk c of a row, f in the order of the lanes' O^T.
template <typename T, typename S>
__device__ __forceinline__ void store_chunk(T* out, int g, int c, int D, const float (&f)[S::EC]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (S::SHARED) {
            const int d = S::element(g, c * 16 + 4 * i);
            if (d < D)
                *(uint2*)(out + d) =
                    make_uint2(pack2<T>(f[4 * i], f[4 * i + 1]), pack2<T>(f[4 * i + 2], f[4 * i + 3]));
        } else {
            const int d = S::element(g, c * 8 + i);
            if (d < D) *(uint32_t*)(out + d) = pack2<T>(f[i], f[4 + i]);
        }
    }
}

// What a wave needs of the item at hand.
struct Item {
    int b, hk, rb;
    Seq sq;
    Span span;
    int tile, end_pages, end_tile;           // the stretch's tiles of it: the pages', the tail's
    int lo_most, hi_least, sinks;            // entries that all rows of the wave attend:
                                             // lo_most to hi_least
    bool idle;                               // the wave has no rows
    // Whether some row attends entry e of the pages; one of the 16 from e on (others are not
    // read); whether no row attends one of the 32 from e on; whether one of the wave's rows
    // does not attend one of these.
    __device__ __forceinline__ bool attended(int e) const {
        return e < sq.len && e <= span.hi && (e >= span.lo || e < sinks);
    }
    // (the window may begin behind the pages' end: the last of the 16 that is there decides)
    __device__ __forceinline__ bool wanted(int e) const {
        const int last = min(e + 15, min(sq.len - 1, span.hi));
        return e <= last && (last >= span.lo || e < sinks);
    }
    __device__ __forceinline__ bool some_idle(int e) const {
        return !(e + 31 < sq.len && e + 31 <= span.hi && (e >= span.lo || e + 31 < sinks));
    }
    // (of the first `there` entries; those behind the pages are the tail's)
    __device__ __forceinline__ bool some_hidden(int e, int there) const {
        return !(e + 31 < there && e + 31 <= hi_least && (e >= lo_most || e + 31 < sinks));
    }
    // `attended` of four entries, as bytes
    __device__ __forceinline__ uint32_t attended_bytes(int e) const {
        uint32_t keep = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) keep |= attended(e + r) ? 0xFFu << (8 * r) : 0;
        return keep;
    }
};

// A page's first byte, from its number, the same in all lanes.
__device__ __forceinline__ int64_t page_at(const AttnArgs& p, int page) {
    page = uniform(page);
    if ((unsigned)page >= (unsigned)p.c.pages) {
        if ((threadIdx.x & 63) == 0) atomicOr(p.c.err, CE_PAGE);
        page = 0;
    }
    return page * p.p.page_stride;
}

// Scores of what a lane's row does not attend made -inf: `entry(i)` is that of score i, behind
// the pages the tail's row entry(i) - len.
template <typename S, bool TAIL, int N, typename Entry, typename Score>
__device__ __forceinline__ void hide(const AttnArgs& p, const Item& it, const Rows<S>& x, int e0,
                                     Entry entry, Score score) {
    const int there = it.sq.len + (TAIL ? it.sq.tail : 0);
    if (TAIL && p.a.mask) {
        const Global<uint8_t> row = global<uint8_t>(p.a.mask) + (int64_t)x.mask * p.a.tail;
        uint8_t named[N];
#pragma unroll
        for (int i = 0; i < N; ++i) named[i] = row[min(entry(i), there - 1) - it.sq.len];
#pragma unroll
        for (int i = 0; i < N; ++i)
            score(i) = ((named[i] != 0) & (entry(i) < there)) ? score(i) : -INFINITY;
    } else if (it.some_hidden(e0, there)) {
        const int hi = min(x.hi, there - 1);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = entry(i);
            score(i) = ((e <= hi) & ((e >= x.lo) | (e < it.sinks))) ? score(i) : -INFINITY;
        }
    }
}

// The exponent of V's pair p among those loaded of a lane's blocks (the first pair's and,
// unless the lane's pairs all lie in one block, the last one's).
template <int NB, int SB>
__device__ __forceinline__ uint32_t v_scale(const uint32_t (&vs)[SB], int n16, int p0, int p) {
    if constexpr (SB == 1) return vs[0];
    else return v_block<NB>(n16, p) == v_block<NB>(n16, p0) ? vs[0] : vs[1];
}
__device__ __forceinline__ float scale_of_entry(uint32_t w, int j) {
    return j == 0 ? scale_at<0>(w) : j == 1 ? scale_at<1>(w) : j == 2 ? scale_at<2>(w) : scale_at<3>(w);
}
template <typename T>
__device__ __forceinline__ uint32_t pair_at(uint32_t codes, float f, int byte) {
    return byte == 0   ? pair_of<T, 0>(codes, f)
           : byte == 1 ? pair_of<T, 1>(codes, f)
           : byte == 2 ? pair_of<T, 2>(codes, f)
                       : pair_of<T, 3>(codes, f);
}

// An item's tiles by waves that have the same rows and share the entries: codes straight into
// registers, operands made there, a wave for itself, the codes of the next tile on their
// way.  (128 single tokens as above: two tiles on their way 113 us for 103, three workgroups a
// compute unit, whose registers spill, 144.)
template <typename T, typename S>
__device__ __forceinline__ void own_tiles(const AttnArgs& p, const Item& it, Rows<S>& x, bool careful) {
    constexpr int NB = S::NB;
    constexpr bool P2 = (NB & (NB - 1)) == 0;
    constexpr int VW = NB <= 4 ? 1 : 2;              // words of an entry's V a lane
    constexpr int SB = P2 ? 1 : 2;                   // blocks that these lie in
    constexpr int KS = P2 ? (NB + 3) / 4 : NB;       // exponents of K a lane
    const CacheDev& c = p.c;
    const rheo_packed_attention_args& a = p.a;
    const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
    const int wt = uniform(threadIdx.x >> 6), D = c.D;
    const Seq& sq = it.sq;
    const float to2 = a.scale * kLog2e;              // scores to exponents of 2
    const float slack = kSlack<T> / to2;
    const int in_page = (1 << c.page_shift) - 1;
    const int scales = 16 * NB << c.page_shift;      // where a head's page has its exponents
    // the lane's offsets from an entry block's first codes and exponents
    const uint32_t k_at = n16 * 16 * NB + 4 * NB * g4, v_at = 4 * g4 * 16 * NB + NB * n16;
    uint32_t kx_at[KS], vx_at[SB];
#pragma unroll
    for (int s = 0; s < KS; ++s) kx_at[s] = (k_block<NB>(g4, P2 ? 4 * s : s) << c.page_shift) + n16;
#pragma unroll
    for (int s = 0; s < SB; ++s)
        vx_at[s] = (v_block<NB>(n16, s * (NB - 1)) << c.page_shift) + 4 * g4;
    const Global<int32_t> row_table = global<int32_t>(a.table) + (int64_t)it.b * c.width;
    const Global<uint8_t> k_head = global<uint8_t>(p.p.k) + it.hk * p.p.head;
    const Global<uint8_t> v_head = global<uint8_t>(p.p.v) + it.hk * p.p.head;

    // a tile's 32 entries of the wave: their pages, two blocks', and their codes
    uint32_t rk[2][NB], rks[2][KS], rv[8][VW], rvs[2][SB];
    int page0 = 0, page1 = 0;
    const auto begins = [&](int k) { return it.span.tile(k) * S::KT + 32 * wt; };
    const auto fetch_pages = [&](int k) {
        if (k >= it.end_pages) return;
        const int e0 = begins(k);
        const bool n0 = it.wanted(e0), n1 = it.wanted(e0 + 16);
        if (!(n0 | n1)) return;
        page0 = row_table[(n0 ? e0 : e0 + 16) >> c.page_shift];
        page1 = row_table[(n1 ? e0 + 16 : e0) >> c.page_shift];
    };
    const auto fetch = [&](int k) {
        if (k >= it.end_pages) return;
        const int e0 = begins(k);
        if (!(it.wanted(e0) | it.wanted(e0 + 16))) return;
        const int64_t page[2] = {page_at(p, page0), page_at(p, page1)};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i0 = (e0 + 16 * u) & in_page;
            const Global<uint8_t> kc = k_head + page[u] + i0 * (16 * NB);
            const Global<uint8_t> vc = v_head + page[u] + i0 * (16 * NB);
            const Global<uint8_t> kx = k_head + page[u] + scales + i0;
            const Global<uint8_t> vx = v_head + page[u] + scales + i0;
#pragma unroll
            for (int s = 0; s < NB; ++s) rk[u][s] = load<uint32_t, 4>(kc + k_at + 4 * s);
#pragma unroll
            for (int s = 0; s < KS; ++s) rks[u][s] = kx[kx_at[s]];
            // (a lane's NB bytes at any place: the whole words' last may be the next entry's,
            // or of the exponents behind the last)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < VW; ++i)
                    rv[4 * u + j][i] = load<uint32_t, VW == NB / 4 ? 4 : 1>(vc + v_at + (j * 16 * NB + 4 * i));
#pragma unroll
            for (int s = 0; s < SB; ++s) rvs[u][s] = load<uint32_t, 4>(vx + vx_at[s]);
        }
    };
    // the scores of 32 entries from e0 on to O, with V's operands at hand
    const auto finish = [&](f32x4 (&sc)[2], const u32x4 (&vo)[2 * NB], int e0, auto tail) {
        hide<S, decltype(tail)::value, 8>(
            p, it, x, e0, [&](int i) { return e0 + 16 * (i >> 2) + 4 * g4 + (i & 3); },
            [&](int i) -> float& { return ((float*)&sc[0])[i]; });
        const float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                               fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
        follow<T, S>(x, mx, to2, slack);
        const u32x4 pt = weights<T>(sc, x.m, to2, &x.l);
#pragma unroll
        for (int t = 0; t < 2 * NB; ++t) x.o[t] = mfma<T>(vo[t], pt, x.o[t]);
    };

    fetch_pages(it.tile);
    fetch(it.tile);
    fetch_pages(it.tile + 1);
#pragma unroll 1
    for (int k = it.tile; k < it.end_pages; ++k) {
        const int e0 = begins(k);
        if (!(it.wanted(e0) | it.wanted(e0 + 16))) {
            fetch(k + 1);
            fetch_pages(k + 2);
            continue;
        }
        if (it.some_idle(e0)) {
            // what nobody attends is any bytes: its exponents 0, so that its values are finite
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t keep = it.attended_bytes(e0 + 16 * u + 4 * g4);
#pragma unroll
                for (int s = 0; s < SB; ++s) rvs[u][s] &= keep;
            }
        }
        f32x4 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NB; ++s) {
                const float f = scale_of(rks[u][P2 ? s / 4 : s]);
                const uint32_t w = rk[u][s];
                const u32x4 ko{pair_of<T, 0>(w, f), pair_of<T, 1>(w, f), pair_of<T, 2>(w, f),
                               pair_of<T, 3>(w, f)};
                sc[u] = mfma<T>(ko, x.q[s], sc[u]);
            }
        }
        u32x4 vo[2 * NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[j] = pair_at<T>(rv[j][q / 4],
                                  scale_of_entry(v_scale<NB>(rvs[j >> 2], n16, 0, q), j & 3), q % 4);
            by_entries(w, &vo[2 * q], &vo[2 * q + 1]);
        }
        fetch(k + 1);
        fetch_pages(k + 2);
        finish(sc, vo, e0, std::false_type());
    }
    const Global<uint8_t> kt = global<uint8_t>(a.k_tail) + 2 * it.hk * D;
    const Global<uint8_t> vt = global<uint8_t>(a.v_tail) + 2 * it.hk * D;
    const int64_t row_bytes = 2 * a.tail_stride;
    const int64_t row0 = (int64_t)it.b * a.tail;
#pragma unroll 1
    for (int k = max(it.tile, it.end_pages); k < it.end_tile; ++k) {
        const int j0 = (it.span.tile(k) - it.span.pages) * S::KT + 32 * wt;
        if (j0 >= sq.tail) continue;
        f32x4 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Global<uint8_t> row = kt + (row0 + min(j0 + 16 * u + n16, sq.tail - 1)) * row_bytes;
            sc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < NB; ++s) {
                const int d = 8 * NB * g4 + 8 * s;
                u32x4 ko = load<u32x4, 16>(row + 2 * min(d, D - 8));
                if (d >= D) ko = u32x4{0, 0, 0, 0};
                sc[u] = mfma<T>(ko, x.q[s], sc[u]);
            }
            // (one block's loads after the other's products: registers, which the loop over
            // the pages has use for)
            __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 vo[2 * NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            __builtin_amdgcn_sched_barrier(0);
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = j0 + 16 * (j >> 2) + 4 * g4 + (j & 3);
                // (pairs past the head are columns that no one stores)
                w[j] = load<uint32_t, 4>(vt + (row0 + min(at, sq.tail - 1)) * row_bytes +
                                         4 * min(NB * n16 + q, D / 2 - 1));
                if (at >= sq.tail) w[j] = 0;
                if (careful) w[j] = finite_pair<T>(w[j]);
            }
            by_entries(w, &vo[2 * q], &vo[2 * q + 1]);
        }
        finish(sc, vo, sq.len + j0, std::true_type());
    }
}

// An item's tiles by waves of different rows, of the pages or of the tail.  The waves make a
// tile's operands together and put them into LDS, K as the lanes take it (`lane` of operand i
// has 16 bytes at (64 i + lane) 16), V as rows of the entries' elements, 32 bytes more than
// they have apart (a third of LDS's busy cycles are bank conflicts; with 64 bytes a fifth, in the
// same time); then each multiplies them with its own rows, as 32x32x16 tiles (half the
// instructions of 16x16x32: issuing them is what bounds this loop).  While tile t is worked
// on, t + RING - 1 is written, whose codes were loaded a tile earlier; so a barrier a tile.
template <typename T, typename S, bool TAIL>
__device__ __forceinline__ void shared_tiles(const AttnArgs& p, const Item& it, Rows<S>& x,
                                             bool careful, char* lds) {
    constexpr int NB = S::NB, KT = S::KT, KS = 2 * NB;
    // the waves to a chunk of 32 entries, and the blocks of 32 elements that each makes of it
    constexpr int U = 2, VP = S::NW / U, NS = (NB + VP - 1) / VP;
    constexpr int V0 = KT * S::DP * 2, ROWB = S::ROWB;       // where a stage has V; bytes between rows
    const CacheDev& c = p.c;
    const rheo_packed_attention_args& a = p.a;
    const int lane = threadIdx.x & 63, n32 = lane & 31, half = lane >> 5;
    const int wave = uniform(threadIdx.x >> 6), D = c.D;
    const Seq& sq = it.sq;
    const float to2 = a.scale * kLog2e;              // scores to exponents of 2
    const float slack = kSlack<T> / to2;
    const int in_page = (1 << c.page_shift) - 1;
    const int vc = wave / VP, part = wave % VP;      // blocks part, part + VP, ... of chunk vc
    const Global<int32_t> row_table = global<int32_t>(a.table) + (int64_t)it.b * c.width;
    const Global<uint8_t> k_head = global<uint8_t>(p.p.k) + it.hk * p.p.head;
    const Global<uint8_t> v_head = global<uint8_t>(p.p.v) + it.hk * p.p.head;
    const Global<uint8_t> kt = global<uint8_t>(a.k_tail) + 2 * it.hk * D;
    const Global<uint8_t> vt = global<uint8_t>(a.v_tail) + 2 * it.hk * D;
    const int64_t row_bytes = 2 * a.tail_stride;
    const int64_t row0 = (int64_t)it.b * a.tail;
    const int begin = TAIL ? max(it.tile, it.end_pages) : it.tile;
    const int end = TAIL ? it.end_tile : it.end_pages;
    if (begin >= end || (TAIL && sq.tail == 0)) return;

    // (of page 0, entry 0: what the lane reads of K; V is as far from it everywhere)
    const Global<uint8_t> k_codes = k_head + (16 * part + 8 * half);
    const Global<uint8_t> k_exps = k_head + ((16 * NB + part) << c.page_shift);
    const int64_t v_less_k = v_head - k_head;
    const uint32_t stride = (uint32_t)p.p.page_stride;

    // Lane 32 h + n makes elements 16 h to 16 h + 15 of its blocks, of entry n of the chunk.
    // A tile's part as loaded: codes and exponents, or (of the tail) the elements themselves.
    uint32_t rk[NS][TAIL ? 8 : 2], rv[NS][TAIL ? 8 : 2], rks[NS], rvs[NS];
    int page = 0;
    bool outside = false;                            // a page's number is
    // (the first entry of tile k's chunk: of the pages, or of the tail)
    const auto first = [&](int k) {
        const int v = it.span.tile(k);
        return (TAIL ? v - it.span.pages : v) * KT + 32 * vc;
    };
    const auto fetch_pages = [&](int k, bool plain = false) {
        if (TAIL || (!plain && k >= end)) return;
        const int e = first(k) + n32;
        if (plain || it.attended(e)) page = row_table[e >> c.page_shift];
    };
    const auto fetch = [&](int k, bool plain = false) {
        if (!plain && k >= end) return;
        const int e = first(k);
        if constexpr (!TAIL) {
            // (an entry that no row attends is not read: it counts as zeros)
            const bool in = plain || it.attended(e + n32);
            if (!in) {
#pragma unroll
                for (int s = 0; s < NS; ++s) rk[s][0] = rk[s][1] = rv[s][0] = rv[s][1] = rks[s] = rvs[s] = 0;
            } else {
                const bool good = (unsigned)page < (unsigned)c.pages;
                outside |= !good;
                const uint32_t entry = (e + n32) & in_page, from = good ? page : 0;
                const Global<uint8_t> kc = k_codes + (uint64_t)from * stride + (uint64_t)entry * (16 * NB);
                const Global<uint8_t> kx = k_exps + (uint64_t)from * stride + entry;
                const Global<uint8_t> vc = kc + v_less_k, vx = kx + v_less_k;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    // (blocks past the last: the last one's, of no use)
                    const int up = NB % VP == 0 ? VP * s : min(VP * s, NB - 1 - part);
                    const u32x2 w = load<u32x2, 8>(kc + 16 * up), y = load<u32x2, 8>(vc + 16 * up);
                    rk[s][0] = w[0];
                    rk[s][1] = w[1];
                    rv[s][0] = y[0];
                    rv[s][1] = y[1];
                    rks[s] = kx[up << c.page_shift];
                    rvs[s] = vx[up << c.page_shift];
                }
            }
        } else {
            const int64_t row = (row0 + min(e + n32, sq.tail - 1)) * row_bytes;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // (elements past the head: the last ones', made 0 in K, of no use in V)
                    const int d = min(32 * (part + VP * s) + 16 * half + 8 * i, D - 8);
                    const u32x4 w = load<u32x4, 16>(kt + row + 2 * d), y = load<u32x4, 16>(vt + row + 2 * d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        rk[s][4 * i + j] = w[j];
                        rv[s][4 * i + j] = y[j];
                    }
                }
        }
    };
    const auto put = [&](int k, int stage, bool plain = false) {
        if (!plain && k >= end) return;
        const int e = first(k);
        char* const ks = lds + stage * S::STAGE + (vc * KS * 64 + n32) * 16;
        char* const vs = lds + stage * S::STAGE + V0 + (32 * vc + n32) * ROWB + 32 * half;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            const int block = part + VP * s;
            if (NB % VP != 0 && block >= NB) continue;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 w, y;
                if constexpr (!TAIL) {
                    const float f = scale_of(rks[s]), g = scale_of(rvs[s]);
                    w = u32x4{pair_of<T, 0>(rk[s][i], f), pair_of<T, 1>(rk[s][i], f),
                              pair_of<T, 2>(rk[s][i], f), pair_of<T, 3>(rk[s][i], f)};
                    y = u32x4{pair_of<T, 0>(rv[s][i], g), pair_of<T, 1>(rv[s][i], g),
                              pair_of<T, 2>(rv[s][i], g), pair_of<T, 3>(rv[s][i], g)};
                } else {
                    const bool there = e + n32 < sq.tail, in = 32 * block + 16 * half + 8 * i < D;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        w[j] = in ? rk[s][4 * i + j] : 0;
                        y[j] = there ? rv[s][4 * i + j] : 0;
                        if (careful) y[j] = finite_pair<T>(y[j]);
                    }
                }
                *(u32x4*)(ks + ((2 * block + half) * 64 + 32 * i) * 16) = w;
                *(u32x4*)(vs + 64 * block + 16 * i) = y;
            }
        }
    };
    const auto barrier = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    constexpr int ON = S::RING - 1;                  // tiles that are written ahead
    __syncthreads();                                 // (the stages are free)
    fetch_pages(begin);
    fetch(begin);
    fetch_pages(begin + 1);
#pragma unroll
    for (int i = 0; i < ON; ++i) {
        put(begin + i, i);
        fetch(begin + i + 1);
        fetch_pages(begin + i + 2);
    }
    barrier();
    // Tiles k to k + ON + 2 of which all rows attend everything: from `easy` on, before `hard`
    int easy = end, hard = end;
    if constexpr (!TAIL) {
        const int lo = max(it.lo_most, it.span.lo), hi = min(it.hi_least, min(it.span.hi, sq.len - 1));
        const int shift = it.span.head - it.span.from;
        easy = max((lo + KT - 1) / KT + shift, it.span.head);
        hard = min((hi + 1) / KT + shift, end) - ON - 2;
    }
    // the lane's place in V's first 4x16 blocks: 4 entries of a half's 16 elements
    const uint32_t v_at = (4 * half + (lane & 15) / 4) * ROWB +
                          (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) * 16 + (lane & 1) * 8;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    constexpr int AHEAD = KS * U < 6 ? KS * U : 6;
    const auto k_part = [&](int stage, int i) {      // K's operand i: step i / U of chunk i % U
        return *(const u32x4*)(lds + stage * S::STAGE + lane * 16 + (i % U * KS + i / U) * 1024);
    };
    u32x4 ahead[AHEAD];
    if constexpr (ON == 2)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) ahead[i] = k_part(0, i);
    int stage = 0;                                   // of tile k
    // A wave without rows makes its part of the operands only.  (32 sequences of 0 to 488 rows
    // over some 20000 entries: 574 us to 524.)
    if (it.idle) {
#pragma unroll 1
        for (int k = begin; k < end; ++k) {
            stage = stage + 1 == S::RING ? 0 : stage + 1;
            put(k + ON, ON == 1 ? stage : stage + 1 == S::RING ? 0 : stage + 1);
            fetch(k + ON + 1);
            fetch_pages(k + ON + 2);
            barrier();
        }
        if (outside) atomicOr(c.err, CE_PAGE);
        return;
    }
#pragma unroll 1
    for (int k = begin; k < end; ++k) {
        const int next = stage + 1 == S::RING ? 0 : stage + 1;
        const int write = ON == 1 ? next : next + 1 == S::RING ? 0 : next + 1;
        const bool plain = k >= easy && k < hard;
        f32x16 sc[U];
#pragma unroll
        for (int u = 0; u < U; ++u) sc[u] = 0.0f;
#pragma unroll
        for (int i = 0; i < KS * U; ++i)
            sc[i % U] = mfma32<T>(ON == 2 && i < AHEAD ? ahead[i] : k_part(stage, i), x.q[i / U], sc[i % U]);
        // reads ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < KS * U - AHEAD; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
        put(k + ON, write, plain);
        fetch(k + ON + 1, plain);
        fetch_pages(k + ON + 2, plain);
        if (!plain) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e0 = (TAIL ? sq.len : 0) + first(k) + 32 * (u - vc);
                hide<S, TAIL, 16>(
                    p, it, x, e0, [&](int i) { return e0 + 4 * half + 8 * (i / 4) + i % 4; },
                    [&](int i) -> float& { return ((float*)&sc[u])[i]; });
            }
        }
        float mx = sc[0][0];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
        follow<T, S>(x, mx, to2, slack);
        // The sum takes the probabilities unrounded, the second product in 16 bits, what the
        // matrix cores take.
        const float ref = ref_of<T>(x.m, to2);
        float sum = 0.0f;
        const uint32_t vp = lds_at + stage * S::STAGE + V0 + v_at;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 pt;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e0 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[u][8 * j + 2 * i], to2, -ref));
                    const float e1 = __builtin_amdgcn_exp2f(__fmaf_rn(sc[u][8 * j + 2 * i + 1], to2, -ref));
                    sum += e0;
                    sum += e1;
                    pt[i] = pack2<T>(e0, e1);
                }
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const uint32_t at = vp + (32 * u + 16 * j) * ROWB + 64 * d;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)at);
                    const s16x4 hi =
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(uintptr_t)(at + 8 * ROWB));
                    const s16x8 va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    x.o[d] = mfma32<T>(__builtin_bit_cast(u32x4, va), pt, x.o[d]);
                }
            }
        }
        x.l += sum;
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
        for (int i = 0; i < NB * U * 2 - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 1);
        // (past the last tile: what is there, of no use)
        if constexpr (ON == 2)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) ahead[i] = k_part(next, i);
        barrier();
        stage = next;
    }
    if (outside) atomicOr(c.err, CE_PAGE);
}

}  // namespace

template <typename T, typename S>
__global__ __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(S::WAVES, S::WAVES))) void
k_packed_attention(AttnArgs p) {
    constexpr int RL = S::RL;
    extern __shared__ __align__(16) char s_lds[];
    __shared__ float s_ml[S::SHARED ? 2 : S::NW * 16 * 2];
    __shared__ int s_order[S::SHARED ? kDealt : 1];    // sequences, the longest first
    const int tid = threadIdx.x, lane = tid & 63, n = lane % RL, g = lane / RL;
    const int wave = uniform(tid >> 6), tile0 = S::SHARED ? wave : 0;
    const CacheDev& c = p.c;
    const rheo_packed_attention_args& a = p.a;
    const int w = blockIdx.x, D = c.D;
    const float to2 = a.scale * kLog2e;              // scores to exponents of 2

    Stretch st = find_stretch<S>(p, w);
    bool dealt = false;
    if constexpr (S::SHARED)
        if (p.whole && st.groups == p.groups)
            dealt = uniform(deal_items<S>(p, st.total, st.setup, s_order)) != 0;
    if (tid == 0) p.desc[8 * w] = 0;
    if (!dealt && st.t0 >= st.t1) return;
    // the item at hand: sequence, key head, row block, its tile to begin with; the
    // tiles left of the stretch, or the round of the deal
    int b = 0, hk = 0, rb = 0, tile = 0, round = 0;
    int64_t left = 0;
    Seq sq;
    auto next_dealt = [&]() {
        for (; S::SHARED && round * p.groups < c.B * c.K; ++round) {
            const int i = dealt_item(round, w, p.groups);
            if (i >= c.B * c.K) continue;
            b = uniform(s_order[i / c.K]);
            hk = i % c.K;
            sq = uniform(seq_of<S>(p, b));
            if (sq.nrb) {
                left = uniform(span_of<S>(p, sq, 0, st.setup).length);
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
        sq = st.of;
        int64_t rel = st.t0 - st.before;
        const int64_t per_head = length_of_head<S>(p, sq, st.setup);
        hk = uniform((int)quotient(rel, per_head));
        rel -= hk * per_head;
        for (int n; rel >= (n = span_of<S>(p, sq, rb, st.setup).length); ++rb) rel -= n;
        rb = uniform(rb);
        tile = uniform((int)rel);
        left = st.t1 - st.t0;
        // the join of the first item, by the first cut inside it
        const int64_t begins = st.t0 - tile, ends = begins + span_of<S>(p, sq, rb, st.setup).length;
        if (tid == 0 && tile > 0 && stretch_start(st.total, st.groups, w - 1) <= begins) {
            int* d = p.desc + 8 * w;
            d[0] = stretch_of(st.total, st.groups, ends - 1) - w + 2;    // partial results
            d[1] = 2 * (w - 1) + (stretch_start(st.total, st.groups, w - 1) < begins ? 1 : 0);
            d[2] = b;
            d[3] = hk;
            d[4] = rb;
        }
    }

    for (bool first = true; left > 0; first = false) {
        const Span span = uniform(span_of<S>(p, sq, rb, st.setup));
        const int end_place = (int)min((int64_t)span.length, tile + left);
        // its tiles in the stretch: of the pages, then of the tail (none: a part of nothing)
        const int begin_tile = max(tile - st.setup, 0), end_tile = max(end_place - st.setup, 0);
        const int end_pages = min(end_tile, span.from < span.pages ? span.pages - span.from + span.head
                                                                   : min(span.head, span.pages));
        Rows<S> x;
        int lo_most = 0, hi_least = 0x7FFFFFFF;
        const int row = rb * S::ROWS + tile0 * RL + n;
        const bool live = row < sq.rows * p.g;
        const int qi = live ? row / p.g : 0, qh = hk * p.g + (live ? row - qi * p.g : 0);
        const int64_t qrow = (int64_t)b * a.n + qi;
        {
            const T* q = (const T*)a.q + qrow * a.q_stride + (int64_t)qh * D;
#pragma unroll
            for (int s = 0; s < Rows<S>::QS; ++s) {
                const int d = S::SHARED ? 16 * s + 8 * g : 8 * S::NB * g + 8 * s;
                x.q[s] = u32x4{0, 0, 0, 0};
                if (live && d < D) x.q[s] = *(const u32x4*)(q + d);
            }
            int at = sq.len + a.tail - a.n + qi;     // the row's position
            if (a.mask) at = a.window && a.positions ? max(a.positions[qrow], sq.len) : sq.len;
            x.hi = a.mask ? sq.len - 1 : at;
            x.lo = a.window ? window_begin(at, a.window) : 0;
            x.mask = (uint32_t)qrow;
            if (live) {
                lo_most = max(lo_most, x.lo);
                hi_least = x.hi;
            } else {
                x.hi = -1;                           // (what it would attend may be any bytes)
            }
        }
        for (int o = 1; o < RL; o <<= 1) {
            lo_most = max(lo_most, __shfl_xor(lo_most, o));
            hi_least = min(hi_least, __shfl_xor(hi_least, o));
        }
        lo_most = uniform(lo_most);
        hi_least = uniform(hi_least);
        const int sinks = a.window ? a.sinks : 0;

        const Item it{uniform(b),         uniform(hk),       uniform(rb), sq,       span, uniform(begin_tile),
                      uniform(end_pages), uniform(end_tile), lo_most,     hi_least, sinks,
                      !uniform(__any(live))};
        bool careful = false;
        for (;;) {                                   // again where the tail is not finite
#pragma unroll
            for (int t = 0; t < S::EL / Rows<S>::VL; ++t) x.o[t] = 0.0f;
            x.m = -INFINITY;
            x.l = 0.0f;
            if constexpr (S::SHARED) {
                shared_tiles<T, S, false>(p, it, x, careful, s_lds);
                shared_tiles<T, S, true>(p, it, x, careful, s_lds);
            } else {
                own_tiles<T, S>(p, it, x, careful);
            }
            if (careful) break;
            // A value that is infinite or NaN has left none of its sums finite, a row's that
            // does not attend it (0 times it is NaN) neither: then once more without them.
            float z = 0.0f;
#pragma unroll
            for (int e = 0; e < S::EL; ++e) z = __fmaf_rn(x.at(e), 0.0f, z);
            careful = __syncthreads_or(live && !(z == 0.0f) && end_tile > end_pages) != 0;
            if (!careful) break;
        }

        // a row's lanes put together, and waves of the same rows
#pragma unroll
        for (int o = RL; o < 64; o <<= 1) x.l += __shfl_xor(x.l, o);
        if constexpr (!S::SHARED) {
            __syncthreads();                         // (the last item's have been read)
            if (g == 0) {
                s_ml[(wave * 16 + n) * 2] = x.m;
                s_ml[(wave * 16 + n) * 2 + 1] = x.l;
            }
            __syncthreads();
            float* out = (float*)s_lds;
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int k = 0; k < S::NW; ++k) m = fmaxf(m, s_ml[(k * 16 + n) * 2]);
            const float ref = ref_of<T>(m, to2);
#pragma unroll
            for (int k = 0; k < S::NW; ++k) {
                const float* ml = s_ml + (k * 16 + n) * 2;
                l += ml[1] * __builtin_amdgcn_exp2f((ml[0] * to2 - kRise<T>) - ref);
            }
            const float f = __builtin_amdgcn_exp2f((x.m * to2 - kRise<T>) - ref);
#pragma unroll
            for (int t = 0; t < S::EL / 4; ++t) {
                x.o[t] *= f;
                if (wave > 0)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        out[((wave - 1) * S::EL + 4 * t + r) * 64 + lane] = x.o[t][r];
            }
            x.m = m;
            x.l = l;
            __syncthreads();
            if (wave == 0)
#pragma unroll 1
                for (int k = 1; k < S::NW; ++k)
#pragma unroll
                    for (int t = 0; t < S::EL / 4; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            x.o[t][r] += out[((k - 1) * S::EL + 4 * t + r) * 64 + lane];
        }
        if (S::SHARED || wave == 0) {
            const bool whole = tile == 0 && end_place == span.length;
            if (whole) {
                if (live) {
                    const float inv = x.l == 0.0f ? 0.0f : 1.0f / x.l;
                    T* o = (T*)a.out + qrow * a.out_stride + (int64_t)qh * D;
#pragma unroll
                    for (int k = 0; k < S::NB; ++k) {
                        float f[S::EC];
#pragma unroll
                        for (int i = 0; i < S::EC; ++i) f[i] = x.at(k * S::EC + i) * inv;
                        store_chunk<T, S>(o, g, k, D, f);
                    }
                    if (a.lse && g == 0) a.lse[qrow * c.H + qh] = lse_of<T>(x.m, x.l, a.scale);
                    if (careful)
                        for (int k = 0; k < S::NB; ++k) add_unfinite<T, S>(p, b, hk, sq, qi, o, g, k);
                }
            } else {
                float* part = c.part + (int64_t)(2 * w + (first ? 0 : 1)) * S::PART;
#pragma unroll
                for (int e = 0; e < S::EL; ++e) part[(tile0 * S::EL + e) * 64 + lane] = x.at(e);
                if (g == 0) {
                    float* ml = part + S::ROWS * S::DP + (tile0 * RL + n) * 2;
                    ml[0] = x.m;
                    ml[1] = x.l;
                }
                if (tid == 0) ((int*)part)[S::PART - 1] = careful;
            }
        }
        // the next item
        left -= end_place - tile;
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
// stretch y describes, block x a chunk of its row tiles (x runs first, so an item's blocks
// spread over the chip's XCDs).  The four waves share the partial results and are added up
// in LDS.
constexpr int NTJ = 256, NWJ = 4;

template <typename T, typename S>
__global__ __launch_bounds__(NTJ) void k_packed_join(AttnArgs p) {
    constexpr int EC = S::EC, RL = S::RL;
    __shared__ float s_o[NWJ][EC][64], s_m[NWJ][RL], s_l[NWJ][RL];
    __shared__ int s_flag[NWJ];
    const int* desc = p.desc + 8 * blockIdx.y;
    const int n = desc[0];
    if (n == 0) return;
    const int slot0 = desc[1], b = desc[2], hk = desc[3], rb = desc[4];
    const int lane = threadIdx.x & 63, row = lane % RL, g = lane / RL;
    const int wave = uniform(threadIdx.x >> 6), rt = blockIdx.x / S::NB, ch = blockIdx.x % S::NB;
    const rheo_packed_attention_args& a = p.a;
    const CacheDev& c = p.c;
    const Seq sq = seq_of<S>(p, b);
    const int rows = sq.rows * p.g;
    if (rb * S::ROWS + rt * RL >= rows) return;
    const float to2 = a.scale * kLog2e;
    // (slot0 is the first stretch's, maybe its second; the others' first)
    const int w0 = slot0 >> 1, ml = S::ROWS * S::DP + (rt * RL + row) * 2;
    const int oi = (rt * S::EL + ch * EC) * 64 + lane;
    float m = -INFINITY, l = 0.0f, o[EC];
    int bad = 0;
#pragma unroll
    for (int e = 0; e < EC; ++e) o[e] = 0.0f;
#pragma unroll 1
    for (int k = wave; k < n; k += 2 * NWJ) {
        // two at a time (the second may be there twice, with weight 0)
        const bool both = k + NWJ < n;
        const int k1 = both ? k + NWJ : k;
        const float* q0 = c.part + (int64_t)(k ? 2 * (w0 + k) : slot0) * S::PART;
        const float* q1 = c.part + (int64_t)(k1 ? 2 * (w0 + k1) : slot0) * S::PART;
        float y0[EC], y1[EC];
#pragma unroll
        for (int e = 0; e < EC; ++e) {
            y0[e] = q0[oi + 64 * e];
            y1[e] = q1[oi + 64 * e];
        }
        const float m0 = q0[ml], l0 = q0[ml + 1], m1 = both ? q1[ml] : -INFINITY, l1 = q1[ml + 1];
        bad |= ((const int*)q0)[S::PART - 1] | ((const int*)q1)[S::PART - 1];
        const float top = fmaxf(m, fmaxf(m0, m1)), ref = ref_of<T>(top, to2);
        const float f = __builtin_amdgcn_exp2f((m * to2 - kRise<T>) - ref);
        const float f0 = __builtin_amdgcn_exp2f((m0 * to2 - kRise<T>) - ref);
        const float f1 = both ? __builtin_amdgcn_exp2f((m1 * to2 - kRise<T>) - ref) : 0.0f;
        m = top;
        l = __fmaf_rn(l0, f0, l * f);
        if (both) l = __fmaf_rn(l1, f1, l);
#pragma unroll
        for (int e = 0; e < EC; ++e) {
            o[e] = __fmaf_rn(y0[e], f0, o[e] * f);
            if (both) o[e] = __fmaf_rn(y1[e], f1, o[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < EC; ++e) s_o[wave][e][lane] = o[e];
    if (g == 0) {
        s_m[wave][row] = m;
        s_l[wave][row] = l;
    }
    if (lane == 0) s_flag[wave] = bad;
    __syncthreads();
    if (wave) return;
    m = -INFINITY;
    for (int k = 0; k < NWJ; ++k) m = fmaxf(m, s_m[k][row]);
    const float ref = ref_of<T>(m, to2);
    l = 0.0f;
    bad = 0;
#pragma unroll
    for (int e = 0; e < EC; ++e) o[e] = 0.0f;
    for (int k = 0; k < NWJ; ++k) {
        const float f = __builtin_amdgcn_exp2f((s_m[k][row] * to2 - kRise<T>) - ref);
        l = __fmaf_rn(s_l[k][row], f, l);
        bad |= s_flag[k];
#pragma unroll
        for (int e = 0; e < EC; ++e) o[e] = __fmaf_rn(s_o[k][e][lane], f, o[e]);
    }
    const int r = rb * S::ROWS + rt * RL + row;
    if (r >= rows) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int qi = r / p.g, qh = hk * p.g + r - qi * p.g;
    const int64_t qrow = (int64_t)b * a.n + qi;
    T* out = (T*)a.out + qrow * a.out_stride + (int64_t)qh * c.D;
#pragma unroll
    for (int e = 0; e < EC; ++e) o[e] *= inv;
    store_chunk<T, S>(out, g, ch, c.D, o);
    if (a.lse && g == 0 && ch == 0) a.lse[qrow * c.H + qh] = lse_of<T>(m, l, a.scale);
    if (bad) add_unfinite<T, S>(p, b, hk, sq, qi, out, g, ch);
}

namespace {

// Shapes for up to 16, 64, 128 and more rows of an item.  us a call for 32 sequences of 1024 to
// 4096 entries, 8 key heads of 128 (bytes at the copy's rate: 18), with
//         1    12    24    40    60   100   128   200   250 rows
//   R1   39    39    59    79    97   161   181   287   362
//   R4   63    61    62    64    64   103   103   178   192
//   R8   66    65    66    74    74    83    85   129   145
//  R16   90    90    90    92    94    98    99   118   136
// (R1, which takes such rows 16 at a time, would do for a few more than 16.)  Two row tiles a wave
// of own_tiles take 70 us at 24 rows (registers spill), 103 at 40.  Heads of more than 128
// elements leave registers for half the waves: 24 rows of 256 by two shared waves 174 us, by four
// 144 (bytes: 36; R1 127, but 177 for 149 at 40 rows); up to 16 rows of 256 by two waves a SIMD,
// which spill, 118, by one 73.
template <int NB>
struct Shapes {
    static constexpr bool W = NB > 4;
    typedef PShape<NB, false, 4, W ? 1 : 2> R1;
    typedef PShape<NB, true, W ? 4 : 2, W ? 1 : 2> R4;
    typedef PShape<NB, true, 4, W ? 1 : 2> R8;
    typedef PShape<NB, true, W ? 4 : 8, 1> R16;
};

template <typename S>
size_t part_floats(int units) {
    return (size_t)units * S::RES * 2 * S::PART;
}

template <int NB>
size_t workspace(int units) {
    typedef Shapes<NB> H;
    const size_t n[4] = {part_floats<typename H::R1>(units), part_floats<typename H::R4>(units),
                         part_floats<typename H::R8>(units), part_floats<typename H::R16>(units)};
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
    k_packed_attention<T, S><<<p.groups, S::NT, S::LDS, s>>>(p);
    k_packed_join<T, S><<<dim3(S::ROWS / S::RL * S::NB, p.groups), NTJ, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T, int NB>
hipError_t start_rows(const AttnArgs& p, hipStream_t s) {
    typedef Shapes<NB> H;
    const int64_t rows = (int64_t)p.a.n * p.g;
    if (rows <= 16) return start<T, typename H::R1>(p, s);
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
    if (e == hipSuccess) e = allow_lds<T, typename H::R4>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R8>();
    return e == hipSuccess ? allow_lds<T, typename H::R16>() : e;
}

template <int NB>
hipError_t prepare(int dtype) {
    return dtype == RHEO_BF16 ? prepare_rows<__bf16, NB>() : prepare_rows<_Float16, NB>();
}

template <int NB>
hipError_t launch(const CacheDev& c, const PackedDev& d, const rheo_packed_attention_args& a, int* desc,
                  hipStream_t s) {
    AttnArgs p{};
    p.c = c;
    p.p = d;
    p.a = a;
    p.g = c.H / c.K;
    p.desc = desc;
    return c.dtype == RHEO_BF16 ? start_rows<__bf16, NB>(p, s) : start_rows<_Float16, NB>(p, s);
}

template <int NB>
PackedHeads packed_heads() {
    return PackedHeads{prepare<NB>, workspace<NB>, launch<NB>};
}

}  // namespace

}  // namespace rheo
