// Attention of a drafted tree's rows over the paged cache (rheo_tree_attention).
//
// o_i = sum_j p_ij v_j with p = softmax_j(scale q_i.k_j), in one pass over the
// entries with a running maximum and sum.  The g = heads / kv_heads query heads
// of a key head read the same entries, so a sequence's rows and these heads
// together are the M = n * g rows of one product, and every entry is read
// once for up to 256 of them.
//
// Both products run on the matrix cores transposed, S^T = K Q^T and O^T = V^T
// P^T, as 32x32x16 tiles: a lane's S^T values all belong to one row (column
// lane % 32), so the softmax needs one exchange, between the two halves of the
// wave, and its result is the second product's right operand as it stands:
// lane h*32 + c holds S^T rows 8i + 4h + (0..3) of column c, and numbering the
// second product's inner index 8h + j <-> entry (j < 4 ? 4h + j : 4 + 4h + j)
// of each 16 makes those its values.  V^T comes from row-major V by LDS reads that
// transpose 4x16 blocks (ds_read_b64_tr_b16) in the same numbering.
//
// Work is cut by tiles, not by sequences: the tiles of all (sequence, key
// head, block of rows) items form one line, cut into equal stretches, one a
// workgroup.  So lengths may differ at will.  An item that a cut goes through
// leaves partial results (fp32, with maximum and sum), which k_attn_join
// adds up.
//
// What bounds it: few rows, memory: 128 single tokens over 8191 entries (4 key heads of
// 128, fp16, 1.34 GB) 260 us, 5.2 TB/s.  Up to 256 rows, the products and the softmax
// beside them: 64 trees of 244 rows over 1000 to 4096 entries (8 key heads, 0.79 GB,
// 176 GFLOP) 233 us, 755 TFLOP/s; the floor is 164, by the bytes.  There the loads alone
// take 180 us and the rest alone 218; a SIMD's two waves keep its matrix core busy for 178
// of 423 thousand cycles and its vector unit for 202 (an exponential is 16 cycles, the other
// operations 4), mostly one after the other: both waves pass a barrier at the top of each
// tile, so they do products together and then exponentials together.  No gain came from
// waves not kept in step, from products and exponentials of one wave and tile
// interleaved (10 to 20 us slower) and from one wave given priority.  Scores of the
// next tile computed beside this one's second product, and the two waves half a tile
// apart, are not tried.
#include <type_traits>

#include "cache_state.h"
#include "half_types.h"
#include "softmax_ref.h"

namespace rheo {

namespace {

// A launch's shape: DT head elements (head_dim padded), RT blocks of 32 rows
// and NW waves to a workgroup; NW / RT waves share the entries of a tile, U
// blocks of 32 of them each; P tiles are on their way while one is worked on.
template <int DT_, int RT_, int NW_, int U_, int P_>
struct Shape {
    static constexpr int DT = DT_, RT = RT_, NW = NW_, U = U_, P = P_;
    static constexpr int KW = NW / RT;               // waves to a row block
    static constexpr int KT = 32 * KW * U;           // entries of a tile
    static constexpr int ROWS = 32 * RT;
    static constexpr bool DEAL = ROWS >= 128;        // see deal_items
    static constexpr int NT = 64 * NW;
    static constexpr int KS = DT / 16, DB = DT / 32; // steps of QK, blocks of O's columns
    static constexpr int ROWB = DT * 2;              // bytes of an LDS row
    static constexpr int HALF = KT * ROWB;           // of a tile's K, and of its V
    static constexpr int J = HALF / (NW * 1024);     // loads of 1024 bytes of each a wave
    static constexpr int RPW = KT / NW;              // rows of each that a wave loads
    static constexpr int RPL = 1024 / ROWB;          // rows of a load
    static constexpr int RING = (P + 1) * 2 * HALF;
    static constexpr int PAGES = P * NW * 64 * 4;    // page numbers on their way
    static constexpr int LDS = RING + PAGES;
    static constexpr int RESIDENT = LDS <= 79 * 1024 && NW <= 4 ? 2 : 1;   // workgroups a unit
    static constexpr int WAVES = (RESIDENT * NW + 3) / 4;                  // waves a SIMD
    // a partial result: O^T as the lanes hold it, maximum and sum of each row, a flag
    static constexpr int PART = ROWS * DT + 2 * ROWS + 64;
    static_assert(HALF % (NW * 1024) == 0 && NW % RT == 0 && RPW <= 64, "shape");
    static_assert(KW == 1 || (NW - RT) * 64 * DB * 16 * 4 <= RING, "joining the waves in the ring");
    static_assert((P - 1) * (2 * J + 1) < 64 && P * (2 * J + 1) < 64, "loads in flight");
};

struct AttnArgs {
    CacheDev c;
    rheo_attention_args a;
    int g;                         // query heads of a key head
    int* desc;                     // [groups][8]: what k_attn_join adds up
    int groups;                    // most stretches (workgroups)
    int whole;                     // whole items may be given out (see deal_items)
};

// A sequence's part of the line.
struct Seq {
    int len, rows, tail, nrb;      // prefix, rows there, entries behind it, row blocks
    int entries;                   // len + tail
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
    if (s.len < 0 || s.len + (int64_t)s.tail > room) {
        if (s.rows) atomicOr(p.c.err, CE_TABLE);
        s.len = (int)min((int64_t)max(s.len, 0), room);
        s.tail = (int)min((int64_t)s.tail, room - s.len);
    }
    s.entries = s.len + s.tail;
    s.nrb = (s.rows * p.g + S::ROWS - 1) / S::ROWS;
    return s;
}

// Tiles of row block rb, at least one: without a mask no row attends past what
// its last row does.
template <typename S>
__device__ __forceinline__ int tiles_of(const AttnArgs& p, const Seq& s, int rb) {
    int end = s.entries;
    if (!p.a.mask) {
        const int last = min(((rb + 1) * S::ROWS - 1) / p.g, s.rows - 1);
        end = min(end, s.len + last + p.a.tail - p.a.n + 1);
    }
    return max((end + S::KT - 1) / S::KT, 1);
}

// ... of all row blocks, for one key head
template <typename S>
__device__ __forceinline__ int64_t tiles_of_head(const AttnArgs& p, const Seq& s) {
    if (p.a.mask) return (int64_t)s.nrb * tiles_of<S>(p, s, 0);
    int64_t t = 0;
    for (int rb = 0; rb < s.nrb; ++rb) t += tiles_of<S>(p, s, rb);
    return t;
}

// What is the same in all lanes, said so: it then takes scalar registers.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
__device__ __forceinline__ Seq uniform(const Seq& s) {
    return Seq{uniform(s.len), uniform(s.rows), uniform(s.tail), uniform(s.nrb), uniform(s.entries)};
}

// Stretch w of the line: tiles [t0, t1) of it, the sequence that t0 is in and
// the tiles before that sequence.  All threads of the block call it.
struct Stretch {
    int64_t total, t0, t1, before;
    int groups, seq;
};

__device__ __forceinline__ int64_t stretch_start(int64_t total, int groups, int w) {
    return total * w / groups;
}

template <typename S>
__device__ Stretch find_stretch(const AttnArgs& p, int w) {
    __shared__ int64_t s_wave[S::NW], s_before;
    __shared__ int s_seq;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = p.c.B;
    const int per = (B + S::NT - 1) / S::NT, b0 = min(tid * per, B), b1 = min(b0 + per, B);
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
    for (int v = 0; v < S::NW; ++v) {
        if (v < wave) excl += s_wave[v];
        total += s_wave[v];
    }
    total = uniform64(total);
    Stretch r;
    r.total = total;
    r.groups = (int)(total < p.groups ? total : p.groups);
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

// Whole items dealt out instead of stretches, where that is nearly as even: the
// sequences sorted by length, their items given to the workgroups in order, there and
// back (the longest with the shortest).  A cut costs the partial results' way out and
// back, as long as some four tiles of 256 rows each, and the join: 64 trees of 244
// rows over 1000 to 4096 entries 271 us in stretches, 237 dealt.  (Partial results
// of 64 rows and fewer are too small for that: 3 % slower.)  All threads call it;
// at most kDealt sequences, an item a key head each: every workgroup ranks all sequences
// by counting, and their order is in LDS.  More are cut (256 sequences of 500 to 2000
// entries, 61 rows, 32/8 heads, 504 us; 257 560).
constexpr int kDealt = 256;

__device__ __forceinline__ int dealt_item(int round, int w, int groups) {
    return round * groups + (round & 1 ? groups - 1 - w : w);
}

template <typename S>
__device__ bool deal_items(const AttnArgs& p, int64_t total, int* s_order) {
    __shared__ int s_tiles[kDealt], s_most[S::NW];
    const int tid = threadIdx.x, B = p.c.B, K = p.c.K, items = B * K;
    __syncthreads();
    for (int b = tid; b < B; b += S::NT) {
        const Seq s = seq_of<S>(p, b);
        s_tiles[b] = s.nrb ? tiles_of<S>(p, s, 0) : 0;
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
    return most <= mean + mean / 16 + 4;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lds_s4;

template <typename T>
__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, const f32x16& c) {
    typedef typename Pack<T>::v8 v8;
    if constexpr (std::is_same<T, __bf16>::value)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
}

// Loads from global memory straight into LDS, 16 or 4 bytes a lane, the lanes'
// next to each other from `lds` on.  They are in flight until wait_loads; the
// compiler does not know of them, which only makes its own waits longer.  (Its
// builtin would make every LDS read wait for all of them.)  No register is
// written but m0, which nothing else here uses (the compiler reserves it).
__device__ __forceinline__ void load_lds16(uint32_t lds, const void* p) {
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p)
                 : "memory");
}
__device__ __forceinline__ void load_lds4(uint32_t lds, const void* p) {
    lds = __builtin_amdgcn_readfirstlane(lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(p)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// The 16-byte vectors of an LDS row lie in another order, so that reads of one
// column hit different banks: vector c of row r at place c ^ k_turn(r) for K (16
// rows, one vector each), c ^ v_turn(r) for V (4 rows, four vectors each).
template <int DT>
__device__ __forceinline__ int k_turn(int r) { return DT == 64 ? (r >> 1) & 7 : r & 15; }
template <int DT>
__device__ __forceinline__ int v_turn(int r) { return DT == 64 ? (r << 1) & 4 : (r << 2) & 12; }

// A value of the lane's own and of the other half's lane of the same column.
__device__ __forceinline__ f32x2 both_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// Elements that are infinite or NaN made 0; whether there was one.
template <typename T>
__device__ __forceinline__ bool drop_unfinite(uint4& v) {
    constexpr uint32_t E = Pack<T>::kExp;
    bool bad = false;
    uint32_t* w = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool lo = (w[i] & E) == E, hi = (w[i] & E << 16) == E << 16;
        w[i] = (lo ? 0 : w[i] & 0xFFFFu) | (hi ? 0 : w[i] & 0xFFFF0000u);
        bad |= lo | hi;
    }
    return bad;
}

// The infinite and NaN values of entries behind the prefix, which the products
// left out, added to an output row that attends them: `at` and the three
// elements behind it of each of the lane's fours, 8 apart.  Their
// probabilities are not 0, so the values themselves decide.  Rare and slow; by the
// lanes that wrote the row.
template <typename T>
__device__ __forceinline__ void add_unfinite(const AttnArgs& p, int b, int hk, const Seq& sq, int qi,
                                             T* out, int at, int step) {
    const CacheDev& c = p.c;
    const int64_t qrow = (int64_t)b * p.a.n + qi;
#pragma unroll 1
    for (int j = 0; j < sq.tail; ++j) {
        const bool seen = p.a.mask ? p.a.mask[qrow * p.a.tail + j] != 0 : j <= qi + p.a.tail - p.a.n;
        if (!seen) continue;
        const int e = sq.len + j;
        int page = p.a.table[(int64_t)b * c.width + (e >> c.page_shift)];
        page = min(max(page, 0), c.pages - 1);
        const T* v = (const T*)p.a.v_cache + page * c.page_stride +
                     ((int64_t)(e & ((1 << c.page_shift) - 1)) * c.K + hk) * c.D;
#pragma unroll 1
        for (int d = at; d < c.D; d += step)
#pragma unroll 1
            for (int i = d; i < d + 4; ++i) {
                const float x = (float)v[i];
                if (!(fabsf(x) < INFINITY)) out[i] = (T)((float)out[i] + x);
            }
    }
}

// What a row block's waves hold while they go through an item's tiles.
template <typename S>
struct Rows {
    u32x4 q[S::KS];                // Q^T: the lane's row, elements 16s + 8h + (0..7)
    f32x16 o[S::DB];               // O^T: row, elements 32db + 8(r/4) + 4h + r%4
    float m, l;                    // the exponents' reference, a score; its half's sum
};

}  // namespace

template <typename T, typename S>
__global__ __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(S::WAVES, S::WAVES))) void
k_tree_attention(AttnArgs p) {
    extern __shared__ __align__(1024) char s_lds[];
    __shared__ float s_ml[S::KW > 1 ? S::NW * 64 : 2];
    __shared__ int s_bad;                            // values left out of the item's products
    __shared__ int s_order[S::DEAL ? kDealt : 1];    // sequences, the longest first
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rt = wave % S::RT, kw = wave / S::RT;
    const CacheDev& c = p.c;
    const rheo_attention_args& a = p.a;
    const int w = blockIdx.x, D = c.D;
    const float to2 = a.scale * kLog2e;              // scores to exponents of 2
    const float slack = kSlack<T> / to2;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_lds;
    const uint32_t lds_mine = __builtin_amdgcn_readfirstlane(lds0 + wave * (S::J * 1024));
    const uint32_t lds_pages = __builtin_amdgcn_readfirstlane(lds0 + S::RING + wave * 256);
    const int* const pages = (const int*)(s_lds + S::RING + wave * 256);
    // byte offsets in their rows of the lane's K vector for s = 0 and its part of a
    // 4x16 block of V for d = 0 (others: exclusive or of 32 s, 64 d)
    const int k_at = (half ^ k_turn<S::DT>(col)) * 16;
    const int v_at = ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ v_turn<S::DT>((lane & 15) / 4)) * 16 +
                     (lane & 1) * 8;
    if (tid == 0) s_bad = 0;

    Stretch st = find_stretch<S>(p, w);
    bool dealt = false;
    if constexpr (S::DEAL)
        if (p.whole && st.groups == p.groups)
            dealt = uniform(deal_items<S>(p, st.total, s_order)) != 0;
    if (!dealt && st.t0 >= st.t1) {
        if (tid == 0) p.desc[8 * w] = 0;
        return;
    }
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
                left = tiles_of<S>(p, sq, 0);
                ++round;
                return true;
            }
        }
        return false;
    };
    if (tid == 0) p.desc[8 * w] = 0;
    if (dealt) {
        if (!next_dealt()) return;
    } else {
        b = st.seq;
        sq = uniform(seq_of<S>(p, b));
        int64_t rel = st.t0 - st.before;
        const int64_t per_head = tiles_of_head<S>(p, sq);
        hk = uniform((int)(rel / per_head));
        rel -= hk * per_head;
        while (rel >= tiles_of<S>(p, sq, rb)) rel -= tiles_of<S>(p, sq, rb++);
        tile = (int)rel;
        left = st.t1 - st.t0;
        // the join of the first item, by the first cut inside it
        const int64_t begins = st.t0 - tile, ends = begins + tiles_of<S>(p, sq, rb);
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
        const int tiles = tiles_of<S>(p, sq, rb);
        const int end_tile = (int)min((int64_t)tiles, tile + left);
        const int32_t* row_table = a.table + (int64_t)b * c.width;
        const int entries = sq.entries, len = sq.len;
        const T* const k_head = (const T*)a.k_cache + (int64_t)hk * D;
        const T* const v_head = (const T*)a.v_cache + (int64_t)hk * D;

        // Tile t's page numbers, those of the rows that the wave loads; then its
        // entries.  (Rows past the last entry and vectors past the head's last
        // load the last one's again.)
        auto fetch_pages = [&](int t) {
            const int e = t * S::KT + wave * S::RPW + min(lane, S::RPW - 1);
            load_lds4(lds_pages + t % S::P * (S::NW * 256),
                      row_table + (min(e, entries - 1) >> c.page_shift));
        };
        auto fetch = [&](int t) {
            const uint32_t to = lds_mine + t % (S::P + 1) * (2 * S::HALF);
            const int in_page = (1 << c.page_shift) - 1;
#pragma unroll
            for (int j = 0; j < S::J; ++j) {
                const int sub = j * S::RPL + lane * 16 / S::ROWB, row = wave * S::RPW + sub;
                const int place = lane * 16 % S::ROWB / 16;
                int page = pages[t % S::P * (S::NW * 64) + sub];
                if ((unsigned)page >= (unsigned)c.pages) {
                    atomicOr(c.err, CE_PAGE);
                    page = 0;
                }
                const int e = min(t * S::KT + row, entries - 1);
                const int64_t at = page * c.page_stride + (e & in_page) * (c.K * D);
                load_lds16(to + j * 1024, k_head + at + min(place ^ k_turn<S::DT>(row), D / 8 - 1) * 8);
                load_lds16(to + S::HALF + j * 1024,
                           v_head + at + min(place ^ v_turn<S::DT>(row), D / 8 - 1) * 8);
            }
        };
        Rows<S> x;
        const int r = rb * S::ROWS + rt * 32 + col;  // the lane's row of the item
        const bool live = r < sq.rows * p.g;
        const int qi = live ? r / p.g : 0, qh = hk * p.g + (live ? r - qi * p.g : 0);
        const int64_t qrow = (int64_t)b * a.n + qi;
        {
            const T* q = (const T*)a.q + qrow * a.q_stride + (int64_t)qh * D;
#pragma unroll
            for (int s = 0; s < S::KS; ++s) {
                const int d = 16 * s + 8 * half;
                x.q[s] = u32x4{0, 0, 0, 0};
                if (live && d < D) x.q[s] = *(const u32x4*)(q + d);
            }
        }
        __syncthreads();                             // the ring is free
        if (entries > 0) {
#pragma unroll
            for (int i = 0; i < S::P; ++i)
                if (tile + i < end_tile) fetch_pages(tile + i);
        }
        wait_loads<0>();
        // (q is here, too: said so that no wait for it stands in the loop)
#pragma unroll
        for (int s = 0; s < S::KS; ++s) asm volatile("" : "+v"(x.q[s]));
        if (entries > 0) {
#pragma unroll
            for (int i = 0; i < S::P; ++i) {
                if (tile + i < end_tile) fetch(tile + i);
                if (tile + i + S::P < end_tile) fetch_pages(tile + i + S::P);
            }
        }

#pragma unroll
        for (int d = 0; d < S::DB; ++d) x.o[d] = 0.0f;
        x.m = -INFINITY;
        x.l = 0.0f;
        const uint8_t* mrow = a.mask ? a.mask + qrow * a.tail : nullptr;
        const int reach = qi + a.tail - a.n;         // without a mask: tail entries seen, less 1

        for (int t = tile; t < end_tile && entries > 0; ++t) {
            // Loads come in in order, so tile t's and the page numbers of tile t + P are
            // there when no more are out than were sent after them
            {
                const int rd = min(S::P - 1, end_tile - 1 - t);
                if (end_tile - 1 - t - S::P >= S::P - 1) wait_loads<(S::P - 1) * (2 * S::J + 1)>();
                else if (S::P > 2 && rd == 2) wait_loads<(S::P > 2 ? 2 : 0) * 2 * S::J>();
                else if (S::P > 1 && rd == 1) wait_loads<(S::P > 1 ? 1 : 0) * 2 * S::J>();
                else wait_loads<0>();
            }
            char* const s_k = s_lds + t % (S::P + 1) * (2 * S::HALF);
            char* const s_v = s_k + S::HALF;
            const bool tail_tile = (t + 1) * S::KT > len;
            if (tail_tile) {
                // An entry that some row does not attend must not reach it: 0 * inf
                // is not 0.  Such values become zeros and are added at the end.
#pragma unroll
                for (int j = 0; j < S::J; ++j) {
                    const int e = t * S::KT + wave * S::RPW + j * S::RPL + lane * 16 / S::ROWB;
                    if (e >= len) {
                        uint4* v = (uint4*)(s_v + (wave * S::J + j) * 1024 + lane * 16);
                        uint4 x = *v;
                        const bool bad = drop_unfinite<T>(x);
                        if (e >= entries) x = make_uint4(0, 0, 0, 0);
                        else if (bad) s_bad = 1;
                        *v = x;
                    }
                }
            }
            // (with one row block a wave works on the rows it has loaded itself)
            if (S::RT > 1) __syncthreads();

            // S^T of the wave's U blocks of 32 entries
            const int e0 = kw * S::U * 32;           // (of the tile)
            f32x16 sc[S::U];
#pragma unroll
            for (int u = 0; u < S::U; ++u) sc[u] = 0.0f;
            const char* const kp = s_k + (e0 + col) * S::ROWB;
#pragma unroll
            for (int s = 0; s < S::KS; ++s)
#pragma unroll
                for (int u = 0; u < S::U; ++u)
                    sc[u] = mfma<T>(*(const u32x4*)(kp + (k_at ^ s * 32) + u * 32 * S::ROWB), x.q[s],
                                    sc[u]);
            // six reads ahead of the products
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int i = 0; i < S::KS * S::U - 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
            // (the products are under way: time for the loads' addresses)
            if (t + S::P < end_tile) fetch(t + S::P);
            if (t + 2 * S::P < end_tile) fetch_pages(t + 2 * S::P);
            if (tail_tile) {
                const int eh = t * S::KT + e0 + 4 * half;
                if (mrow && sq.tail > 0) {
#pragma unroll
                    for (int u = 0; u < S::U; ++u) {
                        uint8_t named[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            named[i] = mrow[min(max(eh + u * 32 + 8 * (i / 4) + i % 4 - len, 0),
                                                sq.tail - 1)];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int e = eh + u * 32 + 8 * (i / 4) + i % 4;
                            const bool seen = (e < len) | ((e < entries) & (named[i] != 0));
                            sc[u][i] = seen ? sc[u][i] : -INFINITY;
                        }
                    }
                } else {
                    const int end = mrow ? entries : min(len + reach + 1, entries);
#pragma unroll
                    for (int u = 0; u < S::U; ++u)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sc[u][i] = eh + u * 32 + 8 * (i / 4) + i % 4 < end ? sc[u][i] : -INFINITY;
                }
            }
            // The exponents' reference follows the row's maximum by steps (kSlack): what holds
            // the probabilities takes them, and O is rescaled once or twice an item instead
            // of at most tiles (some row of 32 has a new maximum).
            float mx = sc[0][0];
#pragma unroll
            for (int u = 0; u < S::U; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
            const f32x2 mb = both_halves(mx);
            const float m = fmaxf(x.m, fmaxf(mb[0], mb[1]));
            const bool up = m > x.m + slack;
            if (__any(up)) {
                // (both references as the exponents have them, rounded; a row whose own
                // maximum has not risen so far keeps its reference, so that what other rows
                // attend does not show in its roundings)
                const float f =
                    up ? __builtin_amdgcn_exp2f((x.m * to2 - kRise<T>) - ref_of<T>(m, to2)) : 1.0f;
                x.l *= f;
#pragma unroll
                for (int d = 0; d < S::DB; ++d) x.o[d] *= f;
                x.m = up ? m : x.m;
            }
            const float ref = ref_of<T>(x.m, to2);
            float sum = 0.0f;
#pragma unroll
            for (int u = 0; u < S::U; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[u][i] = __builtin_amdgcn_exp2f(__fmaf_rn(sc[u][i], to2, -ref));
                    sum += sc[u][i];
                }
            x.l += sum;
            // O^T += V^T P^T.  The matrix cores take the probabilities in the cache's 16 bits;
            // the sum of the denominator has them unrounded.  That is a choice: rounding them
            // is off by as much again as rounding the output (single bf16 tokens over 4096
            // entries: 2.30e-3 of the norm, 1.66e-3 by the output's rounding alone).  A
            // second product with what the rounding left over takes that away, but it
            // costs 95 us for 91 at 40 rows, 129 for 118 at 100, 295 for 242 at 244 (under
            // 1 % up to 32 rows, where memory is the bound), and what is left over may be 0
            // or negative, where an infinite value would make NaN of an infinite output.
#pragma unroll
            for (int u = 0; u < S::U; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    u32x4 pt;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        pt[i] = pack2<T>(sc[u][8 * k + 2 * i], sc[u][8 * k + 2 * i + 1]);
                    const char* vp = s_v + (e0 + u * 32 + 16 * k + 4 * half + (lane & 15) / 4) * S::ROWB;
#pragma unroll
                    for (int d = 0; d < S::DB; ++d) {
                        const char* vd = vp + (v_at ^ d * 64);
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)vd);
                        const s16x4 hi =
                            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(vd + 8 * S::ROWB));
                        const s16x8 va = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        x.o[d] = mfma<T>(__builtin_bit_cast(u32x4, va), pt, x.o[d]);
                    }
                }
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
            for (int i = 0; i < S::DB * S::U * 2 - 4; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 1);
        }

        // the waves of a row block put together
        const f32x2 lb = both_halves(x.l);
        x.l = lb[0] + lb[1];
        if constexpr (S::KW > 1) {
            if (!half) {
                s_ml[(wave * 32 + col) * 2] = x.m;
                s_ml[(wave * 32 + col) * 2 + 1] = x.l;
            }
            __syncthreads();
            float m = -INFINITY, l = 0.0f;
#pragma unroll
            for (int k = 0; k < S::KW; ++k) m = fmaxf(m, s_ml[((k * S::RT + rt) * 32 + col) * 2]);
            const float ref = ref_of<T>(m, to2);
#pragma unroll
            for (int k = 0; k < S::KW; ++k) {
                const float* ml = s_ml + ((k * S::RT + rt) * 32 + col) * 2;
                l += ml[1] * __builtin_amdgcn_exp2f((ml[0] * to2 - kRise<T>) - ref);
            }
            const float f = __builtin_amdgcn_exp2f((x.m * to2 - kRise<T>) - ref);
            float* out = (float*)s_lds;
#pragma unroll
            for (int d = 0; d < S::DB; ++d) {
                x.o[d] *= f;
                if (kw > 0)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        out[(((wave - S::RT) * S::DB + d) * 16 + i) * 64 + lane] = x.o[d][i];
            }
            __syncthreads();
            if (kw == 0)
#pragma unroll 1
                for (int k = 1; k < S::KW; ++k)
#pragma unroll
                    for (int d = 0; d < S::DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            x.o[d][i] += out[((((k - 1) * S::RT + rt) * S::DB + d) * 16 + i) * 64 + lane];
            x.m = m;
            x.l = l;
        }
        const int bad = s_bad;
        __syncthreads();
        if (tid == 0) s_bad = 0;
        if (kw == 0) {
            if (tile == 0 && end_tile == tiles) {
                const float inv = x.l == 0.0f ? 0.0f : 1.0f / x.l;
                T* o = (T*)a.out + qrow * a.out_stride + (int64_t)qh * D;
                if (live) {
#pragma unroll
                    for (int d = 0; d < S::DB; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int at = 32 * d + 8 * i + 4 * half;
                            if (at < D)
                                *(uint2*)(o + at) = make_uint2(
                                    pack2<T>(x.o[d][4 * i] * inv, x.o[d][4 * i + 1] * inv),
                                    pack2<T>(x.o[d][4 * i + 2] * inv, x.o[d][4 * i + 3] * inv));
                        }
                    if (a.lse && !half) a.lse[qrow * c.H + qh] = lse_of<T>(x.m, x.l, a.scale);
                    if (bad) add_unfinite<T>(p, b, hk, sq, qi, o, 4 * half, 8);
                }
            } else {
                float* part = c.part + (int64_t)(2 * w + (first ? 0 : 1)) * S::PART;
#pragma unroll
                for (int d = 0; d < S::DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        part[((rt * S::DB + d) * 16 + i) * 64 + lane] = x.o[d][i];
                if (!half) {
                    float* ml = part + S::ROWS * S::DT + (rt * 32 + col) * 2;
                    ml[0] = x.m;
                    ml[1] = x.l;
                }
                if (tid == 0) ((int*)part)[S::PART - 1] = bad;
            }
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

// The partial results of one cut item added up: block y of a launch has the item
// that stretch y describes (see k_tree_attention), block x its 32 rows and WD
// blocks of 32 elements, one of them a wave.  (x runs first, so an item's blocks
// spread over the chip's XCDs; with y first, items cut 32 times all fell to one:
// 57 us instead of 13.)  8 / WD waves share the partial
// results of each and are added up in turn.
constexpr int NTJ = 512;

template <typename T, typename S, int WD>
__global__ __launch_bounds__(NTJ) void k_attn_join(AttnArgs p) {
    constexpr int NS = NTJ / 64 / WD;
    __shared__ float s_o[NS][WD][16][64], s_m[NS][32], s_l[NS][32];
    __shared__ int s_flag[NS];
    const int* desc = p.desc + 8 * blockIdx.y;
    const int n = desc[0];
    if (n == 0) return;
    const int slot0 = desc[1], b = desc[2], hk = desc[3], rb = desc[4];
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = threadIdx.x >> 6, wd = wave % WD, part0 = wave / WD;
    const int rt = blockIdx.x / (S::DB / WD), d0 = blockIdx.x % (S::DB / WD) * WD, d = d0 + wd;
    const rheo_attention_args& a = p.a;
    const CacheDev& c = p.c;
    const Seq sq = seq_of<S>(p, b);
    const int rows = sq.rows * p.g;
    if (rb * S::ROWS + rt * 32 >= rows || 32 * d0 >= c.D) return;
    const float to2 = a.scale * kLog2e;
    // (slot0 is the first stretch's, maybe its second; the others' first)
    const int w0 = slot0 >> 1, ml = S::ROWS * S::DT + (rt * 32 + col) * 2;
    const int oi = (rt * S::DB + d) * 16 * 64 + lane;
    float m = -INFINITY, l = 0.0f, o[16];
    int bad = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = 0.0f;
    const int last = n - 1;
    for (int k = part0; k < n; k += 2 * NS) {
        // two at a time (the second may be there twice, with weight 0)
        const int k1 = min(k + NS, last);
        const float* q0 = c.part + (int64_t)(k ? 2 * (w0 + k) : slot0) * S::PART;
        const float* q1 = c.part + (int64_t)(k1 ? 2 * (w0 + k1) : slot0) * S::PART;
        float x0[16], x1[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x0[e] = q0[oi + 64 * e];
            x1[e] = q1[oi + 64 * e];
        }
        const float m0 = q0[ml], l0 = q0[ml + 1];
        const float m1 = k + NS < n ? q1[ml] : -INFINITY, l1 = q1[ml + 1];
        bad |= ((const int*)q0)[S::PART - 1] | ((const int*)q1)[S::PART - 1];
        const float top = fmaxf(m, fmaxf(m0, m1)), ref = ref_of<T>(top, to2);
        const float f = __builtin_amdgcn_exp2f((m * to2 - kRise<T>) - ref);
        const float g0 = __builtin_amdgcn_exp2f((m0 * to2 - kRise<T>) - ref);
        const float g1 = __builtin_amdgcn_exp2f((m1 * to2 - kRise<T>) - ref);
        m = top;
        l = l * f + l0 * g0;
        if (k + NS < n) l = __fmaf_rn(l1, g1, l);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            o[e] = __fmaf_rn(x0[e], g0, o[e] * f);
            if (k + NS < n) o[e] = __fmaf_rn(x1[e], g1, o[e]);
        }
    }
    if (part0 < n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s_o[part0][wd][e][lane] = o[e];
        if (wd == 0) {
            if (!half) {
                s_m[part0][col] = m;
                s_l[part0][col] = l;
            }
            if (lane == 0) s_flag[part0] = bad;
        }
    }
    __syncthreads();
    const int parts = min(n, NS), r = rb * S::ROWS + rt * 32 + col;
    m = -INFINITY;
    for (int k = 0; k < parts; ++k) m = fmaxf(m, s_m[k][col]);
    const float ref = ref_of<T>(m, to2);
    l = 0.0f;
    bad = 0;
    for (int k = 0; k < parts; ++k) {
        l = __fmaf_rn(s_l[k][col], __builtin_amdgcn_exp2f((s_m[k][col] * to2 - kRise<T>) - ref), l);
        bad |= s_flag[k];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int qi = r / p.g, qh = hk * p.g + r - qi * p.g;
    const int64_t qrow = (int64_t)b * a.n + qi;
    T* out = (T*)a.out + qrow * a.out_stride + (int64_t)qh * c.D;
    // four elements a lane and turn: registers 4i .. 4i + 3 of a block of 32
    for (int f = wave; f < 4 * WD; f += NTJ / 64) {
        const int i = f % 4, at = 32 * (d0 + f / 4) + 8 * i + 4 * half;
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < parts; ++k) {
            const float g = __builtin_amdgcn_exp2f((s_m[k][col] * to2 - kRise<T>) - ref);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = __fmaf_rn(s_o[k][f / 4][4 * i + e][lane], g, x[e]);
        }
        if (r >= rows || at >= c.D) continue;
        *(uint2*)(out + at) =
            make_uint2(pack2<T>(x[0] * inv, x[1] * inv), pack2<T>(x[2] * inv, x[3] * inv));
        if (a.lse && at == 0) a.lse[qrow * c.H + qh] = lse_of<T>(m, l, a.scale);
        if (bad) add_unfinite<T>(p, b, hk, sq, qi, out, at, c.D);
    }
}

namespace {

// Shapes for up to 32, 64, 128 and more rows of an item: for 128 elements the fastest of
// those that fit, of two or three tried each.  Few rows are bound by memory, and the
// waves of a workgroup share the entries; many by the products and the vector work
// between them.  us for 32 sequences of 1024 to 4096 entries, 8 key heads (bytes at the
// copy's rate: 34, 68, 135 for 64, 128, 256 elements), with
//                 4 rows   40 rows   100 rows   244 rows
//   64 elements     49       59        68         114      (the shapes of 128, no others tried)
//   128             85       90       119         161
//   256            197      205       208         390
// Of 128, 4 rows by two waves and three tiles ahead took 1.05 times as long, 40 rows by
// eight waves 1.4 times and with one tile ahead 1.28, 100 rows by eight waves 1.14.  The
// kernel for up to 64 rows of 256 elements spills 22 vector registers, most of it
// between items.
template <int DT>
struct Shapes;
template <>
struct Shapes<64> {
    typedef Shape<64, 1, 4, 1, 1> R1;
    typedef Shape<64, 2, 4, 1, 3> R2;
    typedef Shape<64, 4, 4, 2, 3> R4;
    typedef Shape<64, 8, 8, 2, 3> R8;
};
template <>
struct Shapes<128> {
    typedef Shape<128, 1, 4, 1, 1> R1;
    typedef Shape<128, 2, 4, 1, 3> R2;
    typedef Shape<128, 4, 4, 2, 3> R4;
    typedef Shape<128, 8, 8, 2, 3> R8;
};
template <>
struct Shapes<256> {
    typedef Shape<256, 2, 2, 1, 3> R2;
    typedef R2 R1;                 // (two waves on 32 rows, one tile ahead: 168 us for 120)
    typedef Shape<256, 4, 4, 1, 3> R4;
    typedef R4 R8;                 // (256 rows of 256 do not fit the registers)
};

template <typename S>
size_t part_floats(int units) {
    return (size_t)units * S::RESIDENT * 2 * S::PART;
}

template <int DT>
size_t workspace(int units) {
    typedef Shapes<DT> H;
    size_t n = part_floats<typename H::R1>(units);
    const size_t r2 = part_floats<typename H::R2>(units), r4 = part_floats<typename H::R4>(units),
                 r8 = part_floats<typename H::R8>(units);
    n = n > r2 ? n : r2;
    n = n > r4 ? n : r4;
    return n > r8 ? n : r8;
}

template <typename T, typename S>
hipError_t start(AttnArgs p, hipStream_t s) {
    static_assert(S::LDS <= 156 * 1024, "LDS");
    p.groups = p.c.slots * S::RESIDENT;
    // (fewer items than workgroups: the cuts are what fills them)
    p.whole = (int64_t)p.a.n * p.g <= S::ROWS && p.c.B <= kDealt &&
              (int64_t)p.c.B * p.c.K >= p.groups;
    k_tree_attention<T, S><<<p.groups, S::NT, S::LDS, s>>>(p);
    // Items that are cut once or twice take a wave a block of 32 elements (255 of them
    // 24 us; eight waves each 52), those of which many stretches have a part eight
    // waves (eight items of 32 parts 12 us; 19 with two)
    constexpr int WD = S::DB < 4 ? S::DB : 4;
    const int64_t items = (int64_t)p.c.B * p.c.K * (((int64_t)p.a.n * p.g + S::ROWS - 1) / S::ROWS);
    if (items * 4 >= p.groups)
        k_attn_join<T, S, WD><<<dim3(S::RT * (S::DB / WD), p.groups), NTJ, 0, s>>>(p);
    else
        k_attn_join<T, S, 1><<<dim3(S::RT * S::DB, p.groups), NTJ, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T, int DT>
hipError_t start_rows(const AttnArgs& p, hipStream_t s) {
    typedef Shapes<DT> H;
    const int64_t rows = (int64_t)p.a.n * p.g;
    if (rows <= 32) return start<T, typename H::R1>(p, s);
    if (rows <= 64) return start<T, typename H::R2>(p, s);
    if (rows <= 128 || DT > 128) return start<T, typename H::R4>(p, s);
    return start<T, typename H::R8>(p, s);
}

template <typename T>
hipError_t start_dim(const AttnArgs& p, hipStream_t s) {
    if (p.c.D <= 64) return start_rows<T, 64>(p, s);
    if (p.c.D <= 128) return start_rows<T, 128>(p, s);
    return start_rows<T, 256>(p, s);
}

template <typename T, typename S>
hipError_t allow_lds() {
    return hipFuncSetAttribute((const void*)k_tree_attention<T, S>,
                               hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
}

template <typename T, int DT>
hipError_t prepare_dim() {
    typedef Shapes<DT> H;
    hipError_t e = allow_lds<T, typename H::R1>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R2>();
    if (e == hipSuccess) e = allow_lds<T, typename H::R4>();
    return e == hipSuccess ? allow_lds<T, typename H::R8>() : e;
}

template <typename T>
hipError_t prepare_type(int D) {
    return D <= 64 ? prepare_dim<T, 64>() : D <= 128 ? prepare_dim<T, 128>() : prepare_dim<T, 256>();
}

}  // namespace

hipError_t prepare_attention(const CacheDev& c) {
    return c.dtype == RHEO_BF16 ? prepare_type<__bf16>(c.D) : prepare_type<_Float16>(c.D);
}

size_t attention_workspace(const CacheDev& c) {
    const size_t n = c.D <= 64 ? workspace<64>(c.slots) : c.D <= 128 ? workspace<128>(c.slots)
                                                                     : workspace<256>(c.slots);
    return n + (size_t)c.slots * 2 * 8;      // and the descriptions of the joins
}

hipError_t launch_tree_attention(const CacheDev& c, const rheo_attention_args& a, hipStream_t s) {
    AttnArgs p{};
    p.c = c;
    p.a = a;
    p.g = c.H / c.K;
    p.desc = (int*)(c.part + attention_workspace(c) - (size_t)c.slots * 2 * 8);
    return c.dtype == RHEO_BF16 ? start_dim<__bf16>(p, s) : start_dim<_Float16>(p, s);
}

}  // namespace rheo
