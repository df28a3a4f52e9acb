// Head norms, position rotation and the store into the pages (rheo_cache_write).
#include "cache_state.h"
#include "half_types.h"

namespace rheo {

namespace {

constexpr int NTW = 256;

// How a head's rotated pairs lie in its vectors of eight elements
enum Pairs { NONE = 0, HALVES = 1, NEIGHBOURS = 2, ODD_HALVES = 3 };

}  // namespace

// A head x becomes x / sqrt(mean(x^2) + eps) * w, and its pairs (a, b) become
// (a cos - b sin, b cos + a sin).  LPH lanes hold a head, 16 elements each as
// two 16-byte vectors: with pairs (j, j + rot/2) one vector of the first half
// and the one rot/2 behind it, so that both of a pair are in one lane and only
// the sum of squares crosses lanes; the elements behind rot_dim and heads of
// neighbouring pairs take vectors 2t and 2t+1.  (rot/2 no multiple of 8,
// ODD_HALVES: partners are loaded element by element.)
//
// Reading q, k and v and writing them once is all there is: 2 bytes an
// element each way against some 6 operations.  A group of LPH lanes takes
// a token's heads one after another, with its cosines and sines in registers
// (the table's row, 4 bytes an element, is as long as two heads) and the next head's
// vectors on their way: 5200 rows of 120 heads (316 MB) 65 us, 4.9 TB/s, what a large
// copy reaches; without the head ahead 114 us.  61 rows: 4.2 us, launch and latency.
template <typename T, int LPH, int MODE>
__global__ __launch_bounds__(NTW) void k_cache_write(CacheDev c, rheo_write_args a, int rows,
                                                     int parts) {
    constexpr int GROUPS = 64 / LPH;                 // heads a wave works on at once
    const int lane = threadIdx.x & 63;
    const int t = lane % LPH, g = lane / LPH;
    const int unit = blockIdx.x * (NTW / 64) + threadIdx.x / 64;    // a wave's (row, part)
    const int row = unit / parts, part = unit - row * parts;
    if (row >= rows) return;
    const int64_t slot = a.slots[row];
    if (slot < 0) return;
    const int64_t place_mask = ((int64_t)1 << c.page_shift) - 1;
    if (slot >= ((int64_t)c.pages << c.page_shift)) {
        if (lane == 0) atomicOr(c.err, CE_SLOT);
        return;
    }
    const int D = c.D, NV = D >> 3, r = a.rot_dim, half = r >> 1;
    // the lane's two vectors
    int va, vb;
    const int rl = MODE == HALVES ? half >> 3 : 0;   // lanes of rotated halves
    if (t < rl) {
        va = t;
        vb = t + rl;
    } else {
        va = 2 * rl + 2 * (t - rl);
        vb = va + 1;
    }
    const bool has_a = va < NV, has_b = vb < NV;

    float cs[16], sn[16];
    if (MODE != NONE) {
        const int pos = a.positions[row];
        if ((unsigned)pos >= (unsigned)a.max_position) {
            if (lane == 0) atomicOr(c.err, CE_POSITION);
            return;
        }
        const float* line = a.rotation + (int64_t)pos * r;
        if (MODE == HALVES) {
            if (t < rl) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    cs[j] = line[8 * t + j];
                    sn[j] = line[half + 8 * t + j];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int e = 8 * (j < 8 ? va : vb) + (j & 7);
                const int k = MODE == NEIGHBOURS ? e >> 1 : e < half ? e : e - half;
                const bool in = e < r;
                if (MODE == ODD_HALVES || !(j & 1)) {
                    cs[j] = in ? line[k] : 1.0f;
                    sn[j] = in ? line[half + k] : 0.0f;
                }
            }
        }
    }

    const int64_t entry = (slot >> c.page_shift) * c.page_stride +
                          (slot & place_mask) * ((int64_t)c.K * D);
    const int first = a.q ? 0 : c.H, heads = c.H + 2 * c.K;
    auto source = [&](int h) {
        return h < c.H ? (const T*)a.q + (int64_t)row * a.q_stride + (int64_t)h * D
               : h < c.H + c.K ? (const T*)a.k + (int64_t)row * a.k_stride + (int64_t)(h - c.H) * D
                               : (const T*)a.v + (int64_t)row * a.v_stride + (int64_t)(h - c.H - c.K) * D;
    };
    int h = first + part * GROUPS + g;
    uint4 na = {0, 0, 0, 0}, nb = {0, 0, 0, 0};      // the next head's vectors, on their way
    if (h < heads) {
        const T* src = source(h);
        if (has_a) na = *(const uint4*)(src + 8 * va);
        if (has_b) nb = *(const uint4*)(src + 8 * vb);
    }
    for (; h < heads; h += parts * GROUPS) {
        const T* const src = source(h);
        T* dst;
        const T* w = nullptr;
        const bool value = h >= c.H + c.K;
        if (h < c.H) {
            dst = (T*)a.q_out + (int64_t)row * a.q_out_stride + (int64_t)h * D;
            w = (const T*)a.q_weight;
        } else if (!value) {
            dst = (T*)a.k_cache + entry + (int64_t)(h - c.H) * D;
            w = (const T*)a.k_weight;
        } else {
            dst = (T*)a.v_cache + entry + (int64_t)(h - c.H - c.K) * D;
        }
        uint4 xa = na, xb = nb;
        if (h + parts * GROUPS < heads) {
            const T* s1 = source(h + parts * GROUPS);
            if (has_a) na = *(const uint4*)(s1 + 8 * va);
            if (has_b) nb = *(const uint4*)(s1 + 8 * vb);
        }
        if (!value) {
            float x[16];
            unpack8<T>(xa, x);
            unpack8<T>(xb, x + 8);
            float inv = 1.0f;
            if (w) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 16; ++j) sum = __fmaf_rn(x[j], x[j], sum);
#pragma unroll
                for (int o = LPH / 2; o; o >>= 1) sum += __shfl_xor(sum, o);
                inv = 1.0f / sqrtf(__fmaf_rn(sum, 1.0f / (float)D, a.eps));
            }
            float y[16];                             // the partners, where loaded apart
            if (MODE == ODD_HALVES) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int e = 8 * (j < 8 ? va : vb) + (j & 7);
                    const int p = e < half ? e + half : e - half;
                    y[j] = 0.0f;
                    if (e < r) {
                        y[j] = (float)src[p] * inv;
                        if (w) y[j] *= (float)w[p];
                        if (e < half) y[j] = -y[j];
                    }
                }
            }
            if (w) {
                float wf[16];
                uint4 wa = {0, 0, 0, 0}, wb = {0, 0, 0, 0};
                if (has_a) wa = *(const uint4*)(w + 8 * va);
                if (has_b) wb = *(const uint4*)(w + 8 * vb);
                unpack8<T>(wa, wf);
                unpack8<T>(wb, wf + 8);
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = x[j] * inv * wf[j];
            }
            if (MODE == HALVES) {
                if (t < rl) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float p = x[j], q = x[j + 8];
                        x[j] = p * cs[j] - q * sn[j];
                        x[j + 8] = q * cs[j] + p * sn[j];
                    }
                }
            } else if (MODE == NEIGHBOURS) {
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float p = x[j], q = x[j + 1];
                    x[j] = p * cs[j] - q * sn[j];
                    x[j + 1] = q * cs[j] + p * sn[j];
                }
            } else if (MODE == ODD_HALVES) {
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = x[j] * cs[j] + y[j] * sn[j];
            }
            xa = pack8<T>(x);
            xb = pack8<T>(x + 8);
        }
        if (has_a) *(uint4*)(dst + 8 * va) = xa;
        if (has_b) *(uint4*)(dst + 8 * vb) = xb;
    }
}

namespace {

template <typename T, int LPH>
void start(const CacheDev& c, const rheo_write_args& a, int blocks, int rows, int parts,
           hipStream_t s) {
    if (a.rot_dim == 0)
        k_cache_write<T, LPH, NONE><<<blocks, NTW, 0, s>>>(c, a, rows, parts);
    else if (a.interleaved)
        k_cache_write<T, LPH, NEIGHBOURS><<<blocks, NTW, 0, s>>>(c, a, rows, parts);
    else if (a.rot_dim % 16 == 0)
        k_cache_write<T, LPH, HALVES><<<blocks, NTW, 0, s>>>(c, a, rows, parts);
    else
        k_cache_write<T, LPH, ODD_HALVES><<<blocks, NTW, 0, s>>>(c, a, rows, parts);
}

template <typename T>
void start_lph(const CacheDev& c, const rheo_write_args& a, int blocks, int rows, int parts,
               int lph, hipStream_t s) {
    if (lph == 4) start<T, 4>(c, a, blocks, rows, parts, s);
    else if (lph == 8) start<T, 8>(c, a, blocks, rows, parts, s);
    else start<T, 16>(c, a, blocks, rows, parts, s);
}

}  // namespace

hipError_t launch_cache_write(const CacheDev& c, const rheo_write_args& a, hipStream_t s) {
    const int rows = c.B * a.n;
    // two vectors a lane: D / 16 lanes and, behind halves of an odd number of
    // vectors, none more (rot_dim % 16 == 0 leaves (D - rot) / 8 vectors in pairs)
    const int lph = c.D <= 64 ? 4 : c.D <= 128 ? 8 : 16;
    const int heads = (a.q ? c.H : 0) + 2 * c.K, rounds = (heads + 64 / lph - 1) / (64 / lph);
    // A wave takes four rounds of a row's heads (120 heads in one wave of 15 rounds:
    // 70 us for 65), and fewer where that leaves less than 16 waves to each of 256 compute
    // units and latency counts
    int parts = (rounds + 3) / 4;
    if ((int64_t)rows * parts < 4096) parts = 4096 / rows < rounds ? 4096 / rows : rounds;
    if (rows * (int64_t)parts > kWriteRows) parts = (int)(kWriteRows / rows);
    const int64_t waves = (int64_t)rows * parts;
    const int blocks = (int)((waves + NTW / 64 - 1) / (NTW / 64));
    if (c.dtype == RHEO_BF16) start_lph<__bf16>(c, a, blocks, rows, parts, lph, s);
    else start_lph<_Float16>(c, a, blocks, rows, parts, lph, s);
    return hipGetLastError();
}

}  // namespace rheo
