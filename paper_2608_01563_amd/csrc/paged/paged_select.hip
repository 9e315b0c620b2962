// paged_select.hip -- the pages that each query row reads: scores from the pages'
// bounds, and the largest of them.
//
// sum_c max(q_c lo_c, q_c hi_c) is sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c: a
// matrix product of pages and rows over 2 d channels.  It runs on the f64 matrix
// units, as the choice must not hang on a sum's order: products of bf16 values are
// exact, and so are nearly all of their sums.  (f32 sums would let pages next to
// the border change places with the tile they are computed in.)
#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
typedef double f64x4 __attribute__((ext_vector_type(4)));

struct ScoreArgs {
    const char *Q, *bounds;
    float *score;
    const int32_t *table, *key_len, *q_len;
    int H, G, Lq, P, N, shift, causal, per, tiles, parts;   // per: rows i of a tile
};

// A wave takes 16 pages and as many rows i as have their G heads in 16 (one row,
// heads in turns, where G is above 16).
template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void paged_scores(ScoreArgs a) {
    constexpr int RB = D * (int)sizeof(T), NP = RB / 64, NE = 16 / (int)sizeof(T);
    __shared__ float out[kWaves][16][17];
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = blockIdx.x % a.parts, at = blockIdx.x / a.parts;
    const int tile = at % a.tiles, bh = at / a.tiles;
    const int b = bh / a.H, h = bh - b * a.H;
    const int p0 = (part * kWaves + w) * 16;
    const PagedMask mask = paged_mask(a.key_len, a.q_len, b, a.P << a.shift, a.Lq, a.causal);
    if ((p0 << a.shift) >= mask.n) return;
    const int i0 = tile * a.per, ni = min(a.per, a.Lq - i0);
    if (i0 >= mask.rows) return;

    const int id = a.table[(size_t)b * a.P + min(p0 + c, a.P - 1)];
    const bool known = (uint32_t)id < (uint32_t)a.N;
    const char *lo = a.bounds + ((size_t)(known ? id : 0) * a.H + h) * 2 * RB + 16 * g;
    u32x4 bound[2][NP];
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e)
            bound[e][s] = *reinterpret_cast<const u32x4 *>(lo + e * RB + 64 * s);

    float best = NAN;
    for (int g0 = 0; g0 < a.G; g0 += 16) {
        const int il = a.G > 16 ? 0 : c / a.G, head = a.G > 16 ? g0 + c : c - il * a.G;
        const bool in = il < ni && head < a.G;
        const char *q = a.Q + (((size_t)bh * a.G + (in ? head : 0)) * a.Lq + i0 + (in ? il : 0)) * RB +
                        16 * g;
        f64x4 sum = {0., 0., 0., 0.};
#pragma unroll
        for (int s = 0; s < NP; ++s) {
            const u32x4 qs = *reinterpret_cast<const u32x4 *>(q + 64 * s);
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const auto value = [&](u32x4 v) {
                    if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
                    else return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
                };
                const float x = value(qs);
                // (x != x: NaN in both)
                sum = __builtin_amdgcn_mfma_f64_16x16x4f64(
                    (double)value(bound[1][s]), (double)(x < 0.f ? 0.f : x), sum, 0, 0, 0);
                sum = __builtin_amdgcn_mfma_f64_16x16x4f64(
                    (double)value(bound[0][s]), (double)(x > 0.f ? 0.f : x), sum, 0, 0, 0);
            }
        }
        // lane (c, g) has pages 4 e + g of row c; then the largest over a row's heads
#pragma unroll
        for (int e = 0; e < 4; ++e) out[w][c][4 * e + g] = (float)sum[e];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (a.G > 16) {
            for (int k = 0; k < min(16, a.G - g0); ++k) best = fmaxf(best, out[w][k][c]);
        } else {
            for (int j = g; j < ni; j += 4) {
                best = NAN;
                for (int k = 0; k < a.G; ++k) best = fmaxf(best, out[w][j * a.G + k][c]);
                if (p0 + c < a.P)   // (+ 0: the two zeros are one score)
                    a.score[((size_t)bh * a.Lq + i0 + j) * a.P + p0 + c] = known ? best + 0.f : NAN;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (a.G > 16 && g == 0 && p0 + c < a.P)
        a.score[((size_t)bh * a.Lq + i0) * a.P + p0 + c] = known ? best + 0.f : NAN;
}

// ------------------------------------------------------------------ selection --
struct SelectArgs {
    const float *score;
    int32_t *index;
    const int32_t *key_len, *q_len;
    int H, Lq, P, shift, causal, keep, first, recent;
};

// Scores in the order of unsigned numbers, NaN lowest.
__device__ __forceinline__ uint32_t key_of(float s) {
    const uint32_t u = __float_as_uint(s);
    if (s != s) return 0;
    return u >> 31 ? ~u : u | 0x80000000u;
}

// A workgroup takes a row: the key of the last page kept, by its digits of 8 bits
// from the top, each from counts in LDS; then pages in order.
template <int THREADS>
__global__ __launch_bounds__(THREADS)
void paged_select(SelectArgs a) {
    constexpr int W = THREADS / 64;
    __shared__ uint32_t counts[256];
    __shared__ uint32_t found[2];
    __shared__ int totals[2][W];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int i = blockIdx.x % a.Lq, bh = blockIdx.x / a.Lq, b = bh / a.H;
    const PagedMask mask = paged_mask(a.key_len, a.q_len, b, a.P << a.shift, a.Lq, a.causal);
    const int m = (mask.limit(i) + (1 << a.shift) - 1) >> a.shift;
    const float *score = a.score + (size_t)blockIdx.x * a.P;
    int32_t *index = a.index + (size_t)blockIdx.x * a.keep;
    if (m <= a.keep) {
        for (int k = tid; k < a.keep; k += THREADS) index[k] = k < m ? k : -1;
        return;
    }
    const int from = a.first, to = m - a.recent;
    int left = a.keep - a.first - a.recent;   // to be found among pages from .. to - 1
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int k = tid; k < 256; k += THREADS) counts[k] = 0;
        __syncthreads();
        for (int p = from + tid; p < to; p += THREADS) {
            const uint32_t key = key_of(score[p]);
            if (shift == 24 || (key ^ prefix) >> (shift + 8) == 0)
                atomicAdd(&counts[key >> shift & 255], 1u);
        }
        __syncthreads();
        if (w == 0) {
            // lane l has digits 255 - 4 l down to 252 - 4 l
            uint32_t n[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) n[e] = counts[255 - 4 * lane - e], sum += n[e];
            const uint32_t upto = wave_scan(sum);
            uint32_t above = upto - sum;
            if (above < (uint32_t)left && upto >= (uint32_t)left)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < (uint32_t)left && above + n[e] >= (uint32_t)left) {
                        found[0] = 255 - 4 * lane - e;
                        found[1] = left - above;
                    }
                    above += n[e];
                }
        }
        __syncthreads();
        if (left > 0) {
            prefix |= found[0] << shift;
            left = found[1];
        }
    }
    // keys above the prefix stay, and the first `left` of those equal to it
    const bool some = a.keep > a.first + a.recent;
    int equal = 0, kept = 0;
    for (int p0 = 0; p0 < m; p0 += THREADS) {
        const int p = p0 + tid;
        const bool fixed = p < from || (p >= to && p < m);
        const uint32_t key = some && p >= from && p < to ? key_of(score[p]) : 0;
        const bool inside = some && p >= from && p < to;
        const bool same = inside && key == prefix;
        const uint64_t below = (1ull << lane) - 1;
        const uint64_t sames = __ballot(same);
        if (lane == 0) totals[0][w] = __popcll(sames);
        __syncthreads();
        int rank = equal + __popcll(sames & below);
        for (int k = 0; k < W; ++k) {
            if (k < w) rank += totals[0][k];
            equal += totals[0][k];
        }
        const bool stays = fixed || (inside && key > prefix) || (same && rank < left);
        const uint64_t stay = __ballot(stays);
        if (lane == 0) totals[1][w] = __popcll(stay);
        __syncthreads();
        int at = kept + __popcll(stay & below);
        for (int k = 0; k < W; ++k) {
            if (k < w) at += totals[1][k];
            kept += totals[1][k];
        }
        if (stays) index[at] = p;
    }
}

template <typename T, int D>
hipError_t scores(const PagedSelect &p, const void *Q, const void *bounds, float *score,
                  hipStream_t s) {
    const int per = p.G >= 16 ? 1 : 16 / p.G, tiles = (p.Lq + per - 1) / per;
    const ScoreArgs a = {static_cast<const char *>(Q), static_cast<const char *>(bounds), score,
                         p.table, p.key_len, p.q_len, p.H, p.G, p.Lq, p.P, p.N, p.shift, p.causal,
                         per, tiles, (p.P + 16 * kWaves - 1) / (16 * kWaves)};
    const unsigned grid = (unsigned)((int64_t)a.parts * p.B * p.H * tiles);
    paged_scores<T, D><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_scores(const PagedSelect &p, const void *Q, const void *bounds, bool bf16,
                               float *score, hipStream_t s) {
    if (bf16)
        return p.d == 32 ? scores<uint16_t, 32>(p, Q, bounds, score, s)
             : p.d == 64 ? scores<uint16_t, 64>(p, Q, bounds, score, s)
                         : scores<uint16_t, 128>(p, Q, bounds, score, s);
    return p.d == 32 ? scores<float, 32>(p, Q, bounds, score, s)
         : p.d == 64 ? scores<float, 64>(p, Q, bounds, score, s)
                     : scores<float, 128>(p, Q, bounds, score, s);
}

hipError_t launch_paged_select(const PagedSelect &p, const float *score, int32_t *index,
                               hipStream_t s) {
    const SelectArgs a = {score, index, p.key_len, p.q_len, p.H, p.Lq, p.P, p.shift, p.causal,
                          p.keep, p.first, p.recent};
    const unsigned grid = (unsigned)(p.B * p.H * p.Lq);
    if (p.P <= 1024) paged_select<256><<<grid, 256, 0, s>>>(a);
    else paged_select<1024><<<grid, 1024, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace mg
