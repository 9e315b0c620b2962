// paged_select.hip -- the pages that each query row reads: scores from the pages'
// bounds, and the largest of them.
//
// sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c (where lo <= hi: max(q_c lo_c, q_c hi_c)) is
// a matrix product of pages and rows over 2 d channels.  A channel of NaN alone, whose
// bounds are reversed, makes the sum as low as it goes.  It runs on the f64 matrix
// units, as the choice must not hang on a sum's order: products of bf16 values are
// exact, and so are nearly all of their sums.  (f32 sums would let pages next to
// the border change places with the tile they are computed in.)
#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct ScoreArgs {
    const char *Q, *bounds;
    float *score;
    const int32_t *table, *key_len, *q_len;
    int H, G, Lq, P, N, shift, causal, per, tiles, parts;   // per: rows i of a tile
};

// A wave takes 16 pages and four query rows: 4x4x4 products in four blocks.  Lane l is
// of block (l / 4) % 4, with page l % 4 of the block's four, query row l % 4 and the
// l / 16-th 16 bytes of channels out of every 64; of the result it has query row l % 4
// and page l / 16.  The rows are those of as many i as have their G heads in
// four, or of one i with its heads in turns.  (16x16x4 products take four times as
// long, whatever G is.)
//
// max(q, 0) and min(q, 0) lie in LDS as 64-bit numbers, made once for the workgroup's
// 64 pages: conversions would cost more than the products.
template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void paged_scores(ScoreArgs a) {
    constexpr int RB = D * (int)sizeof(T), NP = RB / 64, NE = 16 / (int)sizeof(T);
    __shared__ double2 query[NP][NE][16];   // of lane (k, c), 4 k + c
    const int tid = threadIdx.x, lane = tid & 63;
    const int c = lane & 3, block = lane >> 2 & 3, k = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (turned, so that the first parts, which all sequences have, are not on the same XCDs)
    const int at = blockIdx.x / a.parts;
    const int part = (blockIdx.x % a.parts + 3 * (at % a.parts)) % a.parts;
    const int tile = at % a.tiles, bh = at / a.tiles;
    const int b = bh / a.H, h = bh - b * a.H;
    const int p0 = (part * kWaves + w) * 16;
    const int entry = a.table[(size_t)b * a.P + min(p0 + 4 * block + c, a.P - 1)];
    const int i0 = tile * a.per, ni = min(a.per, a.Lq - i0);

    // head g0 + .. or heads of rows il as above, of query row j of four
    struct Row {
        int il, head;
        bool in;
    };
    const auto row_of = [&](int g0, int j) {
        const int il = a.G > 4 ? 0 : j / a.G, head = a.G > 4 ? g0 + j : j - il * a.G;
        return Row{il, head, il < ni && head < a.G};
    };
    const auto value = [](u32x4 v, int e) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
        else return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    };
    // threads below 16 NP take 16 bytes each
    const int qj = tid & 3, qk = tid >> 2 & 3, qs = tid >> 4;
    const auto read_query = [&](int g0) {
        const Row r = row_of(g0, qj);
        const char *q = a.Q + (((size_t)bh * a.G + (r.in ? r.head : 0)) * a.Lq + i0 +
                               (r.in ? r.il : 0)) * RB + 64 * qs + 16 * qk;
        return qs < NP && r.in ? *reinterpret_cast<const u32x4 *>(q) : u32x4{0, 0, 0, 0};
    };
    u32x4 q = read_query(0);
    const PagedMask mask = paged_mask(a.key_len, a.q_len, b, a.P << a.shift, a.Lq, a.causal);
    if (((part * kWaves * 16) << a.shift) >= mask.n || i0 >= mask.rows) return;

    const bool known = (uint32_t)entry < (uint32_t)a.N && p0 << a.shift < mask.n;
    const char *lo = a.bounds + ((size_t)(known ? entry : 0) * a.H + h) * 2 * RB + 16 * k;
    u32x4 bound[2][NP];
#pragma unroll
    for (int s = 0; s < NP; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e)
            bound[e][s] = *reinterpret_cast<const u32x4 *>(lo + e * RB + 64 * s);

    float best = NAN;
    for (int g0 = 0; g0 < a.G; g0 += 4) {
        if (qs < NP)
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const float x = value(q, e);   // (x != x: NaN in both)
                query[qs][e][4 * qk + qj] = make_double2(x < 0.f ? 0.f : x, x > 0.f ? 0.f : x);
            }
        if (g0 + 4 < a.G) q = read_query(g0 + 4);
        __syncthreads();
        double sum[2] = {0., 0.};
#pragma unroll
        for (int s = 0; s < NP; ++s)
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const double2 x = query[s][e][4 * k + c];
                sum[0] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)value(bound[1][s], e), x.x,
                                                            sum[0], 0, 0, 0);
                sum[1] = __builtin_amdgcn_mfma_f64_4x4x4f64((double)value(bound[0][s], e), x.y,
                                                            sum[1], 0, 0, 0);
            }
        if (row_of(g0, c).in) best = fmaxf(best, (float)(sum[0] + sum[1]));
        if (g0 + 4 < a.G) __syncthreads();
    }
    const int il = a.G > 4 ? 0 : c / a.G;
    // the largest over a row's heads, which are c of the same k and block
    if (a.G > 1) best = fmaxf(best, other_lane<0>(best));
    if (a.G > 2) best = fmaxf(best, other_lane<1>(best));
    const int p = p0 + 4 * block + k;
    const bool page_known = __shfl((int)known, 4 * block + k, 64);
    const bool first = a.G > 2 ? c == 0 : c == il * a.G;
    if (first && il < ni && p < a.P && p << a.shift < mask.n)   // (+ 0: the two zeros are one score)
        a.score[((size_t)bh * a.Lq + i0 + il) * a.P + p] = page_known ? best + 0.f : NAN;
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

// The digit (256 of them, from the top) with the left-th key, and which of the digit's
// keys that is; by one wave.
__device__ __forceinline__ void find_digit(const uint32_t *counts, uint32_t left,
                                           uint32_t *found) {
    // lane l has digits 255 - 4 l down to 252 - 4 l
    const int lane = threadIdx.x & 63;
    uint32_t n[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) n[e] = counts[255 - 4 * lane - e], sum += n[e];
    const uint32_t upto = wave_scan(sum);
    uint32_t above = upto - sum;
    if (above >= left || upto < left) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (above < left && above + n[e] >= left) {
            found[0] = 255 - 4 * lane - e;
            found[1] = left - above;
        }
        above += n[e];
    }
}

// What is to be found among pages from .. to - 1 of a row's m: `left` of them.
struct Wanted {
    int m, from, to, left;
};

// The general way: the key of the last page kept, by its digits of 8 bits from the
// top, each from counts in LDS; then pages in order.
template <int THREADS>
__device__ __forceinline__ void select_by_digits(const Wanted &r, const float *score,
                                                 int32_t *index) {
    constexpr int W = THREADS / 64;
    __shared__ uint32_t counts[256];
    __shared__ uint32_t found[2];
    __shared__ int totals[2][W];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int left = r.left;
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int k = tid; k < 256; k += THREADS) counts[k] = 0;
        __syncthreads();
        for (int p = r.from + tid; p < r.to; p += THREADS) {
            const uint32_t key = key_of(score[p]);
            if (shift == 24 || (key ^ prefix) >> (shift + 8) == 0)
                atomicAdd(&counts[key >> shift & 255], 1u);
        }
        __syncthreads();
        if (w == 0) find_digit(counts, left, found);
        __syncthreads();
        prefix |= found[0] << shift;
        left = found[1];
    }
    // keys above the prefix stay, and the first `left` of those equal to it
    int equal = 0, kept = 0;
    for (int p0 = 0; p0 < r.m; p0 += THREADS) {
        const int p = p0 + tid;
        const bool inside = p >= r.from && p < r.to;
        const uint32_t key = inside ? key_of(score[p]) : 0;
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
        const bool stays =
            (p < r.m && !inside) || (inside && key > prefix) || (same && rank < left);
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

// A workgroup takes a row.  With at most K pages a thread, scores stay in registers:
// they are counted in 256 equal steps from the smallest to the largest, the few that
// share the last page's step are ranked one by one, and places follow from one more
// count.  Where too many share it (equal scores), or pages are too many: by digits.
template <int THREADS, int K>
__global__ __launch_bounds__(THREADS)
void paged_select(SelectArgs a) {
    constexpr int W = THREADS / 64;
    static_assert(K * W <= 64, "a lane for every wave's count");
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int i = blockIdx.x % a.Lq, bh = blockIdx.x / a.Lq, b = bh / a.H;
    const float *score = a.score + (size_t)blockIdx.x * a.P;
    float s[K > 0 ? K : 1];   // (also of pages behind the sequence's, unused)
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = score[min(tid + k * THREADS, a.P - 1)];
    const PagedMask mask = paged_mask(a.key_len, a.q_len, b, a.P << a.shift, a.Lq, a.causal);
    const int m = (mask.limit(i) + (1 << a.shift) - 1) >> a.shift;
    int32_t *index = a.index + (size_t)blockIdx.x * a.keep;
    if (m <= a.keep) {
        for (int k = tid; k < a.keep; k += THREADS) index[k] = k < m ? k : -1;
        return;
    }
    const Wanted r = {m, a.first, m - a.recent, a.keep - a.first - a.recent};
    if (r.left == 0) {
        for (int k = tid; k < a.keep; k += THREADS) index[k] = k < a.first ? k : m - a.keep + k;
        return;
    }
    if constexpr (K == 0) {
        select_by_digits<THREADS>(r, score, index);
    } else {
        constexpr int LIST = 256;
        __shared__ float ends[2][W];
        __shared__ uint32_t counts[256], found[2], list_key[LIST], last_key;
        __shared__ int listed, list_page[LIST], last_page, totals[64];
        for (int k = tid; k < 256; k += THREADS) counts[k] = 0;
        if (tid == 0) listed = 0;
        const auto page_of = [&](int k) { return tid + k * THREADS; };
        const auto inside = [&](int k) { return page_of(k) >= r.from && page_of(k) < r.to; };
        float top = -INFINITY, low = -INFINITY;   // of s, of -s
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (inside(k) && fabsf(s[k]) < INFINITY) {
                top = fmaxf(top, s[k]);
                low = fmaxf(low, -s[k]);
            }
        top = max_xor32(max_xor16(max_of<16>(top)));
        low = max_xor32(max_xor16(max_of<16>(low)));
        if (lane == 0) ends[0][w] = top, ends[1][w] = low;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < W; ++k) {
            top = fmaxf(top, ends[0][k]);
            low = fmaxf(low, ends[1][k]);
        }
        // rising with the score: each of these operations is
        const float width = top + low, steps = width > 0.f && width < INFINITY ? 254.f / width : 0.f;
        const auto step_of = [&](float x) {
            if (x != x) return 0;
            return 1 + (int)fminf(fmaxf((x + low) * steps, 0.f), 254.f);
        };
        int step[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            step[k] = step_of(s[k]);
            if (inside(k)) atomicAdd(&counts[step[k]], 1u);
        }
        __syncthreads();
        if (w == 0) find_digit(counts, r.left, found);
        __syncthreads();
        const int last = found[0], left = found[1];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (inside(k) && step[k] == last) {
                const int at = atomicAdd(&listed, 1);
                if (at < LIST) list_key[at] = key_of(s[k]), list_page[at] = page_of(k);
            }
        __syncthreads();
        const int n = listed;
        if (n > LIST) {
            select_by_digits<THREADS>(r, score, index);
            return;
        }
        if (tid < n) {
            const uint32_t key = list_key[tid];
            const int page = list_page[tid];
            int rank = 0;
            for (int k = 0; k < n; ++k)
                rank += list_key[k] > key || (list_key[k] == key && list_page[k] < page);
            if (rank == left - 1) last_key = key, last_page = page;
        }
        __syncthreads();
        uint64_t stay[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const uint32_t key = key_of(s[k]);
            stay[k] = __ballot(inside(k) ? step[k] > last ||
                                               (step[k] == last &&
                                                (key > last_key ||
                                                 (key == last_key && page_of(k) <= last_page)))
                                         : page_of(k) < m);
            if (lane == 0) totals[k * W + w] = __popcll(stay[k]);
        }
        __syncthreads();
        const uint32_t upto = wave_scan(lane < K * W ? (uint32_t)totals[lane] : 0u);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int unit = k * W + __builtin_amdgcn_readfirstlane(w);
            const int before = unit == 0 ? 0 : __builtin_amdgcn_readlane(upto, unit - 1);
            if (stay[k] >> lane & 1)
                index[before + __popcll(stay[k] & ((1ull << lane) - 1))] = page_of(k);
        }
    }
}

template <typename T, int D>
hipError_t scores(const PagedSelect &p, const void *Q, const void *bounds, float *score,
                  hipStream_t s) {
    const int per = p.G >= 4 ? 1 : 4 / p.G, tiles = (p.Lq + per - 1) / per;
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
    if (p.P <= 1024) paged_select<256, 4><<<grid, 256, 0, s>>>(a);
    else if (p.P <= 4096) paged_select<1024, 4><<<grid, 1024, 0, s>>>(a);
    else paged_select<1024, 0><<<grid, 1024, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace mg
