// kv4_sweep.h -- one wave's online softmax of 16 query rows over 32-token blocks of
// the 4-bit cache, on the codes themselves: what kv4_rows.hip is made of, and what
// kv4_many.hip turns to for rows that its tiles do not suit.
//
// Scores: kv4_tile.h.  The second product is O^T = V^T P^T on V's codes:
//   O = sum_j (p_j scale_j) code_j + sum_j p_j min_j
// (strict: code - 8, with min + 8 scale) with p scale rounded to f16 (half a step
// 2^-11, where a bf16 result has 2^-8; strict: two parts, 2^-23) and the second
// sum in f32 from the unrounded p.  f16 holds p scale because both
// factors are taken relative to a running bound of the row: p to 2^kRowSlack
// above 1, and the scales to a power of two, moved up (and the sums rescaled, as
// for a new maximum) when a block has a larger one that the row sees.  kRaise
// lifts the products to the top of f16's range, so that products 2^-25 below the
// largest scale's keep all their bits (of the two strict parts: 2^-13).
#pragma once

#include "kv4_tile.h"

namespace mg {

constexpr int kSweepRows = 16;
constexpr float kRowSlack = 4.f;
constexpr int kRaise = 11;    // 2^(slack + 11) = 2^15 at most
constexpr int kExpMax = 100;  // bound on the scales' exponent (|V| about 2^104)
// Least e, and how far a minimum may lie above 2^e: sums of 2^24 p and p min in
// units of 2^(e - kRaise) stay below 2^(4 + 11 + 80 + 24).
constexpr int kExpMin = -80;

// Where row r = i * G + g of a cache head lies among the query rows.
struct RowAt {
    int i;
    size_t at;   // row of [B][Hq][Lq]
};
__device__ __forceinline__ RowAt row_at(int r, int bh, int G, int Lq) {
    const int i = r / G;
    return {i, ((size_t)bh * G + (r - i * G)) * Lq + i};
}

template <int D>
struct Kv4Values {
    static constexpr int NB = Kv4Dim<D>::kBlocks, W = Kv4Dim<D>::kWide;
    uint32_t w[NB];   // word of channel 16b + c of the lane's octet

    __device__ __forceinline__ void load(const uint32_t *words, int block, int c, int g) {
        typedef uint32_t wv __attribute__((ext_vector_type(W)));
        const uint32_t at = 4u * ((4 * block + g) * D + W * c);
#pragma unroll
        for (int h = 0; h < NB / W; ++h) {
            const wv v = *reinterpret_cast<const wv *>(reinterpret_cast<const char *>(words) +
                                                       (at + 64u * W * h));
#pragma unroll
            for (int i = 0; i < W; ++i) w[W * h + i] = v[i];
        }
    }
};

// The f32 bits of a V scale, or of what stands for its minimum if that is more; 0
// for a token that is not finite, which moves nothing.  (Words order as the scales
// in their upper halves do.)
__device__ __forceinline__ uint32_t value_bound(uint32_t scale, uint32_t size) {
    constexpr uint32_t kBelow = (uint32_t)-kExpMin << 23;
    return scale < 0x7f800000u ? max(scale, max(size, kBelow) - kBelow) : 0u;
}

template <int NG>
struct BlockGroups {   // a block's groups in LDS, token k's at k * NG
    float scale[2][32 * NG], base[2][32 * NG];   // of K, V
};

// A block's group words, brought in by the wave's lanes (a word of K and one of V
// each, or with one group a word of either), taken apart there and handed over
// through LDS.
template <int NG>
struct Kv4GroupWords {
    uint32_t w[NG];   // NG = 2: K's, V's; NG = 1: K's in lanes below 32, else V's

    __device__ __forceinline__ void load(const uint32_t *kp, const uint32_t *vp, int block,
                                         int lane) {
        if (NG == 2) {
            const uint32_t at = 4u * (64 * block + lane);
            w[0] = *reinterpret_cast<const uint32_t *>(reinterpret_cast<const char *>(kp) + at);
            w[NG - 1] = *reinterpret_cast<const uint32_t *>(reinterpret_cast<const char *>(vp) + at);
        } else {
            w[0] = (lane < 32 ? kp : vp)[32 * block + (lane & 31)];
        }
    }
    // taken apart, K's times `unit` (a power of two; in lanes that hold V's alone 1);
    // 0 for tokens at or behind n
    template <int NP>
    __device__ __forceinline__ void put(BlockGroups<NG> &to, int block, int n, float unit,
                                        int lane) {
        const bool in = 32 * block + (NG == 2 ? lane >> 1 : lane & 31) < n;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            w[i] = in ? w[i] : 0u;
            float *scale = &to.scale[0][0], *base = &to.base[0][0];
            const float times = i == 0 ? unit : 1.f;
            scale[64 * i + lane] = group_scale(w[i]) * times;
            base[64 * i + lane] = base_of<NP>(w[i]) * times;
        }
    }
    // the lane's V word as a bound of its token, or 0
    __device__ __forceinline__ uint32_t bound(int lane) const {
        const uint32_t v = NG == 2 || lane >= 32 ? w[NG - 1] : 0u;
        return value_bound(v, (v & 0x7fffu) << 16);
    }
};

// The sums of a wave's 16 rows.  A lane holds row c = lane % 16, of a block the tokens
// 8g .. 8g + 7 with g = lane / 16.
template <int D, int NP>
struct Kv4Sweep {
    static constexpr int NG = Kv4Dim<D>::kGroups, NB = Kv4Dim<D>::kBlocks;

    float m = -INFINITY;               // running maximum (base 2) rounded up, of the row
    int e = kExpMin;                   // V's scales that the row sees are below 2^e, its
                                       // minima (strict: bases) below 2^(e + 80)
    uint32_t most = 0;                 // ... as a value_bound
    float off = kRaise - kExpMin;      // of exponents: kRaise - e - m
    float l = 0.f;                     // sum of p 2^(kRaise - e)
    float low[NG];                     // sums of p base in the same units
    f32x4 o[NB];                       // O^T[16 b + 4g + r][row c], over kCodeUnit

    __device__ __forceinline__ Kv4Sweep() {
#pragma unroll
        for (int i = 0; i < NG; ++i) low[i] = 0.f;
#pragma unroll
        for (int i = 0; i < NB; ++i) o[i] = zero4();
    }

    // The row's products are scores times 1 / factor where K's groups are taken times unit.
    struct Factors {
        float factor, unit;
    };
    static __device__ __forceinline__ Factors factors(const Kv4Query<D, NP> &q, float scale_log2,
                                                      int lane) {
        // (a size is a whole number that f32 holds)
        const int unit = __builtin_amdgcn_readfirstlane(
            key_unit(scale_log2, (int)max_of<16>((float)q.size)));
        return {positive_factor(scale_log2, q.exponent, unit),
                NG == 2 || lane < 32 ? power_of_two(unit) : 1.f};
    }

    // One block, later ones later.  The row sees tokens below `limit`, every row of the
    // wave those below `all`; `n`: the sequence's tokens; `keep` gets the scores first.
    template <typename Keep>
    __device__ __forceinline__ void step(int block, const Kv4Query<D, NP> &q, Factors f,
                                         int limit, int all, int n, const Kv4Keys<D> &key,
                                         const Kv4Values<D> &val, Kv4GroupWords<NG> &words,
                                         BlockGroups<NG> &groups, int lane, Keep &&keep) {
        const int c = lane & 15, g = lane >> 4;
        const float factor = f.factor;
        words.template put<NP>(groups, block, n, f.unit, lane);
        __builtin_amdgcn_wave_barrier();   // one wave's LDS accesses stay in order
        f32x4 s[2];
        key.scores(s, q, groups.scale[0], groups.base[0], c, g);
        float vs[8 * NG], vm[8 * NG];   // of the lane's octet
#pragma unroll
        for (int i = 0; i < 2 * NG; ++i) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(&groups.scale[1][8 * g * NG + 4 * i]);
            const f32x4 y = *reinterpret_cast<const f32x4 *>(&groups.base[1][8 * g * NG + 4 * i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                vs[4 * i + k] = x[k];
                vm[4 * i + k] = y[k];
            }
        }
        uint32_t top = words.bound(lane);
        const bool partly = 32 * (block + 1) > all;
        if (partly) {
            // tokens out of sight: no score, and groups that add nothing and bound
            // nothing (a token that is not finite, or far above the others, must not
            // reach rows that do not see it)
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (32 * block + 8 * g + k >= limit) {
                    s[k >> 2][k & 3] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < NG; ++i) vs[k * NG + i] = vm[k * NG + i] = 0.f;
                }
            float scale = 0.f, base = 0.f;
#pragma unroll
            for (int i = 0; i < 8 * NG; ++i) {
                scale = fmaxf(scale, vs[i]);
                base = fmaxf(base, fabsf(vm[i]));
            }
            top = value_bound(__float_as_uint(max_over_groups(scale)),
                              __float_as_uint(max_over_groups(base)));
        }
        keep(s);
        float mx = max3_f32(max3_f32(s[0][0], s[0][1], s[0][2]),
                            max3_f32(s[0][3], s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]));
        mx = max_over_groups(mx) * factor;
        // (blocks that rows see part of come last, so `most` is the same in all lanes
        // up to the first of them)
        if (__any(mx > m + kRowSlack || top > most)) {
            const float m_new = fmaxf(m, ceilf(mx));
            const uint32_t high =
                partly ? top : __float_as_uint(max_of_wave(__uint_as_float(top)));
            const int e_new = max(e, min(kExpMax, (int)(high >> 23) - 126));
            const float lower = m_new == -INFINITY ? 1.f : exp2_fast(m - m_new);
            l = ldexpf(l * lower, e - e_new);   // (where the factor alone would be 0)
            const float alpha = ldexpf(lower, e - e_new);
#pragma unroll
            for (int i = 0; i < NG; ++i) low[i] *= alpha;
#pragma unroll
            for (int i = 0; i < NB; ++i) o[i] *= alpha;
            m = m_new;
            e = e_new;
            most = e == kExpMax ? 0xffffffffu : ((uint32_t)(e + 127) << 23) - 1;
            off = (float)(kRaise - e) - (m == -INFINITY ? 0.f : m);
        }
        float p[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            p[k] = exp2_fast(fmaf(s[k >> 2][k & 3], factor, off));
            l += p[k];
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            float x[8];
            f16x8 part[NP];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[k] = p[k] * vs[k * NG + i];
                low[i] = fmaf(p[k], vm[k * NG + i], low[i]);
            }
            split_operand<NP>(part, x);
#pragma unroll
            for (int cb = i * (NB / NG); cb < (i + 1) * (NB / NG); ++cb) {
                const f16x8 v = operand_of<NP>(val.w[cb]);
#pragma unroll
                for (int k = NP - 1; k >= 0; --k) o[cb] = mfma16x16x32f16(v, part[k], o[cb]);
            }
        }
    }

    // Out of the running units: sums of p 2^m and p v 2^m, O^T in the layout of o.
    __device__ __forceinline__ void finish() {
        l = ldexpf(sum_over_groups(l), e - kRaise);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const float base = sum_over_groups(low[i]);
#pragma unroll
            for (int cb = i * (NB / NG); cb < (i + 1) * (NB / NG); ++cb)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[cb][k] = ldexpf(fmaf(o[cb][k], kCodeUnit, base), e - kRaise);
        }
    }
};

}  // namespace mg
