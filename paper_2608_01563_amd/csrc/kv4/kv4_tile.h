// kv4_tile.h -- scores of 16 query rows against 32 cached tokens, on the
// 4-bit codes themselves.
//
//   q . k = sum over groups  scale (q_g . code_g) + min (sum of q_g)
//
// A byte that holds a code is that code times 2^-9 as an E4M3 number (the seven
// subnormals and the first eight normals are evenly spaced), so two masks, a
// shift and four conversions make the eight f16 operands of a word, exactly and
// normal: about 24 clocks a wave.  (Codes masked in place into f16 subnormals cost
// 12, but matrix products align operands by their exponent fields and lose the
// leading zeros' bits: scores were off by 1.2e-5 where they are now off by 4e-7.)
//
// Products are S^T = K Q^T: a wave's 32 tokens are the rows of two 16x16x32
// products, in the order that leaves lane group g = lane/16 with the eight
// tokens 8g..8g+7 of its query row lane%16: row i of product t is token
// 8(i/4) + 4t + i%4.  Those eight are an octet of V's words, so the
// probabilities feed the second product from the lanes that hold them.
#pragma once

#include "kv4_device.h"

namespace mg {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Which of eight consecutive values operand slot k holds: the order in which
// code_operand finds a word's nibbles.
__device__ __forceinline__ constexpr int slot_value(int k) { return k < 4 ? 2 * k : 2 * k - 7; }
constexpr float kCodeUnit = 0x1p9f;   // an operand is a code over this

template <int TIMES = 1>   // 512: the codes themselves
__device__ __forceinline__ f16x8 code_operand(uint32_t w) {
    const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, TIMES, false);
    const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(even, TIMES, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, TIMES, false);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(odd, TIMES, true);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The same of the codes less 8 (strict): a group's value is then scale (code - 8) +
// (min + 8 scale), two parts that no longer cancel where values lie on both sides
// of zero (O of up to 1,500 tokens: off by up to 1.3e-6 without, 9e-8 to 9e-7 over
// six draws with it).
__device__ __forceinline__ f16x8 centred_operand(uint32_t w) {
    return code_operand(w) - (_Float16)(8.f / kCodeUnit);
}
template <int NP>
__device__ __forceinline__ f16x8 operand_of(uint32_t w) {
    return NP > 1 ? centred_operand(w) : code_operand(w);
}
template <int NP>
__device__ __forceinline__ float base_of(uint32_t w) {   // what goes with it
    return NP > 1 ? fmaf(8.f, group_scale(w), group_min(w)) : group_min(w);
}

__device__ __forceinline__ f32x4 mfma16x16x32f16(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight f32 values as NP f16 operands in the slots of code_operand: one value
// each within 2^-12, two parts together within 2^-23.
template <int NP>
__device__ __forceinline__ void split_operand(f16x8 (&out)[NP], const float (&x)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float v = x[slot_value(k)];
        // Rounded to f32 here: where v is a product, a conversion fused with it rounds
        // once and, next to a tie, to another h than the one taken off below.
        if constexpr (NP > 1) asm("" : "+v"(v));
        const _Float16 h = (_Float16)v;
        out[0][k] = h;
        if constexpr (NP > 1) out[1][k] = (_Float16)(v - (float)h);
    }
}

// Exponent of a row's largest value; 0 for zero, infinity and NaN, which have no size.
constexpr int kNoSize = -1000;
__device__ __forceinline__ int query_exponent(float top, int *size) {
    const int e = __builtin_amdgcn_frexp_expf(top);
    *size = top > 0.f && top < INFINITY ? e : kNoSize;
    return e;
}

// A query row as operands: q[p][s] holds channels 32s + 8g + e of part p, times
// 2^(15 - exponent of the row's largest value); sum is one group's sum in the
// units of a product with codes.
template <int D, int NP>
struct Kv4Query {
    f16x8 q[NP][D / 32];
    float sum;      // of group g (0 where there is none)
    int exponent;   // scores = products * 2^(exponent - 6)
    int size;       // the same, kNoSize for a row of zeros or not finite

    template <typename T>
    __device__ __forceinline__ void load(const T *row, bool valid, int g, bool negate) {
        constexpr int NS = D / 32, NG = Kv4Dim<D>::kGroups;
        float x[NS][8];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) load_row(x[s], row + 32 * s + 8 * g);   // a row that is there
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[s][e] = valid ? x[s][e] : 0.f;
                top = fmaxf(top, fabsf(x[s][e]));
                if (negate) x[s][e] = -x[s][e];
            }
        top = max_over_groups(top);
        exponent = query_exponent(top, &size);
        sum = 0.f;
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            float t = 0.f;
#pragma unroll
            for (int s = gr * (NS / NG); s < (gr + 1) * (NS / NG); ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) t += ldexpf(x[s][e], -exponent);
            t = sum_over_groups(t) * 0x1p6f;
            if (g == gr) sum = t;
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            float y[8];
            f16x8 part[NP];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = ldexpf(x[s][e], 15 - exponent);
            split_operand<NP>(part, y);
#pragma unroll
            for (int p = 0; p < NP; ++p) q[p][s] = part[p];
        }
    }
};

// The K words of 32 tokens, two products' worth.
template <int D>
struct Kv4Keys {
    static constexpr int NG = Kv4Dim<D>::kGroups, NW = D / 32;
    uint32_t w[2][NW];

    // `words`: the head's region (below 4 GiB).  c = lane%16, g = lane/16.
    __device__ __forceinline__ void load(const uint32_t *words, int block, int c, int g) {
        typedef uint32_t wv __attribute__((ext_vector_type(NW)));
        const uint32_t at = (32 * block + 8 * (c >> 2) + (c & 3)) * (D / 8u) + g * NW;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const wv v = *reinterpret_cast<const wv *>(
                reinterpret_cast<const char *>(words) + (4 * at + 2u * t * D));
#pragma unroll
            for (int i = 0; i < NW; ++i) w[t][i] = NW == 1 ? v[0] : v[i];
        }
    }

    // s[t][r] = score of token 8g + 4t + r for the lane's row, before the row's
    // factor.  `scale`, `low`: the block's group scales and bases in LDS, token
    // k's at k * NG.
    template <int NP>
    __device__ __forceinline__ void scores(f32x4 (&s)[2], const Kv4Query<D, NP> &q,
                                           const float *scale, const float *low, int c,
                                           int g) const {
        f32x4 m[2][NG];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            // the bases' part: one product over the groups (sum is 0 behind them)
            s[t] = mfma16x16x4(low[(8 * (c >> 2) + 4 * t + (c & 3)) * NG + g % NG], q.sum,
                               zero4());
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                m[t][gr] = zero4();
#pragma unroll
                for (int i = gr * (NW / NG); i < (gr + 1) * (NW / NG); ++i) {
                    const f16x8 a = operand_of<NP>(w[t][i]);
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        m[t][gr] = mfma16x16x32f16(a, q.q[p][i], m[t][gr]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < NG; ++i) {   // (8g + 4t) NG + 4i ..+3
                const f32x4 v = *reinterpret_cast<const f32x4 *>(scale + (8 * g + 4 * t) * NG +
                                                                 4 * i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = (4 * i + k) / NG, gr = (4 * i + k) % NG;
                    s[t][r] = fmaf(v[k], m[t][gr][r], s[t][r]);
                }
            }
    }
};

// K's scales and minima enter scores times 2^key_unit, so that a product with codes is in
// range whenever the score is, and too small only where the score is nothing: the
// factor of the largest of the rows that share them (its size; kNoSize if none has one).
__device__ __forceinline__ int key_unit(float scale_log2, int size) {
    return scale_log2 == 0.f ? -126
         : min(max(__builtin_amdgcn_frexp_expf(scale_log2) + size - 6, -126), 126);
}

// 2^e of a normal number (in scalar registers where e is).
__device__ __forceinline__ float power_of_two(int e) {
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// What a row's products, in units of 2^unit, are multiplied with: the scale times log2 e
// (its sign went into Q) and the row's power of two; at least the smallest normal (-inf
// times it stays -inf where the scale is 0, and only nothing is less) and finite (a
// row of zeros).
__device__ __forceinline__ float positive_factor(float scale_log2, int exponent, int unit) {
    const float f = ldexpf(fabsf(scale_log2), max(min(exponent - 6 - unit, 1000), -1000));
    return fminf(fmaxf(f, 0x1p-126f), 0x1p126f);
}

// One sequence's lengths and mask: row i sees tokens below limit(i).
struct Kv4Mask {
    int n, rows, causal;   // tokens, query rows

    __device__ __forceinline__ int limit(int i) const {
        return causal ? min(n, i + 1 + n - rows) : n;
    }
};
__device__ __forceinline__ Kv4Mask sequence_mask(const int32_t *key_len, const int32_t *q_len,
                                                 int b, int L, int Lq, int causal) {
    return {optional_len(key_len, b, L), optional_len(q_len, b, Lq), causal};
}

// ---- 32x32x16 products (many rows)
__device__ __forceinline__ f32x16 mfma32x32x16f16(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32x32x2(float a, float b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// 16-byte pieces of LDS rows of N (4, 8 or 16) pieces and one of padding: 16
// rows read at the same piece fall on different banks, and a row's pieces are
// at constant offsets.
template <int N>
__device__ __forceinline__ int piece(int row, int p) {
    return row * (N + 1) + p;
}

// Maximum and sum over the wave.
__device__ __forceinline__ float max_of_wave(float v) {
    return max_xor32(max_xor16(max_of<16>(v)));
}
__device__ __forceinline__ float sum_of_wave(float v) {
    return sum_xor32(sum_xor16(sum_of<16>(v)));
}

// Token (of 32) in row i of a score product.
__device__ __forceinline__ int token_of(int i) {
    return (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1;
}

}  // namespace mg
