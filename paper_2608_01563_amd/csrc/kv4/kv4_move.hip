// kv4_move.hip -- rows into the 4-bit cache and back.
//
// A wave takes one octet of a head's tokens (8 positions that share V's words):
// lane 8e + c holds D/8 channels of token e.  A group's extremes are a
// reduction over the 4 or 8 lanes that hold it; K's words are the lane's own
// codes; V's gather the eight tokens of a channel, which three exchange steps
// over the lane's token bits do (half of the words change sides in each, so a
// lane ends with D/64 whole words).  Tokens of the octet that are not written
// keep their bits: their words are read, merged and written by this wave alone.
//
// Both directions are bound by HBM: 2 D elements and D + 8 max(1, D/64) cache
// bytes a token and head, with a few tens of vector instructions a value.
#include "kv4_device.h"
#include "kv4_launch.h"
#include "cdiv.h"

namespace mg {
namespace {

constexpr int kThreads = 256;

// Which positions a wave's octet holds.  Rows j in [0, n) become tokens at + j.
struct Octet {
    int bh, pos;        // head of the batch, first position
    int at, rows;       // start and number of the sequence's new rows
};
__device__ __forceinline__ bool take_octet(Octet *o, int B, int H, int n, int L, int octets,
                                           const int32_t *start, const int32_t *count) {
    const int64_t id = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    const int bh = (int)(id / octets), k = (int)(id - (int64_t)bh * octets);
    if (bh >= B * H) return false;
    const int b = bh / H;
    // clamped so that at + j cannot overflow; beyond these no row lands in [0, L)
    const int at = start == nullptr ? 0 : min(max(start[b], -n), L);
    o->bh = bh;
    o->at = at;
    o->rows = min(optional_len(count, b, n), L - at);
    o->pos = ((max(at, 0) >> 3) + k) << 3;
    return o->pos < at + o->rows;
}

// x + the value of the lane 8 away in its row of 16.
__device__ __forceinline__ uint32_t other8(uint32_t v) {
    return __builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false);   // row rotate by 8
}
// Both halves' words of a pair: lanes below end with x of both, above with y.
__device__ __forceinline__ uint32_t join32(uint32_t x, uint32_t y) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return r[0] | r[1];
}
__device__ __forceinline__ uint32_t join16(uint32_t x, uint32_t y) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    return r[0] | r[1];
}

// The code of t = x - mn for scale sc > 0 and inv = 1 / sc: the quotient in
// f32, and next to a border between two codes (ties are common among bf16
// values) the side it falls on in 64 bits, ties to the even code.
__device__ __forceinline__ uint32_t code_of(float x, float mn, float sc, float inv) {
    const float q = (x - mn) * inv;
    const float k = floorf(q), f = q - k;
    float code = k + (f > 0.5f ? 1.f : 0.f);
    if (fabsf(f - 0.5f) < 0x1p-16f) {
        const double over = __builtin_fma(-(double)sc, (double)k + 0.5, (double)x - (double)mn);
        code = k + (over > 0.0 || (over == 0.0 && ((int)k & 1)) ? 1.f : 0.f);
    }
    return (uint32_t)fminf(fmaxf(code, 0.f), 15.f);
}

// A lane's CH channels of one row: codes (0 where the lane holds no row) and,
// in the first lane of a group, the group's word.
template <int CH, int LANES>
__device__ __forceinline__ uint32_t quantise(const float (&x)[CH], uint32_t (&code)[CH]) {
    float lo = x[0], hi = x[0];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);   // fmin and fmax skip NaN
    }
#pragma unroll
    for (int m = 1; m < LANES; m *= 2) {
        lo = fminf(lo, __shfl_xor(lo, m, 64));
        hi = fmaxf(hi, __shfl_xor(hi, m, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
    }
    const uint32_t mb = f32_to_bf16_rne(lo);
    uint32_t sb = f32_to_bf16_rne((hi - lo) / 15.f);
    if (sb < 0x0080u) sb = 0;   // below the smallest normal
    const float mn = bf16_to_f32((uint16_t)mb), sc = bf16_to_f32((uint16_t)sb);
    const bool good = top < 0x7f800000u && fabsf(mn) < INFINITY && sc < INFINITY;
    if (!good || sb == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) code[i] = 0;
        return good ? mb : 0x7fc07fc0u;
    }
    const float inv = 1.f / sc;
#pragma unroll
    for (int i = 0; i < CH; ++i) code[i] = code_of(x[i], mn, sc, inv);
    return sb << 16 | mb;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void kv4_append(const T *__restrict__ K, const T *__restrict__ V, uint32_t *__restrict__ kw,
                uint32_t *__restrict__ vw, uint32_t *__restrict__ kp, uint32_t *__restrict__ vp,
                float *__restrict__ weight, const int32_t *__restrict__ start,
                const int32_t *__restrict__ count, int B, int H, int n, int L, int Lp,
                int octets) {
    constexpr int CH = D / 8, NG = Kv4Dim<D>::kGroups, LANES = 8 / NG;
    Octet o;
    if (!take_octet(&o, B, H, n, L, octets, start, count)) return;
    const int lane = threadIdx.x & 63, e = lane >> 3, c = lane & 7;
    const int p = o.pos + e, j = p - o.at;
    const bool there = j >= 0 && j < o.rows;   // rows are clamped to positions below L
    const size_t row = ((size_t)o.bh * n + (there ? j : 0)) * D + c * CH;
    float x[CH];
    uint32_t code[CH];

    // K: the lane's own words
    load_row(x, K + row);
    uint32_t word = quantise<CH, LANES>(x, code);
    const size_t tok = (size_t)o.bh * Lp + p;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < CH; ++i) w[i >> 3] |= code[i] << (4 * (i & 7));
    if (CH == 4) w[0] |= (uint32_t)__shfl_xor((int)w[0], 1, 64) << 16;   // even lanes: both halves
    if (there) {
        if (CH >= 8 || (c & 1) == 0) kw[tok * (D / 8) + k_word<D>(c * CH / 8)] = w[0];
        if (CH == 16) kw[tok * (D / 8) + k_word<D>(2 * c + 1)] = w[1];
        if (c % LANES == 0) kp[tok * NG + c / LANES] = word;
        if (weight != nullptr && c == 0) weight[(size_t)o.bh * L + p] = 0.f;
    }

    // V: a channel's eight tokens in one word
    load_row(x, V + row);
    word = quantise<CH, LANES>(x, code);
    if (there && c % LANES == 0) vp[tok * NG + c / LANES] = word;
    const uint32_t mask = there ? 0xfu << (4 * e) : 0u;
    uint32_t v[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) v[i] = (code[i] << (4 * e)) & mask;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) v[i] = join32(v[i], v[i + CH / 2]);
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) v[i] = join16(v[i], v[i + CH / 4]);
    uint32_t all = join32(mask, mask);
    all = join16(all, all);
    all |= other8(all);
    int ch = c * CH + (e >> 2) * (CH / 2) + ((e >> 1) & 1) * (CH / 4);
    constexpr int LEFT = CH / 4 > 1 ? CH / 8 : 1;
    if (CH / 4 > 1) {
        const bool up = e & 1;
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            const uint32_t keep = up ? v[i + LEFT] : v[i], give = up ? v[i] : v[i + LEFT];
            v[i] = keep | other8(give);
        }
        ch += up ? LEFT : 0;
    } else {
        v[0] |= other8(v[0]);
    }
    uint32_t *out = vw + ((size_t)o.bh * (Lp / 8) + o.pos / 8) * D;
    if (CH / 4 > 1 || (e & 1) == 0) {
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            uint32_t *at = out + v_word<D>(ch + i);
            *at = all == 0xffffffffu ? v[i] : (*at & ~all) | v[i];
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void kv4_read(const uint32_t *__restrict__ kw, const uint32_t *__restrict__ vw,
              const uint32_t *__restrict__ kp, const uint32_t *__restrict__ vp,
              T *__restrict__ K, T *__restrict__ V, const int32_t *__restrict__ start,
              const int32_t *__restrict__ count, int B, int H, int n, int L, int Lp, int octets) {
    constexpr int CH = D / 8, NG = Kv4Dim<D>::kGroups, LANES = 8 / NG;
    Octet o;
    if (!take_octet(&o, B, H, n, L, octets, start, count)) return;
    const int lane = threadIdx.x & 63, e = lane >> 3, c = lane & 7;
    const int p = o.pos + e, j = p - o.at;
    if (j < 0 || j >= o.rows) return;
    const size_t row = ((size_t)o.bh * n + j) * D + c * CH;
    const size_t tok = (size_t)o.bh * Lp + p;
    const uint32_t kg = kp[tok * NG + c / LANES], vg = vp[tok * NG + c / LANES];
    uint32_t w[2];
    w[0] = kw[tok * (D / 8) + k_word<D>(c * CH / 8)];
    if (CH == 16) w[1] = kw[tok * (D / 8) + k_word<D>(2 * c + 1)];
    if (CH == 4) w[0] >>= 16 * (c & 1);
    float x[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i)
        x[i] = fmaf(group_scale(kg), (float)(w[i >> 3] >> (4 * (i & 7)) & 15u), group_min(kg));
    store_row(K + row, x);
    const uint32_t *in = vw + ((size_t)o.bh * (Lp / 8) + p / 8) * D;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        x[i] = fmaf(group_scale(vg), (float)(in[v_word<D>(c * CH + i)] >> (4 * e) & 15u),
                    group_min(vg));
    store_row(V + row, x);
}

// Octets that n rows from any start can touch.
int octets_of(int n) { return cdiv(n, 8) + (n > 1 ? 1 : 0); }

unsigned groups_of(const Kv4Move &p) {
    return (unsigned)(((int64_t)p.B * p.H * octets_of(p.n) + kThreads / 64 - 1) / (kThreads / 64));
}

template <typename T, int D>
hipError_t append(const Kv4Move &p, const void *K, const void *V, const Kv4Cache<uint32_t> &c,
                  float *weight, hipStream_t s) {
    kv4_append<T, D><<<groups_of(p), kThreads, 0, s>>>(
        static_cast<const T *>(K), static_cast<const T *>(V), c.k, c.v, c.kp, c.vp, weight,
        p.start, p.count, p.B, p.H, p.n, p.L, kv4_padded(p.L), octets_of(p.n));
    return hipGetLastError();
}

template <typename T, int D>
hipError_t read(const Kv4Move &p, const Kv4Cache<const uint32_t> &c, void *K, void *V,
                hipStream_t s) {
    kv4_read<T, D><<<groups_of(p), kThreads, 0, s>>>(
        c.k, c.v, c.kp, c.vp, static_cast<T *>(K), static_cast<T *>(V), p.start, p.count, p.B,
        p.H, p.n, p.L, kv4_padded(p.L), octets_of(p.n));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Move &p, const void *K, const void *V, bool bf16,
                             const Kv4Cache<uint32_t> &c, float *weight, hipStream_t s) {
    if (bf16)
        return p.d == 32 ? append<uint16_t, 32>(p, K, V, c, weight, s)
             : p.d == 64 ? append<uint16_t, 64>(p, K, V, c, weight, s)
                         : append<uint16_t, 128>(p, K, V, c, weight, s);
    return p.d == 32 ? append<float, 32>(p, K, V, c, weight, s)
         : p.d == 64 ? append<float, 64>(p, K, V, c, weight, s)
                     : append<float, 128>(p, K, V, c, weight, s);
}

hipError_t launch_kv4_read(const Kv4Move &p, const Kv4Cache<const uint32_t> &c, void *K, void *V,
                           bool bf16, hipStream_t s) {
    if (bf16)
        return p.d == 32 ? read<uint16_t, 32>(p, c, K, V, s)
             : p.d == 64 ? read<uint16_t, 64>(p, c, K, V, s)
                         : read<uint16_t, 128>(p, c, K, V, s);
    return p.d == 32 ? read<float, 32>(p, c, K, V, s)
         : p.d == 64 ? read<float, 64>(p, c, K, V, s)
                     : read<float, 128>(p, c, K, V, s);
}

}  // namespace mg
