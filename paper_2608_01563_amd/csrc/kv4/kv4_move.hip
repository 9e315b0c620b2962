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
// Either way moves 2 D elements and D + 8 max(1, D/64) cache bytes a token and head.
// 4 x 8 heads of up to 8,192 bf16 tokens of 128 channels (108 MB each way): 22 us read
// back, 4.9 TB/s, and 134 MB of f32 25 us, 5.9 TB/s: bound by HBM.  Written in 29 us,
// 3.7 TB/s: the 700 vector instructions of an octet take some 70 % of a SIMD's issue
// time beside it.  A wave an octet, because V's words then have one writer and rows are
// read whole.
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
    // (fewer than 2^28 octets)
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t id = blockIdx.x * (kThreads / 64) + wave;
    const int bh = (int)(id / (uint32_t)octets), k = (int)(id - (uint32_t)bh * octets);
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

// A lane holds PIECES pieces of PIECE consecutive channels of its token, piece i at
// channel (8 i + c) PIECE: the eight lanes of a token read and write 128 (d = 32
// bf16: 64) consecutive bytes at a time.
template <typename T, int D>
struct Pieces {
    static constexpr int PIECE = 16 / (int)sizeof(T) < D / 8 ? 16 / (int)sizeof(T) : D / 8;
    static constexpr int PIECES = D / 8 / PIECE, NG = Kv4Dim<D>::kGroups;
    static_assert(PIECES % NG == 0, "a piece index belongs to one group");
    static constexpr int PER = PIECES / NG;   // pieces a group

    static __device__ __forceinline__ int channel(int i, int c) { return (8 * i + c) * PIECE; }
};

// Codes of a lane's pieces of one row, each plus the bits of kRound, and the groups'
// words; all codes 0 where the lane holds no row.
//
// code = round((x - min) / scale): the quotient of the f32 difference, correctly
// rounded (a product with 1 / scale, at most 2^125 and normal, to an ulp or so, and
// one exact residual), so that ties, which are common among bf16 values, go to the
// even code when kRound is added.  A bf16
// difference is exact unless x and min are 2^16 apart.  f32 values within 2^-20 of a
// border are settled exactly, with the rounding error of the difference.
constexpr float kRound = 0x1p23f;   // ulp 1: adding it rounds, the code is in the low bits
constexpr uint32_t kRoundBits = 0x4b000000u;
constexpr float kFifteenth = 1.f / 15.f;

template <typename T, int D>
__device__ __forceinline__ void quantise(const float (&x)[Pieces<T, D>::PIECES][Pieces<T, D>::PIECE],
                                         uint32_t (&code)[Pieces<T, D>::PIECES][Pieces<T, D>::PIECE],
                                         uint32_t (&word)[Kv4Dim<D>::kGroups], bool there) {
    using P = Pieces<T, D>;
    // minimum and maximum of numbers, NaN where one is NaN
    const auto least = [](float a, float b) { return __builtin_elementwise_minimum(a, b); };
    const auto most = [](float a, float b) { return __builtin_elementwise_maximum(a, b); };
#pragma unroll
    for (int g = 0; g < P::NG; ++g) {
        float lo = x[g * P::PER][0], hi = lo;
#pragma unroll
        for (int i = g * P::PER; i < (g + 1) * P::PER; ++i)
#pragma unroll
            for (int k = 0; k < P::PIECE; k += 2) {
                lo = least(least(lo, x[i][k]), x[i][k + 1]);
                hi = most(most(hi, x[i][k]), x[i][k + 1]);
            }
        lo = least(lo, other_lane<0>(lo));
        hi = most(hi, other_lane<0>(hi));
        lo = least(lo, other_lane<1>(lo));
        hi = most(hi, other_lane<1>(hi));
        lo = least(lo, other_lane<2>(lo));
        hi = most(hi, other_lane<2>(hi));
        const uint32_t mb = to_bf16(lo);
        // a fifteenth, correctly rounded as above; NaN or infinite where a value is
        const float wide = hi - lo, part = wide * kFifteenth;
        uint32_t sb = to_bf16(wide < INFINITY ? fmaf(fmaf(-15.f, part, wide), kFifteenth, part)
                                              : wide);
        if (sb < 0x0080u) sb = 0;   // below the smallest normal
        const float mn = bf16_to_f32((uint16_t)mb), sc = bf16_to_f32((uint16_t)sb);
        const bool good = fabsf(mn) < INFINITY && sc < INFINITY;
        const bool flat = !good || sb == 0 || !there;
        const float inv = flat ? 0.f : __builtin_amdgcn_rcpf(sc), from = flat ? 0.f : mn;
        word[g] = good ? sb << 16 | mb : 0x7fc07fc0u;
#pragma unroll
        for (int i = g * P::PER; i < (g + 1) * P::PER; ++i)
#pragma unroll
            for (int k = 0; k < P::PIECE; ++k) {
                const float t = x[i][k] - from, q0 = t * inv;
                float q = fmaf(fmaf(-sc, q0, t), inv, q0);
                if (sizeof(T) == 4) {
                    if (fabsf(q - rintf(q)) > 0.5f - 0x1p-20f) {
                        const float f = floorf(q), b = t - x[i][k];
                        const float lost = (x[i][k] - (t - b)) - (from + b);   // t + lost = x - min
                        const float over = (t - sc * (f + 0.5f)) + lost;       // both exact
                        q = f + (over > 0.f || (over == 0.f && ((int)f & 1)) ? 1.f : 0.f);
                    }
                }
                // (NaN: 0)
                code[i][k] = __float_as_uint(__builtin_amdgcn_fmed3f(q, 0.f, 15.f) + kRound);
            }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void kv4_append(const T *__restrict__ K, const T *__restrict__ V, uint32_t *__restrict__ kw,
                uint32_t *__restrict__ vw, uint32_t *__restrict__ kp, uint32_t *__restrict__ vp,
                float *__restrict__ weight, const int32_t *__restrict__ start,
                const int32_t *__restrict__ count, int B, int H, int n, int L, int Lp,
                int octets) {
    using P = Pieces<T, D>;
    constexpr int CH = D / 8, NG = P::NG, PIECE = P::PIECE;
    Octet o;
    if (!take_octet(&o, B, H, n, L, octets, start, count)) return;
    const int lane = threadIdx.x & 63, e = lane >> 3, c = lane & 7;
    const int p = o.pos + e, j = p - o.at;
    const bool there = j >= 0 && j < o.rows;   // rows are clamped to positions below L
    const size_t row = ((size_t)o.bh * n + (there ? j : 0)) * D;
    float x[P::PIECES][PIECE], y[P::PIECES][PIECE];
    uint32_t code[P::PIECES][PIECE], word[NG];
#pragma unroll
    for (int i = 0; i < P::PIECES; ++i) load_row(x[i], K + row + P::channel(i, c));
#pragma unroll
    for (int i = 0; i < P::PIECES; ++i) load_row(y[i], V + row + P::channel(i, c));

    // K: words of 8 channels, a lane's own or, of 4 each, with its neighbour
    quantise<T, D>(x, code, word, there);
    const size_t tok = (size_t)o.bh * Lp + p;
#pragma unroll
    for (int i = 0; i < P::PIECES; ++i) {
        // sums of codes at their places; kRoundBits' own sum is taken off first
        uint32_t w = 0u - kRoundBits - (kRoundBits << 4);
#pragma unroll
        for (int k = 0; k < PIECE; ++k) w += code[i][k] << (4 * k);
        if (PIECE == 4) w |= (uint32_t)__shfl_xor((int)w, 1, 64) << 16;   // in even lanes
        if (there && (PIECE == 8 || (c & 1) == 0))
            kw[tok * (D / 8) + k_word<D>(P::channel(i, c) / 8)] = w;
    }
    if (there && c == 0) {
#pragma unroll
        for (int g = 0; g < NG; ++g) kp[tok * NG + g] = word[g];
        if (weight != nullptr) weight[(size_t)o.bh * L + p] = 0.f;
    }

    // V: a channel's eight tokens in one word
    quantise<T, D>(y, code, word, there);
    if (there && c == 0) {
#pragma unroll
        for (int g = 0; g < NG; ++g) vp[tok * NG + g] = word[g];
    }
    const uint32_t place = 4u * e, off = 0u - (kRoundBits << place);
    uint32_t v[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) v[i] = (code[i / PIECE][i % PIECE] << place) + off;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) v[i] = join32(v[i], v[i + CH / 2]);
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) v[i] = join16(v[i], v[i + CH / 4]);
    const uint64_t rows = __ballot(there);
    uint32_t all = 0;   // nibbles written
#pragma unroll
    for (int k = 0; k < 8; ++k) all |= (rows >> (8 * k) & 1) ? 0xfu << (4 * k) : 0u;
    int at = (e >> 2) * (CH / 2) + ((e >> 1) & 1) * (CH / 4);   // the first word's place of CH
    constexpr int LEFT = CH / 4 > 1 ? CH / 8 : 1;
    if (CH / 4 > 1) {
        const bool up = e & 1;
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            const uint32_t keep = up ? v[i + LEFT] : v[i], give = up ? v[i] : v[i + LEFT];
            v[i] = keep | other8(give);
        }
        at += up ? LEFT : 0;
    } else {
        v[0] |= other8(v[0]);
    }
    uint32_t *out = vw + ((size_t)o.bh * (Lp / 8) + o.pos / 8) * D;
    if (CH / 4 > 1 || (e & 1) == 0) {
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            const int ch = P::channel((at + i) / PIECE, c) + (at + i) % PIECE;
            uint32_t *to = out + v_word<D>(ch);
            *to = all == 0xffffffffu ? v[i] : (*to & ~all) | v[i];
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void kv4_read(const uint32_t *__restrict__ kw, const uint32_t *__restrict__ vw,
              const uint32_t *__restrict__ kp, const uint32_t *__restrict__ vp,
              T *__restrict__ K, T *__restrict__ V, const int32_t *__restrict__ start,
              const int32_t *__restrict__ count, int B, int H, int n, int L, int Lp, int octets) {
    using P = Pieces<T, D>;
    constexpr int NG = P::NG, PIECE = P::PIECE;
    Octet o;
    if (!take_octet(&o, B, H, n, L, octets, start, count)) return;
    const int lane = threadIdx.x & 63, e = lane >> 3, c = lane & 7;
    const int p = o.pos + e, j = p - o.at;
    if (j < 0 || j >= o.rows) return;
    const size_t row = ((size_t)o.bh * n + j) * D;
    const size_t tok = (size_t)o.bh * Lp + p;
    const uint32_t *in = vw + ((size_t)o.bh * (Lp / 8) + p / 8) * D;
    uint32_t kg[NG], vg[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        kg[g] = kp[tok * NG + g];
        vg[g] = vp[tok * NG + g];
    }
#pragma unroll
    for (int i = 0; i < P::PIECES; ++i) {
        const int ch = P::channel(i, c), g = i / P::PER;
        const uint32_t w = kw[tok * (D / 8) + k_word<D>(ch / 8)] >> (4 * (ch & 7));
        float x[PIECE], y[PIECE];
#pragma unroll
        for (int k = 0; k < PIECE; ++k) {
            x[k] = fmaf(group_scale(kg[g]), (float)(w >> (4 * k) & 15u), group_min(kg[g]));
            y[k] = fmaf(group_scale(vg[g]), (float)(in[v_word<D>(ch + k)] >> (4 * e) & 15u),
                        group_min(vg[g]));
        }
        store_row(K + row + ch, x);
        store_row(V + row + ch, y);
    }
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
