// kv4_many.hip -- attention over the 4-bit cache for many query rows (bf16).
//
// Where kv4_rows.hip has every wave unpack the codes it multiplies, here a
// workgroup of 256 rows unpacks a tile of 64 tokens once into LDS and
// all of its waves read it there (32x32x16 products, 32 rows a wave):
//
//   K   codes as f16, exact; scores are scaled and shifted a group at a time as
//       in kv4_tile.h, the minima's part by one f32 product over the groups
//   V   values v 2^(15-E) rounded to f16 (within 2^-11), E bounding all values
//       so far, so that one product per 16 tokens covers scale and minimum;
//       rows that see a tile in part, and of its values only some that are
//       2^kFar below its E, are computed anew in kv4_sweep.h's form, whose
//       bounds are a row's own (a call with such rows in every tile takes about
//       twice as long, with one token so far above the others no longer at 8,192)
//   P   f16, at most 2^15
//
// The row order of the score product swaps bits 2 and 3 of the token, which
// leaves a lane with whole octets of tokens: V's words (8 tokens of a channel)
// become 16-byte LDS pieces that the second product reads as they are.
//
// A tile's words are loaded an iteration before they are unpacked, and its
// group words one before that, because unpacking V needs them from LDS.
//
// 2 x 32 heads, 2,048 rows over 8,192 tokens of 128 channels, causal: 578 us, 833
// TFLOP/s where a large bf16 product reaches 1,206.  The matrix units are busy 40 %
// of the time and the vector units 55 %, hardly at once; operand reads from LDS cost
// the most of the rest (without them 475 of then 603 us; without unpacking 570, without
// the exponentials 590).  Bounds that leave out what a row does not see, and a unit of K
// for the workgroup's rows, cost 4 us of it.  32x32 products, because they read half as
// much of LDS for their work as 16x16 ones.
#include "cdiv.h"
#include "kv4_launch.h"
#include "kv4_sweep.h"

namespace mg {
namespace {

constexpr int kTokens = 64, kManyWaves = 8, kRows = 32 * kManyWaves;
constexpr float kManySlack = 4.f;
constexpr int kLift = 11;      // P is at most 2^(slack + kLift) = 2^15
constexpr int kManyExp = -100; // least E
constexpr int kFar = 12;       // V's f16 parts are then off by 2^-22 of the largest at most
constexpr int kNone = -1000;   // exponent of nothing but zeros
constexpr int kLeap = 60;      // E may move by this in one tile before f32 sums lose bits
constexpr int kFarTiles = 8;   // tiles in or just before which 128 rows can end, twice

struct ManyArgs {
    const uint16_t *Q;
    const uint32_t *kw, *vw, *kp, *vp;
    uint16_t *O;
    float *LSE, *part, *stat;
    const int32_t *key_len, *q_len;
    int H, G, Lq, L, Lp, causal;
    float scale_log2;
    int splits, row_tiles;
};

// What a workgroup and its wave w work on.
struct ManyPlace {
    int bh, split, G, rows;   // head, share of the tokens, query heads and rows of the head
    Kv4Mask mask;
    int front, back, r0;      // first row in front, at the back, of the wave
    int front_end, back_end;  // tokens that these rows see
    int begin, stop;          // tiles

    // tokens that some of the rows from, ..., from + n - 1 sees
    __device__ __forceinline__ int end_of(int from, int n) const {
        return from < rows && from / G < mask.rows
            ? max(mask.limit(min((min(rows, from + n) - 1) / G, mask.rows - 1)), 0) : 0;
    }
};
__device__ __forceinline__ ManyPlace many_place(const ManyArgs &a, int id, int w) {
    ManyPlace p;
    const int share = id / a.row_tiles, tile = id - share * a.row_tiles;
    p.bh = share / a.splits;
    p.split = share - p.bh * a.splits;
    p.G = a.G;
    p.rows = a.G * a.Lq;
    p.mask = sequence_mask(a.key_len, a.q_len, p.bh / a.H, a.L, a.Lq, a.causal);
    // Four waves take rows from the front and four from the back: causal
    // workgroups differ less in work, the first ones having the most.
    p.front = kRows / 2 * tile;
    p.back = kRows / 2 * (2 * a.row_tiles - 1 - tile);
    p.r0 = w < kManyWaves / 2 ? p.front + 32 * w : p.back + 32 * (w - kManyWaves / 2);
    p.front_end = p.end_of(p.front, kRows / 2);
    p.back_end = p.end_of(p.back, kRows / 2);
    const int tiles = (max(p.front_end, p.back_end) + kTokens - 1) / kTokens;
    const int each = (tiles + a.splits - 1) / a.splits;
    p.begin = p.split * each;
    p.stop = min(tiles, p.begin + each);
    return p;
}

// 32 query rows as operands of 32x32x16 products: lane column l%32, channels
// 16s + 8(l/32) + e, in the slots of code_operand.
template <int D>
struct Query32 {
    f16x8 q[D / 16];
    float sum;      // of group l/32 (0 where there is no second)
    int exponent, size;   // as in Kv4Query

    __device__ __forceinline__ void load(const uint16_t *row, bool valid, int h, bool negate) {
        constexpr int NS = D / 16, NG = Kv4Dim<D>::kGroups;
        float x[NS][8];
        float top = 0.f;
#pragma unroll
        for (int s = 0; s < NS; ++s) load_row(x[s], row + 16 * s + 8 * h);   // a row that is there
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[s][e] = valid ? x[s][e] : 0.f;
                top = fmaxf(top, fabsf(x[s][e]));
                if (negate) x[s][e] = -x[s][e];
            }
        exponent = query_exponent(max_xor32(top), &size);
        float each[2] = {0.f, 0.f};
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
            float t = 0.f;
#pragma unroll
            for (int s = gr * (NS / NG); s < (gr + 1) * (NS / NG); ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) t += ldexpf(x[s][e], -exponent);
            each[gr] = sum_xor32(t) * 0x1p6f;
        }
        sum = h == 0 ? each[0] : each[1];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            f16x8 part[1];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = ldexpf(x[s][e], 15 - exponent);
            split_operand<1>(part, x[s]);
            q[s] = part[0];
        }
    }
};

// Rows first .. first + 15 of a head over blocks begin .. stop - 1 of 32 tokens, in the
// form of few rows, by one wave.
template <int D>
__device__ __forceinline__ void anew(const ManyArgs &a, int bh, int split, int first, int begin,
                                     int stop, const Kv4Mask &mask,
                                     BlockGroups<Kv4Dim<D>::kGroups> &groups, int lane) {
    constexpr int NG = Kv4Dim<D>::kGroups, NB = Kv4Dim<D>::kBlocks;
    const int c = lane & 15, g = lane >> 4, rows = a.G * a.Lq;
    const int r = first + c;
    const bool in = r < rows;
    const RowAt at = row_at(in ? r : rows - 1, bh, a.G, a.Lq);
    const size_t head = (size_t)bh * a.Lp;
    Kv4Query<D, 1> q;
    q.load(a.Q + at.at * D, in && at.i < mask.rows, g, a.scale_log2 < 0.f);
    const auto factors = Kv4Sweep<D, 1>::factors(q, a.scale_log2, lane);
    const int limit = mask.limit(at.i), all = mask.limit(first / a.G);
    Kv4Sweep<D, 1> sweep;
#pragma unroll 1
    for (int block = begin; block < stop; ++block) {
        Kv4Keys<D> key;
        Kv4Values<D> val;
        Kv4GroupWords<NG> words;
        key.load(a.kw + head * (D / 8), block, c, g);
        val.load(a.vw + head / 8 * D, block, c, g);
        words.load(a.kp + head * NG, a.vp + head * NG, block, lane);
        sweep.step(block, q, factors, limit, all, mask.n, key, val, words, groups, lane,
                   [](const f32x4(&)[2]) {});
    }
    sweep.finish();
    if (!in) return;
    const bool valid = at.i < mask.rows;
    if (a.splits > 1) {
        const size_t slot = ((size_t)bh * a.splits + split) * rows + r;
#pragma unroll
        for (int b = 0; b < NB; ++b)
            *reinterpret_cast<f32x4 *>(a.part + slot * D + 16 * b + 4 * g) =
                valid ? sweep.o[b] : zero4();
        if (g == 0) {
            a.stat[2 * slot] = valid ? sweep.m : -INFINITY;
            a.stat[2 * slot + 1] = valid ? sweep.l : 0.f;
        }
        return;
    }
    const float l = valid ? sweep.l : 0.f, inv = 1.f / l;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = l == 0.f ? 0.f : sweep.o[b][k] * inv;
        store_row(a.O + at.at * D + 16 * b + 4 * g, x);
    }
    if (g == 0) a.LSE[at.at] = l != l ? l : row_lse(sweep.m, l);
}

// Those of the wave's rows in `which` anew, by halves of 16.  Last of all and from the
// kernel's arguments, which are read again: with all that this needs kept through the
// tile loop, scalars had to move to vector registers and back there (16 heads of 16,384
// rows over 4,096 tokens of 128 channels: 462 us, so 457, and 451 without this part).
template <int D>
__device__ __forceinline__ void far_rows(uint32_t which, int w, int lane, void *lds) {
    typedef const __attribute__((address_space(4))) ManyArgs *Arguments;
    Arguments p = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
    uint32_t id = blockIdx.x;
    asm volatile("" : "+s"(p), "+s"(id));
    const ManyArgs a = {p->Q, p->kw, p->vw, p->kp, p->vp, p->O, p->LSE, p->part, p->stat,
                        p->key_len, p->q_len, p->H, p->G, p->Lq, p->L, p->Lp, p->causal,
                        p->scale_log2, p->splits, p->row_tiles};
    const ManyPlace at = many_place(a, id, w);
    auto &groups = static_cast<BlockGroups<Kv4Dim<D>::kGroups> *>(lds)[w];
#pragma unroll 1
    for (int half = 0; half < 2; ++half)
        if (which >> (16 * half) & 0xffffu) {
            const int first = at.r0 + 16 * half;
            anew<D>(a, at.bh, at.split, first, 2 * at.begin,
                    min(2 * at.stop, (at.end_of(first, 16) + 31) / 32), at.mask, groups, lane);
        }
}

template <int D>
__global__ __launch_bounds__(64 * kManyWaves) __attribute__((amdgpu_waves_per_eu(2, 8)))
void kv4_many(ManyArgs a) {
    constexpr int NG = Kv4Dim<D>::kGroups, NS = D / 16, NB = D / 32, KR = D / 8;
    constexpr int T = 64 * kManyWaves, WORDS = kTokens * D / 8;
    constexpr int N = WORDS / T < 1 ? 1 : WORDS / T;   // words a thread unpacks
    __shared__ __attribute__((aligned(16))) f16x8 Ks[2][kTokens * (KR + 1)];
    __shared__ __attribute__((aligned(16))) f16x8 Vs[3][D * 9];
    __shared__ __attribute__((aligned(16))) float Ksc[4][NG][kTokens];
    __shared__ float Kmn[4][2][kTokens];
    __shared__ __attribute__((aligned(16))) _Float16 Vsc[4][NG][kTokens], Vmn[4][NG][kTokens];
    __shared__ uint64_t Bad[4][NG];   // tokens whose V is not finite
    __shared__ int Es[4], Sizes[kManyWaves];
    __shared__ int FarCount, Far[kFarTiles][2];   // rows with limits in (first, second]
    __shared__ int Ends[4];   // first and last limit of the rows in front, and at the back

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const ManyPlace place = many_place(a, blockIdx.x, w);
    const Kv4Mask mask = place.mask;
    const int bh = place.bh, split = place.split, rows = place.rows;
    const int begin = place.begin, stop = place.stop;

    const int r0 = place.r0, r = r0 + c;
    const bool in = r < rows;
    const int rr = in ? r : rows - 1, i = rr / a.G;
    const size_t at = ((size_t)bh * a.G + (rr - i * a.G)) * a.Lq + i;
    const int limit = mask.limit(i);
    // tokens that some row of the wave, every row of the wave sees
    const int wave_end = place.end_of(r0, 32);
    const int wave_all = r0 < rows ? mask.limit(r0 / a.G) : 0;
    if (tid == 64) {   // for wave 1, seldom
        FarCount = 0;
        Ends[0] = place.front < rows ? mask.limit(place.front / a.G) : INT32_MAX;
        Ends[1] = place.front_end;
        Ends[2] = place.back < rows ? mask.limit(place.back / a.G) : INT32_MAX;
        Ends[3] = place.back_end;
    }
    __builtin_amdgcn_wave_barrier();   // one wave's LDS accesses stay in order

    const size_t head = (size_t)bh * a.Lp;
    const uint32_t *kw = a.kw + head * KR, *vw = a.vw + head / 8 * D;
    const uint32_t *kp = a.kp + head * NG, *vp = a.vp + head * NG;

    // ---- bringing tiles in
    typedef uint32_t words __attribute__((ext_vector_type(N)));
    const bool brings = WORDS >= T * N || tid * N < WORDS;
    const int ktok = tid * N / KR, kat = tid * N % KR;     // K: token, first word
    const int voct = tid * N / D, vat = tid * N % D;       // V: octet, first word
    words kraw, vraw;
    uint32_t params[NG];   // wave 0: K's, wave 1: V's, of token `lane`
    auto load_words = [&](int t) {
        if (!brings) return;
        // past the padded end (which no row sees) the last block again
        const int k = min(kTokens * t + ktok, a.Lp - 1);
        const int o = min(8 * t + voct, a.Lp / 8 - 1);
        kraw = *reinterpret_cast<const words *>(kw + (size_t)k * KR + kat);
        vraw = *reinterpret_cast<const words *>(vw + (size_t)o * D + vat);
    };
    auto load_params = [&](int t) {
        const int k = kTokens * t + lane;
        const uint32_t *p = w == 0 ? kp : vp;
#pragma unroll
        for (int g = 0; g < NG; ++g)
            params[g] = w < 2 && k < mask.n ? p[(size_t)k * NG + g] : 0u;
    };
    float unit = 1.f;   // of K's groups, in wave 0
    // in wave 1: E, the same of what was not 0, and how many Far tiles there are
    int bound = kManyExp, known = kNone, far_tiles = 0;
    // whether [from, to] holds the limit of a row of the workgroup
    auto limits_in = [&](int from, int to) {
        return max(Ends[0], from) <= min(Ends[1], to) || max(Ends[2], from) <= min(Ends[3], to);
    };
    auto put_params = [&](int t) {
        const int b = t & 3;
        if (w == 0) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                Ksc[b][g][lane] = group_scale(params[g]) * unit;
                Kmn[b][g][lane] = group_min(params[g]) * unit;
            }
            if (NG == 1) Kmn[b][1][lane] = 0.f;
        } else if (w == 1) {
            float size = 0.f;
            bool good[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const float sc = group_scale(params[g]), mn = group_min(params[g]);
                const float v = fmaxf(fabsf(mn), fabsf(fmaf(15.f, sc, mn)));
                good[g] = v < INFINITY;
                size = fmaxf(size, good[g] ? v : 0.f);
                const uint64_t bad = __ballot(!good[g]);
                if (lane == 0) Bad[b][g] = bad;
            }
            const float most = max_of_wave(size);
            if (most > 0.f) bound = max(bound, __builtin_amdgcn_frexp_expf(most));
            if (lane == 0) Es[b] = bound;
            if (__any(bound > known + kFar)) {   // (the same in all lanes)
                // Rows that see nothing of the tile from its first value near E on, if they
                // see a value other than 0; after a leap also what a wave that works on
                // the tile has of rows that end before it.
                const int at = kTokens * t;
                const bool some = known != kNone, leap = some && bound > known + kLeap;
                const int own = max(__builtin_amdgcn_frexp_expf(size), kManyExp);
                const int from = leap ? at - 32 : at;
                const int near = __builtin_ctzll(__ballot(size > 0.f && own + kFar >= bound) |
                                                 1ull << 63);
                const bool seen = some || (__ballot(size > 0.f) & ((1ull << near) - 1)) != 0;
                if (seen && t < stop && limits_in(from + 1, at + near) && far_tiles < kFarTiles) {
                    if (lane == 0) {
                        Far[far_tiles][0] = from;
                        Far[far_tiles][1] = at + near;
                        FarCount = far_tiles + 1;
                    }
                    ++far_tiles;
                }
            }
            if (most > 0.f) known = bound;
            // in the octet's slot order
            const int slot = (lane & 0x38) | (lane & 1) << 2 | (lane & 6) >> 1;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                Vsc[b][g][slot] = (_Float16)(good[g] ? ldexpf(group_scale(params[g]), 15 - bound)
                                                     : 0.f);
                Vmn[b][g][slot] = (_Float16)(good[g] ? ldexpf(group_min(params[g]), 15 - bound)
                                                     : 0.f);
            }
        }
    };
    auto put_words = [&](int t, int vb) {   // vb: V's buffer
        if (!brings) return;
        const int b = t & 1;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int at_ = kat + n;   // g * (D/32) + s holds channels 8 (4s + g)
            const int p = 4 * (at_ % (D / 32)) + at_ / (D / 32);
            Ks[b][piece<KR>(ktok, p)] = code_operand(N == 1 ? kraw[0] : kraw[n]);
        }
        constexpr int W = Kv4Dim<D>::kWide;
        const int g = NG == 1 ? 0 : vat / 64;
        const f16x8 sc = *reinterpret_cast<const f16x8 *>(&Vsc[t & 3][g][8 * voct]);
        const f16x8 mn = *reinterpret_cast<const f16x8 *>(&Vmn[t & 3][g][8 * voct]);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int q = vat + n;
            const int d = 16 * (W * (q / (16 * W)) + q % W) + q / W % 16;
            Vs[vb][piece<8>(d, voct)] =
                __builtin_elementwise_fma(code_operand<512>(N == 1 ? vraw[0] : vraw[n]), sc, mn);
        }
    };

    Query32<D> q;
    // (rows behind the sequence's, whatever they hold, are taken as zeros)
    q.load(a.Q + at * D, in && i < mask.rows, h, a.scale_log2 < 0.f);
    float factor = 0.f;
    float m = -INFINITY, l = 0.f;
    int E = kManyExp;
    f32x16 o[NB];   // O^T[32 b + 8 (v/4) + 4h + v%4][row c] 2^(kLift + 15 - E)
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = zero16();

    // Scores over the row's factor of 32 tokens, register v being token
    // 8 (2 (v/8) + h) + v%8 of the block; -inf where the row does not see it.
    f32x16 part[NG], val;
    auto key_at = [&](int t, int kb, int st) {
        return Ks[t & 1][piece<KR>(32 * kb + token_of(c), 2 * st + h)];
    };
    auto scale_at = [&](int t, int kb, int g, int u) {
        return *reinterpret_cast<const f32x4 *>(
            &Ksc[t & 3][g][32 * kb + 16 * (u >> 1) + 8 * h + 4 * (u & 1)]);
    };
    auto low_at = [&](int t, int kb) { return Kmn[t & 3][h][32 * kb + token_of(c)]; };
    auto hide = [&](int t, int kb) {
        if (kTokens * t + 32 * (kb + 1) > wave_all) {
            const int left = limit - kTokens * t - 32 * kb - 8 * h;
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (16 * (v >> 3) + (v & 7) >= left) val[v] = -INFINITY;
        }
    };
    // Running units that hold scores up to mx and tile t's values.
    auto settle = [&](int t, float mx) {
        mx = max_xor32(mx) * factor;
        const int e_new = __builtin_amdgcn_readfirstlane(Es[t & 3]);
        if (__any(mx > m + kManySlack) || e_new != E) {
            const float m_new = fmaxf(m, ceilf(mx));
            const float alpha = m_new == -INFINITY ? 1.f : exp2_fast(m - m_new);
            l *= alpha;
            const float both = ldexpf(alpha, E - e_new);
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= both;
            m = m_new;
            E = e_new;
        }
    };
    // One block: softmax and P V of the scores in `val` (block kb of tile t, V in
    // buffer vb), and meanwhile the scores of the next one (kn of tile tn).
    // The order is written out: operand reads AHEAD of the products that take
    // them, the softmax between the score products, the sums of the new scores
    // between P V's.  (Left to itself the compiler reads each operand right
    // before its product: 757 against 601 us for 2,048 rows over 8,192 tokens.)
    constexpr int AHEAD = NS < 4 ? NS : 4;
    auto step = [&](int t, int kb, int vb, int tn, int kn) {
        auto value_at = [&](int k) {   // product k of P V: tokens k / NB, channels k % NB
            return Vs[vb][piece<8>(32 * (k % NB) + c, 4 * kb + 2 * (k / NB) + h)];
        };
        f16x8 reg[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) reg[k] = key_at(tn, kn, k);
        const float low_next = low_at(tn, kn);
        auto score_product = [&](int k) {
            const int g = k / (NS / NG);
            if (k % (NS / NG) == 0) part[g] = zero16();
            part[g] = mfma32x32x16f16(reg[k % AHEAD], q.q[k], part[g]);
            reg[k % AHEAD] = k + AHEAD < NS ? key_at(tn, kn, k + AHEAD) : value_at(k + AHEAD - NS);
        };
        // before a wave that unpacks (582 us without, 570)
        __builtin_amdgcn_s_setprio(1);
        // half of the score products hide the maximum ...
        constexpr int HALF = NS / 2, EACH = 16 / HALF;
        float mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < HALF; ++k) {
            score_product(k);
#pragma unroll
            for (int v = k * EACH; v < (k + 1) * EACH; v += 2) mx = max3_f32(mx, val[v], val[v + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        settle(t, mx);
        // ... the other half the exponentials
        const float off = (float)kLift - (m == -INFINITY ? 0.f : m);
        float x[16];
        f16x8 p[2];
#pragma unroll
        for (int k = 0; k < HALF; ++k) {
            score_product(HALF + k);
#pragma unroll
            for (int i = k * EACH; i < (k + 1) * EACH; ++i) {
                x[i] = exp2_fast(fmaf(val[(i & 8) + slot_value(i & 7)], factor, off));
                p[i >> 3][i & 7] = (_Float16)x[i];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // P V, and behind it first the row sums, then, from product FIRST on (the
        // minima's product takes 64 clocks), the new scores, a group of four at a time
        constexpr int SUMS = 4 * NG, FIRST = NS < 8 ? 1 : 2;
        auto sums_before = [](int k) {   // of the SUMS, done before slice k
            return k <= FIRST ? 0 : (k - FIRST) * SUMS / (NS - FIRST);
        };
        constexpr int MOST = (SUMS + NS - FIRST - 1) / (NS - FIRST);
        f32x4 sc[MOST];
        val = mfma32x32x2(low_next, q.sum, zero16());
#pragma unroll
        for (int k = 0; k < NS; ++k) {
            o[k % NB] = mfma32x32x16f16(reg[k % AHEAD], p[k / NB], o[k % NB]);
            const int now = sums_before(k), next = sums_before(k + 1), after = sums_before(k + 2);
#pragma unroll
            for (int i = now; i < next; ++i) {
                const int g = i % NG, u = i / NG;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    val[4 * u + r] = fmaf(part[g][4 * u + r], sc[i - now][r], val[4 * u + r]);
            }
#pragma unroll
            for (int i = next; i < (k + 1 < NS ? after : next); ++i)
                sc[i - next] = scale_at(tn, kn, i % NG, i / NG);
            if (k + AHEAD < NS) reg[k % AHEAD] = value_at(k + AHEAD);
            if (k < FIRST) {
#pragma unroll
                for (int i = 4 * k; i < 16; i += 4 * FIRST)
                    l += (x[i] + x[i + 1]) + (x[i + 2] + x[i + 3]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        hide(tn, kn);
        __builtin_amdgcn_s_setprio(0);
    };
    // a V that is not finite reaches the rows that see its token
    auto spread_bad = [&](int t) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const uint64_t bad = Bad[t & 3][g];
            if (bad != 0) {
                const int seen = min(max(limit - kTokens * t, 0), kTokens);
                const uint64_t visible = seen == 64 ? ~0ull : (1ull << seen) - 1;
                if (bad & visible) {
#pragma unroll
                    for (int b = g * (NB / NG); b < (g + 1) * (NB / NG); ++b)
#pragma unroll
                        for (int v = 0; v < 16; ++v) o[b][v] = __builtin_nanf("");
                }
            }
        }
    };

    if (begin < stop) {
        load_params(begin);
        load_words(begin);
        const float wave_size = max_of<16>(max_xor16((float)q.size));
        if (lane == 0) Sizes[w] = (int)wave_size;
        put_params(begin);
        load_params(begin + 1);
        __syncthreads();
        // one unit of K for the workgroup's rows (the first tile's groups are there)
        int size = Sizes[0];
#pragma unroll
        for (int k = 1; k < kManyWaves; ++k) size = max(size, Sizes[k]);
        const int exponent = __builtin_amdgcn_readfirstlane(key_unit(a.scale_log2, size));
        factor = positive_factor(a.scale_log2, q.exponent, exponent);
        unit = power_of_two(exponent);
        if (w == 0) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                Ksc[begin & 3][g][lane] *= unit;
                Kmn[begin & 3][g][lane] *= unit;
            }
        }
        put_words(begin, 0);
        put_params(begin + 1);
        load_words(begin + 1);
        load_params(begin + 2);
        __syncthreads();
        // the first block's scores
#pragma unroll
        for (int g = 0; g < NG; ++g) part[g] = zero16();
#pragma unroll
        for (int k = 0; k < NS; ++k)
            part[k / (NS / NG)] = mfma32x32x16f16(key_at(begin, 0, k), q.q[k], part[k / (NS / NG)]);
        val = mfma32x32x2(low_at(begin, 0), q.sum, zero16());
#pragma unroll
        for (int i = 0; i < 4 * NG; ++i) {
            const f32x4 sc = scale_at(begin, 0, i % NG, i / NG);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                val[4 * (i / NG) + r] =
                    fmaf(part[i % NG][4 * (i / NG) + r], sc[r], val[4 * (i / NG) + r]);
        }
        hide(begin, 0);
        int vb = 0;
        for (int t = begin; t < stop; ++t) {
            const int next = vb == 2 ? 0 : vb + 1;
            const bool works = wave_end > kTokens * t;
            if (works) step(t, 0, vb, t, 1);
            // tile t + 1 comes in: K over tile t - 1, which all waves are done
            // with, V in a third buffer, as tile t - 1's may still be read
            put_words(t + 1, next);
            put_params(t + 2);
            load_words(t + 2);
            load_params(t + 3);
            __syncthreads();
            if (works) {
                step(t, 1, vb, t + 1, 0);
                spread_bad(t);
            }
            vb = next;
        }
    }

    const bool valid = i < mask.rows;
    uint32_t which = 0;   // rows of the wave that are computed anew (lanes l and l + 32 agree)
    if (begin < stop && FarCount > 0) {
        bool far = false;
        for (int k = 0; k < FarCount; ++k) far |= limit > Far[k][0] && limit <= Far[k][1];
        which = (uint32_t)__ballot(in && valid && far);
        __syncthreads();   // Ks is free
    }

    l = sum_xor32(l);
    const bool stays = in && (which >> (c & 16) & 0xffffu) == 0;
    if (stays && a.splits > 1) {
        const size_t slot = ((size_t)bh * a.splits + split) * rows + r;
        float *to = a.part + slot * D;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f32x4 x;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    x[k] = valid ? ldexpf(o[b][4 * u + k], E - 15 - kLift) : 0.f;
                *reinterpret_cast<f32x4 *>(to + 32 * b + 8 * u + 4 * h) = x;
            }
        if (h == 0) {
            a.stat[2 * slot] = valid ? m : -INFINITY;
            a.stat[2 * slot + 1] = valid ? ldexpf(l, -kLift) : 0.f;
        }
    } else if (stays) {
        if (!valid) l = 0.f;
        const float inv = 1.f / l;   // (2^(E - 15) of it may be below f32's normal numbers)
        uint16_t *to = a.O + at * D;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint16_t x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    x[k] = to_bf16(l == 0.f ? 0.f : ldexpf(o[b][4 * u + k] * inv, E - 15));
                *reinterpret_cast<u32x2 *>(to + 32 * b + 8 * u + 4 * h) =
                    u32x2{x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16};
            }
        if (h == 0) a.LSE[at] = l != l ? l : row_lse(m, ldexpf(l, -kLift));
    }
    if (which != 0) far_rows<D>(which, w, lane, &Ks[0][0]);
}

template <int D>
hipError_t many(const Kv4Attn &p, const Kv4Plan &plan, const void *Q,
                const Kv4Cache<const uint32_t> &c, void *O, float *LSE, char *ws, hipStream_t s) {
    const int tiles = (int)((kv4_rows(p) + kRows - 1) / kRows);
    const ManyArgs a = {static_cast<const uint16_t *>(Q), c.k, c.v, c.kp, c.vp,
                        static_cast<uint16_t *>(O), LSE, (float *)(ws + plan.part),
                        (float *)(ws + plan.stat), p.key_len, p.q_len, p.H, p.G, p.Lq, p.L,
                        kv4_padded(p.L), p.causal, p.scale * kLog2e, plan.splits, tiles};
    kv4_many<D><<<(unsigned)((int64_t)p.B * p.H * plan.splits * tiles), 64 * kManyWaves, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_many(const Kv4Attn &p, const Kv4Plan &plan, const void *Q,
                           const Kv4Cache<const uint32_t> &c, void *O, float *LSE, void *ws,
                           hipStream_t s) {
    char *w = static_cast<char *>(ws);
    return p.d == 32 ? many<32>(p, plan, Q, c, O, LSE, w, s)
         : p.d == 64 ? many<64>(p, plan, Q, c, O, LSE, w, s)
                     : many<128>(p, plan, Q, c, O, LSE, w, s);
}

}  // namespace mg
