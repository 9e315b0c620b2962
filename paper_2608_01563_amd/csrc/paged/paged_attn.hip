// paged_attn.hip -- attention of a few query rows over a paged cache.
//
// A workgroup takes one cache head, 16 to 128 of the rows that share it and one unit:
// a stretch of a sequence's tokens (or of the pages that a row's list names).  Its
// four waves, or the two or one of them that have the same up to 32 rows, take blocks
// of 32 tokens (f32, d = 128: 16) in turn, each with its own online softmax, and join
// through LDS; units of one sequence join in paged_join.
//
// No operand passes through LDS.  A score tile is S^T = K Q^T: lane (c, g) = (l %
// 16, l / 16) holds 16-byte pieces 4 s + g of token c's K row and of row c's Q row,
// whatever channels these are, since a contraction's order is free.  S^T leaves
// lane (c, g) with tokens 4 g .. 4 g + 3 of row c, which is the operand of the
// second product O^T = V^T P^T if V's tokens come in that order: the lane reads
// D/16 channels of the rows 4 g + t, 16 lanes a whole row, and pairs of them are
// put together by one byte permutation a word (bf16).
//
// Pages are found through a table whose next 64 entries a wave keeps in a
// register.  Tiles of 16 tokens are read through buffer descriptors that end where
// the sequence does: behind it zeros come back, and nothing is read.
//
// bf16 probabilities enter as two bf16 parts each, which the matrix units have room
// for.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 16;
constexpr int kOnce = 2;   // cache policy: non-temporal
constexpr uint32_t kShort = 24;   // blocks of a unit
constexpr int kFar = 1 << 30;   // a token that no row sees

// Where lengths decide, every sequence is cut into units of `chunk` blocks at most, at
// least one unit each and all of a sequence alike (so that none is left with a few
// blocks).  Of 8 cache heads, bf16, d = 128, in us, by the workgroups that the lengths are
// cut into:
//
//                                                    384   512   768  1536
//   8 sequences of 16,384 to 65,536 tokens, 1 row    219   180   179   190
//   32 of 1,024 to 4,096, 1 row                             63    60    63
//   4 of 32,768, 1 row                               101    86    87    92
//   8 of 1,000 to 4,001, 28 rows                      31    27    35    35
//
// So: one round, two workgroups a compute unit or (of 16 rows) three, if units of
// some length, at most a third longer than would do without remainders, make no more
// of them and fill them to 13 in 16, or if they are short; `share` units, several
// rounds, otherwise.
__device__ __forceinline__ uint32_t parts_of(uint32_t blocks, uint32_t chunk) {
    return max((blocks + chunk - 1) / chunk, 1u);
}
struct Cut {
    int least, share, round, round_most;   // as PagedPlan's chunk, share, round, round_most

    __device__ __forceinline__ uint32_t within(uint32_t chunk) const {
        return min(max(chunk, (uint32_t)least), 1u << 13);
    }
    __device__ __forceinline__ uint32_t once(uint32_t total) const {
        return within((total + round - 1) / round);
    }
    __device__ __forceinline__ uint32_t rounds(uint32_t total) const {
        return once(total) <= kShort ? once(total) : within((total + share - 1) / share);
    }
};

// What scores stand for: 2^(factor s) with factor = |scale| log2 e, as two numbers (of a
// negative scale, Q's signs are turned).  Weights go by s less the row's largest, which
// is exact where they matter: a product with the factor less a rounded maximum is off by
// half a step of that maximum, which from 2^31 on is more than an exponent holds.
struct Scale {
    float factor, rest;
    float lowest;   // times rest it is finite

    // 2^(factor d), d <= 0 (-inf: 0; NaN stays).  f32: what the factor's rounding leaves
    // counts too, 4e-7 at d = -20.
    template <bool EXACT>
    __device__ __forceinline__ float weight(float d) const {
        if constexpr (EXACT) return exp2_fast(fmaf(d, factor, fmaxf(d, lowest) * rest));
        return exp2_fast(d * factor);
    }
    // (sums of a part without a score above -inf are 0, or NaN where a score is)
    template <bool EXACT>
    __device__ __forceinline__ float of_part(float its_top, float top) const {
        return its_top == -INFINITY ? 1.f : weight<EXACT>(its_top - top);
    }
    // log sum exp of a row with largest score m and sum l of weights: as row_lse, with the
    // part of factor m that its f32 value leaves
    __device__ __forceinline__ float lse(float m, float l) const {
        if (l != l) return l;
        if (!(l > 0.f)) return -INFINITY;
        const float top = m * factor;
        if (!(fabsf(top) < INFINITY)) return top;
        const float e = (float)__builtin_amdgcn_frexp_expf(l);
        const float n = top + e, a = n - top;
        const float low = (top - (n - a)) + (e - a) + (fmaf(m, factor, -top) + m * rest);
        return fmaf(n, kLn2, fmaf(n, kLn2Low, (__builtin_amdgcn_logf(
                                                   __builtin_amdgcn_frexp_mantf(l)) + low) * kLn2));
    }
};

struct AttnArgs {
    const void *Q, *Kp, *Vp;
    void *O;
    float *LSE, *part;
    float2 *stat;
    int2 *info;   // nullptr: every sequence (sparse: row) is one unit, nothing to join
    const int32_t *table, *index, *key_len, *q_len;
    int B, H, G, Lq, P, N, shift, causal, keep;
    Scale scale;
    uint32_t turn;   // Q's sign bits where the scale is negative
    const int32_t *unit_of;   // many sequences: each unit's
    int splits, chunk, groups;
    Cut cut;
};

// One unit: blocks [first, first + count) of sequence b (sparse: of row i's list);
// its sequence has `splits` units, the first of them number `base`.
struct Unit {
    int b, i, first, count, splits, base, split;
};

// Which sequence unit u belongs to; at most 64 M sequences, M a lane.
template <int M>
__device__ __forceinline__ Unit unit_by_length(const AttnArgs &a, const Cut &cut, int u, int lane) {
    uint32_t n[M], mine = 0;
#pragma unroll
    for (int e = 0; e < M; ++e) {
        const int b = M * lane + e;
        n[e] = b < a.B ? (uint32_t)(key_limit(a.key_len, b, a.P << a.shift) + 31) / 32 : 0u;
        mine += n[e];
    }
    const uint32_t total = wave_sum(mine), once = cut.once(total);
    uint32_t chunk = 0;
    for (int round = cut.round; round <= cut.round_most && a.B <= round; round += cut.round / 2) {
        const uint32_t least = cut.within((total + round - 1) / round);
        for (uint32_t turn = 0; chunk == 0 && turn < 6; ++turn) {
            const uint32_t longer = cut.within(least + least * turn / 16);
            if (once > kShort && (uint64_t)16 * total < (uint64_t)13 * round * longer) break;
            // (a quotient that rounds to one more or less changes the cut, not its sense)
            const float inverse = __builtin_amdgcn_rcpf((float)longer);
            uint32_t parts = 0;
#pragma unroll
            for (int e = 0; e < M; ++e)
                if (M * lane + e < a.B) parts += max((uint32_t)ceilf((float)n[e] * inverse), 1u);
            if (wave_sum(parts) <= (uint32_t)round) chunk = longer;
        }
        if (chunk != 0 || cut.round < 2) break;
    }
    if (chunk == 0) chunk = cut.rounds(total);
    uint32_t parts[M], sum = 0;
#pragma unroll
    for (int e = 0; e < M; ++e) {
        parts[e] = M * lane + e < a.B ? parts_of(n[e], chunk) : 0u;
        sum += parts[e];
    }
    const uint32_t end = wave_scan(sum);
    const uint64_t past = __ballot(end > (uint32_t)u);
    if (past == 0) return {-1, 0, 0, 0, 0, 0, 0};
    const int l = __builtin_ctzll(past);
    int base = __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(sum, l);
#pragma unroll
    for (int e = 0; e < M; ++e) {
        const int splits = __builtin_amdgcn_readlane(parts[e], l);
        if (e == M - 1 || base + splits > u) {
            const int count = (__builtin_amdgcn_readlane(n[e], l) + splits - 1) / splits;
            return {M * l + e, 0, (u - base) * count, count, splits, base, u - base};
        }
        base += splits;
    }
    return {-1, 0, 0, 0, 0, 0, 0};
}

// More than kPagedScanned sequences: a workgroup writes for every sequence its first unit and
// how many it has, and for every unit its sequence (-1 behind the last).  It takes 5 us;
// with it and with lengths that every unit scans, of up to 1,000 tokens and 2 cache heads:
// 1,024 sequences 127 and 141 us, 500 73 and 79; of 8 heads, 100: 59 and 57.
constexpr int kCutThreads = 1024;
__global__ __launch_bounds__(kCutThreads)
void paged_cut(const int32_t *key_len, int B, int capacity, int units, Cut cut, int2 *info,
               int32_t *unit_of) {
    __shared__ uint32_t sums[2][kCutThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const auto blocks_of = [&](int b) {
        return b < B ? (uint32_t)(key_limit(key_len, b, capacity) + 31) / 32 : 0u;
    };
    const auto all_of = [&](uint32_t v, uint32_t *to) {   // of the waves' sums, those before
        if (lane == 63) to[w] = v;
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (int k = 0; k < kCutThreads / 64; ++k) {
            before += k < w ? to[k] : 0u;
            all += to[k];
        }
        return make_uint2(before, all);
    };
    uint32_t total = 0;
    for (int b = tid; b < B; b += kCutThreads) total += blocks_of(b);
    total = all_of(wave_scan(total), sums[0]).y;
    const uint32_t chunk = cut.rounds(total);
    uint32_t carry = 0;
    for (int b0 = 0, turn = 1; b0 < B; b0 += kCutThreads, ++turn) {
        const int b = b0 + tid;
        const uint32_t parts = b < B ? parts_of(blocks_of(b), chunk) : 0u, end = wave_scan(parts);
        const uint2 others = all_of(end, sums[turn & 1]);
        const int base = carry + others.x + end - parts;
        if (b < B) {
            info[b] = make_int2(base, parts);
            for (int k = 0; k < (int)parts && base + k < units; ++k) unit_of[base + k] = b;
        }
        carry += others.y;
    }
    for (int u = carry + tid; u < units; u += kCutThreads) unit_of[u] = -1;
}

template <typename T, int D>
struct Shape {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kTiles = !kHalf && D == 128 ? 1 : 2;   // of 16 tokens a block
    static constexpr int kTok = 16 * kTiles;
    static constexpr int kPieces = kRowBytes / 64;   // 16-byte pieces of K a lane
    static constexpr int kN = D / 16;                // channels of V a lane
    static constexpr int kWords = kRowBytes / 64;    // 4-byte words of them
    // channel j (of kN) of the m-th lane that shares a V row
    static __device__ __forceinline__ constexpr int channel(int m, int j) {
        if (!kHalf && D == 128) return 64 * (j / 4) + 4 * m + j % 4;
        return kN * m + j;
    }
};

// A block's K pieces and V words.
template <typename T, int D, int CACHE>
struct Block {
    using S = Shape<T, D>;
    u32x4 k[S::kTiles][S::kPieces];
    uint32_t v[S::kTiles][4][S::kWords];

    __device__ __forceinline__ void load_k(int t, __amdgpu_buffer_rsrc_t r, int at) {
#pragma unroll
        for (int s = 0; s < S::kPieces; ++s)
            k[t][s] = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + 64 * s, 0, CACHE));
    }
    __device__ __forceinline__ void load_v(int t, __amdgpu_buffer_rsrc_t r, int at) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int o = at + x * S::kRowBytes;
            if constexpr (S::kWords >= 4) {
#pragma unroll
                for (int q = 0; q < S::kWords / 4; ++q) {
                    const u32x4 y = __builtin_bit_cast(
                        u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o + 256 * q, 0, CACHE));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[t][x][4 * q + e] = y[e];
                }
            } else if constexpr (S::kWords == 2) {
                const u32x2 y =
                    __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, o, 0, CACHE));
                v[t][x][0] = y[0], v[t][x][1] = y[1];
            } else {
                v[t][x][0] = __builtin_amdgcn_raw_buffer_load_b32(r, o, 0, CACHE);
            }
        }
    }
};

// A block's probabilities as the second product's operand: f32, or two bf16 parts.
// The first part is the next bf16 number below p, so that the second is above 0 where
// p is and an infinite V stays what it is; it leaves less than 2^-7 of p, of which the
// second is within 2^-8.
template <typename T, int D>
struct Operand {
    f32x4 p[Shape<T, D>::kTiles];

    __device__ __forceinline__ void set(const f32x4 (&x)[Shape<T, D>::kTiles]) {
#pragma unroll
        for (int t = 0; t < Shape<T, D>::kTiles; ++t) p[t] = x[t];
    }
};
template <int D>
struct Operand<uint16_t, D> {
    bf16x8 hi, lo;

    __device__ __forceinline__ void set(const f32x4 (&p)[2]) {
        u32x4 high;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            uint32_t u[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float x = p[(e + k) / 4][(e + k) % 4];
                u[k] = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u);
                lo[e + k] = (__bf16)(x - __uint_as_float(u[k] & 0xffff0000u));
            }
            high[e / 2] = __builtin_amdgcn_perm(u[1], u[0], 0x07060302);
        }
        hi = __builtin_bit_cast(bf16x8, high);
    }
};

template <typename T, int D, bool SPARSE, int RT, int TW, int CACHE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 8)))
void paged_attn(AttnArgs a) {
    using S = Shape<T, D>;
    constexpr int NT = S::kTiles, N = S::kN, RB = S::kRowBytes;
    constexpr int LD = D + 4, WV = kWaves / TW, WR = kRows * RT;   // waves, rows a stream
    __shared__ __attribute__((aligned(16))) float Os[kWaves][WR][LD];
    __shared__ float Ms[kWaves][WR], Ls[kWaves][WR];
    __shared__ bool Odd[kWaves];

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = blockIdx.x % a.groups, rest = blockIdx.x / a.groups;
    const int h = rest % a.H, u = rest / a.H;
    Unit un;
    if (a.splits > 0) {
        const int at = u / a.splits;
        un.split = u - at * a.splits;
        un.b = SPARSE ? at / a.Lq : at;
        un.i = SPARSE ? at - un.b * a.Lq : 0;
        un.base = at * a.splits;
        un.splits = a.splits;
        un.count = a.chunk;
        un.first = un.split * a.chunk;
    } else if (a.unit_of != nullptr) {
        un = {__builtin_amdgcn_readfirstlane(a.unit_of[u]), 0, 0, 0, 0, 0, 0};
        if (un.b < 0) return;
        const int2 its = a.info[un.b];
        un.base = its.x;
        un.splits = its.y;
        un.split = u - its.x;
    } else {
        un = a.B <= 64 ? unit_by_length<1>(a, a.cut, u, lane) : unit_by_length<4>(a, a.cut, u, lane);
        if (un.b < 0) return;
    }
    const PagedMask mask =
        paged_mask(a.key_len, a.q_len, un.b, a.P << a.shift, a.Lq, a.causal);
    if (a.splits > 0 && !SPARSE)   // units behind the sequence's end are none
        un.splits = max(1, min(a.splits, ((mask.n + 31) / 32 + a.chunk - 1) / a.chunk));
    if (!SPARSE && a.unit_of != nullptr) {
        un.count = ((mask.n + 31) / 32 + un.splits - 1) / un.splits;
        un.first = un.split * un.count;
    }
    if (!SPARSE && a.unit_of == nullptr && a.info != nullptr && h == 0 && group == 0 &&
        un.split == 0 && tid == 0)
        a.info[un.b] = make_int2(un.base, un.splits);
    if (un.split >= un.splits) return;

    // the lane's rows, one a tile, and what the wave's rows see
    const int rows = SPARSE ? a.G : a.G * a.Lq;
    const int row0 = WR * (group * TW + w % TW);
    int row_i[RT], limit[RT];
    size_t row_at[RT];   // of [B][Hq][Lq]
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + kRows * r + c, rows - 1);
        row_i[r] = SPARSE ? un.i : row / a.G;
        const int head = SPARSE ? row : row - row_i[r] * a.G;
        row_at[r] = ((size_t)(un.b * a.H + h) * a.G + head) * a.Lq + row_i[r];
        limit[r] = row0 + kRows * r + c < rows ? mask.limit(row_i[r]) : 0;
    }
    const int first_i = SPARSE ? un.i : row0 / a.G;
    const int last_i = SPARSE ? un.i : min((min(rows, row0 + WR) - 1) / a.G, mask.rows - 1);
    const bool some = row0 < rows && first_i < mask.rows;
    const int all = some ? mask.limit(first_i) : 0;   // below: every row sees the token
    const int end = some ? mask.limit(last_i) : 0;

    // the pages: entries pb .. pb + 63 of the table (sparse: of the row's list)
    const int32_t *table = a.table + (size_t)un.b * a.P;
    int pb = (32 * un.first) >> a.shift;
    int stop = min(((SPARSE ? a.keep << a.shift : end) + S::kTok - 1) / S::kTok,
                   (un.first + un.count) * (32 / S::kTok));
    const auto entry = [&](int p) { return table[min(p, a.P - 1)]; };
    int ids, ids_next = 0, place = 0;
    if constexpr (SPARSE) {
        const int32_t *list = a.index + (((size_t)un.b * a.H + h) * a.Lq + un.i) * a.keep;
        const int k = pb + lane;
        place = k < a.keep ? list[k] : -1;
        const int before = k > 0 && k <= a.keep ? list[k - 1] : -1;
        const bool good = place > before && place >= 0 && place < a.P;
        ids = good ? table[place] : -1;
        const uint64_t any = __ballot(good);   // nothing is listed behind the last
        const int listed = any == 0 ? 0 : 64 - __builtin_clzll(any);
        stop = min(stop, (((pb + listed) << a.shift) + S::kTok - 1) / S::kTok);
    } else {
        ids = entry(pb + lane);
        ids_next = entry(pb + 64 + lane);
    }

    // where a tile of 16 tokens lies, and its first token (kFar: it is not seen)
    const char *kp = static_cast<const char *>(a.Kp), *vp = static_cast<const char *>(a.Vp);
    const size_t head_bytes = (size_t)RB << a.shift;
    struct Place {
        size_t at;
        int token, bytes;
    };
    const auto place_of = [&](int block, int t) {
        const int v = S::kTok * block + 16 * t, rel = (v >> a.shift) - pb;
        const int row = v & ((1 << a.shift) - 1);
        int id = __builtin_amdgcn_readlane(ids, rel), token = v;
        if constexpr (SPARSE) token = (__builtin_amdgcn_readlane(place, rel) << a.shift) + row;
        if ((uint32_t)id >= (uint32_t)a.N) id = 0, token = kFar;
        const int left = min(max(end - token, 0), 16);
        return Place{((size_t)id * a.H + h) * head_bytes + (size_t)row * RB, token, left * RB};
    };

    Block<T, D, CACHE> x;
    Place now[NT], next[NT];
    const int k_at = c * RB + 16 * g, v_at = 4 * g * RB + (RB / 16 > 16 ? 16 : RB / 16) * c;
    int block = un.first * (32 / S::kTok) + w / TW;
    const bool any = block < stop;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        now[t] = any ? place_of(block, t) : Place{0, kFar, 0};
        x.load_k(t, buffer_rsrc(kp + now[t].at, now[t].bytes), k_at);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) x.load_v(t, buffer_rsrc(vp + now[t].at, now[t].bytes), v_at);

    // (rows that see nothing, whatever they hold, are taken as zeros)
    u32x4 q[RT][S::kPieces];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int s = 0; s < S::kPieces; ++s)
            q[r][s] = limit[r] > 0 ? *reinterpret_cast<const u32x4 *>(
                                         static_cast<const char *>(a.Q) + row_at[r] * RB + 64 * s +
                                         16 * g) ^ a.turn
                                   : u32x4{0, 0, 0, 0};

    float m[RT], l[RT];
    f32x4 o[RT][N];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) o[r][j] = zero4();
    }

    bool left_out = false;   // V of tokens that not all rows see
    while (block < stop) {
        f32x4 s[RT][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                // (two sums for f32, whose roundings are what a score is off by)
                f32x4 sum[2] = {zero4(), zero4()};
#pragma unroll
                for (int y = 0; y < S::kPieces; ++y) {
                    if constexpr (S::kHalf) {
                        sum[0] = mfma16x16x32bf16(__builtin_bit_cast(bf16x8, x.k[t][y]),
                                                  __builtin_bit_cast(bf16x8, q[r][y]), sum[0]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            sum[e % 2] = mfma16x16x4(__uint_as_float(x.k[t][y][e]),
                                                     __uint_as_float(q[r][y][e]), sum[e % 2]);
                    }
                }
                s[r][t] = S::kHalf ? sum[0] : sum[0] + sum[1];
            }
        // the next block's K comes while this one's scores are worked on (behind
        // the last block: descriptors of no bytes)
        const int following = block + WV;
        if (!SPARSE && ((S::kTok * following) >> a.shift) - pb >= 64) {
            pb += 64;
            ids = ids_next;
            ids_next = entry(pb + 64 + lane);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            next[t] = following < stop ? place_of(following, t) : Place{0, kFar, 0};
            x.load_k(t, buffer_rsrc(kp + next[t].at, next[t].bytes), k_at);
        }

        bool partly = false, diagonal = false;   // tokens that not all, that some rows see
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            partly |= now[t].token + 16 > all;
            diagonal |= end > all && now[t].token + 16 > all && now[t].token < end;
        }
        Operand<T, D> operand[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const f32x4 x = s[r][t];
                if (partly) {
                    const int left = limit[r] - now[t].token - 4 * g;
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, e < left ? x[e] : -INFINITY);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, x[e]);
                }
            }
            top = fmaxf(m[r], max_over_groups(top));
            if (__any(top > m[r])) {
                const float alpha =
                    m[r] == -INFINITY ? 0.f : a.scale.template weight<!S::kHalf>(m[r] - top);
                l[r] *= alpha;
#pragma unroll
                for (int j = 0; j < N; ++j) o[r][j] *= alpha;
                m[r] = top;
            }
            const float from = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[r][t][e] = a.scale.template weight<!S::kHalf>(s[r][t][e] - from);
                if (partly) {
                    const int left = limit[r] - now[t].token - 4 * g;
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r][t][e] = e < left ? s[r][t][e] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) l[r] += s[r][t][e];
            }
            operand[r].set(s[r]);
        }

        // channel block j of V^T, from words that `word` gives: an operand (bf16), or
        // the values of tokens 4 g + y of tile t (f32)
        const auto channels = [&](auto word, int j) {
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = __builtin_amdgcn_perm(word(e / 2, 2 * (e % 2) + 1, j / 2),
                                             word(e / 2, 2 * (e % 2), j / 2),
                                             j % 2 ? 0x07060302 : 0x05040100);
            return __builtin_bit_cast(bf16x8, v);
        };
        const auto value = [&](int t, int y, int word) { return x.v[t][y][word]; };
        if (!SPARSE && diagonal) {
            // V that is infinite or NaN and that not all rows see would reach the others as
            // 0 times it: it is left out here and added to the rows that see it in the end
            const auto odd = [](uint32_t v) { return (v & 0x7f800000u) == 0x7f800000u; };
            bool mine = false;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int word = 0; word < S::kWords; ++word) {
                        uint32_t &v = x.v[t][y][word];
                        const bool unseen = now[t].token + 4 * g + y >= all;
                        const bool high = unseen && odd(v);
                        const bool low = unseen && S::kHalf && odd(v << 16);
                        mine |= high || low;
                        v = high ? S::kHalf ? v & 0xffffu : 0u : v;
                        v = low ? v & 0xffff0000u : v;
                    }
            left_out |= __any(mine);
        }
        // O^T += V^T P^T
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (S::kHalf) {
                const bf16x8 v = channels(value, j);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    o[r][j] = mfma16x16x32bf16(v, operand[r].hi, o[r][j]);
                    o[r][j] = mfma16x16x32bf16(v, operand[r].lo, o[r][j]);
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            o[r][j] = mfma16x16x4(__uint_as_float(value(t, y, j)),
                                                  operand[r].p[t][y], o[r][j]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            x.load_v(t, buffer_rsrc(vp + next[t].at, next[t].bytes), v_at);
            now[t] = next[t];
        }
        block = following;
    }

    // the waves' shares through LDS
    if (lane == 0) Odd[w] = left_out;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        l[r] = sum_over_groups(l[r]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < N; ++j)
                Os[w][kRows * r + c][S::channel(4 * g + e, j)] = o[r][j][e];
        if (g == 0) {
            Ms[w][kRows * r + c] = m[r];
            Ls[w][kRows * r + c] = l[r];
        }
    }
    __syncthreads();

    const int d0 = N * (tid & 15);
    for (int at = tid >> 4; at < WR * TW; at += kThreads / 16) {
        const int part = at / WR, row = at % WR, rr = WR * TW * group + at;
        if (rr >= rows) return;
        float top = -INFINITY;
#pragma unroll
        for (int k = part; k < kWaves; k += TW) top = fmaxf(top, Ms[k][row]);
        float sum = 0.f, y[N];
#pragma unroll
        for (int k = 0; k < N; ++k) y[k] = 0.f;
#pragma unroll
        for (int k = part; k < kWaves; k += TW) {
            const float f = a.scale.template of_part<!S::kHalf>(Ms[k][row], top);
            sum = fmaf(f, Ls[k][row], sum);
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = fmaf(f, Os[k][row][d0 + e], y[e]);
        }
        const int ri = SPARSE ? un.i : rr / a.G, rh = SPARSE ? rr : rr - ri * a.G;
        const size_t to = ((size_t)(un.b * a.H + h) * a.G + rh) * a.Lq + ri;
        const bool live = ri < mask.rows;
        bool odd = false;
#pragma unroll
        for (int k = 0; k < WV; ++k) odd |= Odd[part + TW * k];
        if (!SPARSE && odd) {
            const int from = max(mask.limit(WR * (group * TW + part) / a.G), 32 * un.first);
            for (int j = from; j < min(mask.limit(ri), 32 * (un.first + un.count)); ++j) {
                const int id = table[j >> a.shift];
                if ((uint32_t)id >= (uint32_t)a.N) continue;
                const T *v = reinterpret_cast<const T *>(
                    vp + ((size_t)id * a.H + h) * head_bytes +
                    (size_t)(j & ((1 << a.shift) - 1)) * RB) + d0;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    float x;
                    if constexpr (S::kHalf) x = bf16_to_f32(v[e]);
                    else x = v[e];
                    if (!(fabsf(x) < INFINITY)) y[e] += x;
                }
            }
        }
        if (un.splits > 1) {
            const size_t slot = ((size_t)u * a.H + h) * rows + rr;
            float *p = a.part + slot * D + d0;
#pragma unroll
            for (int e = 0; e < N; ++e) p[e] = live ? y[e] : 0.f;
            if (d0 == 0) a.stat[slot] = live ? make_float2(top, sum) : make_float2(-INFINITY, 0.f);
            continue;
        }
        if (!live) sum = 0.f;
        const float inv = 1.f / sum;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = sum == 0.f ? 0.f : y[e] * inv;
        T *out = static_cast<T *>(a.O) + to * D + d0;
        if constexpr (N >= 4) {
            store_row(out, y);
        } else if constexpr (S::kHalf) {
            *reinterpret_cast<uint32_t *>(out) = to_bf16(y[0]) | (uint32_t)to_bf16(y[1]) << 16;
        } else {
            *reinterpret_cast<f32x2 *>(out) = f32x2{y[0], y[1]};
        }
        if (d0 == 0) a.LSE[to] = a.scale.lse(top, sum);
    }
}

// ------------------------------------------------------------------- joining --
struct JoinArgs {
    void *O;
    float *LSE;
    const float *part;
    const float2 *stat;
    const int2 *info;   // nullptr: every sequence (row) has `splits` units
    int H, G, Lq, rows, splits, total;
    Scale scale;
};

// WAVES waves join a row.  Lanes in teams of D / 4, four channels each, take the
// units in turn; the maximum comes first, a unit a lane.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(kThreads)
void paged_join(JoinArgs a) {
    constexpr int TEAMS = 256 / D;
    __shared__ float tops[kWaves];
    __shared__ __attribute__((aligned(16))) float Ys[kWaves][D];
    __shared__ float Sums[kWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int wave = WAVES == 1 ? 0 : w;
    const int id = WAVES == 1 ? blockIdx.x * kWaves + w : blockIdx.x;
    if (id >= a.total) return;   // (a whole workgroup where several waves join a row)
    const int r = id % a.rows, rest = id / a.rows;
    const int h = rest % a.H, seq = rest / a.H;   // sequence, or sparse its row
    const int2 in = a.info ? a.info[seq] : make_int2(seq * a.splits, a.splits);
    if (in.y <= 1) return;
    const auto slot = [&](int k) { return ((size_t)(in.x + k) * a.H + h) * a.rows + r; };

    // four units at a time, so that their reads are on the way together (the first ones
    // beside the maxima's; past the end the last unit again, unused)
    const int team = lane / (D / 4), d0 = 4 * (lane % (D / 4));
    constexpr int STEP = TEAMS * WAVES;
    f32x4 y[4];
    float2 st[4];
    const auto read = [&](int k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const size_t at = slot(min(k + e * STEP, in.y - 1));
            st[e] = a.stat[at];
            y[e] = *reinterpret_cast<const f32x4 *>(a.part + at * D + d0);
        }
    };
    const int k0 = wave * TEAMS + team;
    read(k0);
    float top = -INFINITY;
    for (int k = 64 * wave + lane; k < in.y; k += 64 * WAVES) top = fmaxf(top, a.stat[slot(k)].x);
    top = max_xor32(max_xor16(max_of<16>(top)));
    if constexpr (WAVES > 1) {
        if (lane == 0) tops[w] = top;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < WAVES; ++k) top = fmaxf(top, tops[k]);
    }
    f32x4 x = zero4();
    float sum = 0.f;
    for (int k = k0; k < in.y; k += 4 * STEP) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (k + e * STEP >= in.y) continue;
            const float f = a.scale.template of_part<sizeof(T) == 4>(st[e].x, top);
            sum = fmaf(f, st[e].y, sum);
            x += f * y[e];
        }
        if (k + 4 * STEP < in.y) read(k + 4 * STEP);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (TEAMS >= 2) x[e] = sum_xor32(x[e]);
        if (TEAMS >= 4) x[e] = sum_xor16(x[e]);
        if (TEAMS >= 8) x[e] += xor_lanes(x[e], 8);
    }
    if (TEAMS >= 2) sum = sum_xor32(sum);
    if (TEAMS >= 4) sum = sum_xor16(sum);
    if (TEAMS >= 8) sum += xor_lanes(sum, 8);
    if constexpr (WAVES > 1) {
        if (team == 0) *reinterpret_cast<f32x4 *>(&Ys[w][d0]) = x;
        if (lane == 0) Sums[w] = sum;
        __syncthreads();
        if (w != 0) return;
        x = zero4();
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            x += *reinterpret_cast<const f32x4 *>(&Ys[k][d0]);
            sum += Sums[k];
        }
    }
    // dense: rows r = i G + g of the sequence; sparse: head r of row seq % Lq
    const bool sparse = a.info == nullptr;
    const int b = sparse ? seq / a.Lq : seq;
    const int i = sparse ? seq - b * a.Lq : r / a.G, hd = sparse ? r : r - i * a.G;
    const size_t to = ((size_t)(b * a.H + h) * a.G + hd) * a.Lq + i;
    if (team == 0) {
        const float inv = 1.f / sum;
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = sum == 0.f ? 0.f : x[e] * inv;
        store_row(static_cast<T *>(a.O) + to * D + d0, y);
    }
    if (lane == 0) a.LSE[to] = a.scale.lse(top, sum);
}

Cut cut_of(const PagedPlan &plan) {
    return {plan.chunk, plan.share, plan.round, plan.round_most};
}

Scale scale_of(const PagedAttn &p) {
    const double whole = std::fabs(p.scale * 1.4426950408889634);
    const float factor = (float)whole, rest = (float)(whole - factor);
    return {factor, rest, rest == 0.f ? -FLT_MAX : -(float)std::min<double>(
                                                       FLT_MAX, 0x1p126 / std::fabs(rest))};
}

template <typename T, int D>
hipError_t attn(const PagedAttn &p, const PagedPlan &plan, const void *Q, const void *Kp,
                const void *Vp, void *O, float *LSE, char *ws, hipStream_t s) {
    const AttnArgs a = {Q, Kp, Vp, O, LSE, (float *)(ws + plan.part), (float2 *)(ws + plan.stat),
                        plan.most > 1 ? (int2 *)(ws + plan.info) : nullptr, p.table, p.index,
                        p.key_len, p.q_len, p.B, p.H, p.G, p.Lq, p.P, p.N, p.shift, p.causal,
                        p.keep, scale_of(p),
                        p.scale < 0.f ? p.half ? 0x80008000u : 0x80000000u : 0u,
                        plan.lengths ? (const int32_t *)(ws + plan.map) : nullptr, plan.splits,
                        plan.chunk, plan.groups, cut_of(plan)};
    const unsigned grid = (unsigned)((int64_t)plan.units * p.H * plan.groups);
    const auto run = [&](auto SPARSE, auto RT, auto TW, auto CACHE) {
        paged_attn<T, D, decltype(SPARSE)::value, decltype(RT)::value, decltype(TW)::value,
                   decltype(CACHE)::value><<<grid, kThreads, 0, s>>>(a);
        return hipGetLastError();
    };
    const auto rows = [&](auto SPARSE) {
        const std::integral_constant<int, 0> cached;
        const std::integral_constant<int, kOnce> once;
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        if (plan.rows == 16)
            return plan.once ? run(SPARSE, one, one, once) : run(SPARSE, one, one, cached);
        if (plan.rows == 32)
            return plan.once ? run(SPARSE, two, one, once) : run(SPARSE, two, one, cached);
        return plan.rows == 64 ? run(SPARSE, two, two, cached) : run(SPARSE, two, four, cached);
    };
    return p.index != nullptr ? rows(std::true_type()) : rows(std::false_type());
}

template <typename T, int D>
hipError_t join(const PagedAttn &p, const PagedPlan &plan, void *O, float *LSE, const char *ws,
                hipStream_t s) {
    const bool sparse = p.index != nullptr;
    const int rows = (int)paged_rows(p, sparse);
    const int64_t total = (int64_t)p.B * (sparse ? p.Lq : 1) * p.H * rows;
    const JoinArgs a = {O, LSE, (const float *)(ws + plan.part), (const float2 *)(ws + plan.stat),
                        sparse ? nullptr : (const int2 *)(ws + plan.info), p.H, p.G, p.Lq, rows,
                        plan.splits, (int)total, scale_of(p)};
    if (plan.join_waves == 1)
        paged_join<T, D, 1><<<(unsigned)((total + kWaves - 1) / kWaves), kThreads, 0, s>>>(a);
    else
        paged_join<T, D, kWaves><<<(unsigned)total, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_cut(const PagedAttn &p, const PagedPlan &plan, void *ws, hipStream_t s) {
    char *w = static_cast<char *>(ws);
    paged_cut<<<1, kCutThreads, 0, s>>>(p.key_len, p.B, p.P << p.shift, plan.units, cut_of(plan),
                                        (int2 *)(w + plan.info), (int32_t *)(w + plan.map));
    return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttn &p, const PagedPlan &plan, const void *Q,
                             const void *Kp, const void *Vp, void *O, float *LSE, void *ws,
                             hipStream_t s) {
    char *w = static_cast<char *>(ws);
    if (p.half)
        return p.d == 32 ? attn<uint16_t, 32>(p, plan, Q, Kp, Vp, O, LSE, w, s)
             : p.d == 64 ? attn<uint16_t, 64>(p, plan, Q, Kp, Vp, O, LSE, w, s)
                         : attn<uint16_t, 128>(p, plan, Q, Kp, Vp, O, LSE, w, s);
    return p.d == 32 ? attn<float, 32>(p, plan, Q, Kp, Vp, O, LSE, w, s)
         : p.d == 64 ? attn<float, 64>(p, plan, Q, Kp, Vp, O, LSE, w, s)
                     : attn<float, 128>(p, plan, Q, Kp, Vp, O, LSE, w, s);
}

hipError_t launch_paged_join(const PagedAttn &p, const PagedPlan &plan, void *O, float *LSE,
                             const void *ws, hipStream_t s) {
    const char *w = static_cast<const char *>(ws);
    if (p.half)
        return p.d == 32 ? join<uint16_t, 32>(p, plan, O, LSE, w, s)
             : p.d == 64 ? join<uint16_t, 64>(p, plan, O, LSE, w, s)
                         : join<uint16_t, 128>(p, plan, O, LSE, w, s);
    return p.d == 32 ? join<float, 32>(p, plan, O, LSE, w, s)
         : p.d == 64 ? join<float, 64>(p, plan, O, LSE, w, s)
                     : join<float, 128>(p, plan, O, LSE, w, s);
}

}  // namespace mg
