// kv4_rows.hip -- attention over the 4-bit cache: a workgroup takes 16 of the
// query rows that share a cache head and one chunk of the tokens; its four
// waves take 32-token blocks in turn, each with its own online softmax, and
// join through LDS; chunks join in kv4_join.
//
// A chunk is a fixed number of blocks whatever the sequence's length: chunks
// behind its end are gone at once and the dispatcher evens out sequences of
// different length; and where a wave's first block lies does not wait for the
// length, so words, groups, query row and length are all asked for together.
//
// The products and the online softmax: kv4_sweep.h.
//
// 16 rows are the least a matrix product takes, and enough: one pass over the
// cache is what a decode step costs.  64 heads of up to 32,768 tokens of 128
// channels, 4 rows each (189 MB): 48.7 us with the join, 3.9 TB/s where a large
// copy reaches 5.1.  Instruction issue bounds it (about 290 vector instructions a
// 32-token block, three quarters of a SIMD's time), which is why codes are
// multiplied as they are and scaled afterwards.  Words three blocks ahead instead
// of two: 53 us.  One equal stretch of all sequences' blocks for every workgroup
// instead of fixed chunks: 51 us, and 5 us more for short calls.
#include "cdiv.h"
#include "kv4_launch.h"
#include "kv4_sweep.h"

namespace mg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = kSweepRows;

struct RowsArgs {
    const void *Q;
    const uint32_t *kw, *vw, *kp, *vp;
    void *O;
    float *LSE, *part, *stat, *score;
    const int32_t *key_len, *q_len;
    int H, G, Lq, L, Lp, causal;
    float scale_log2;
    int splits, chunk, row_tiles;   // chunk: blocks
};

template <typename T, int D, int NP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(3, 8)))
void kv4_rows(RowsArgs a) {
    constexpr int NG = Kv4Dim<D>::kGroups, NB = Kv4Dim<D>::kBlocks;
    constexpr int LD = D + 4;
    __shared__ __attribute__((aligned(16))) float Os[kWaves][kRows][LD];
    __shared__ float Ms[kWaves][kRows], Ls[kWaves][kRows];
    __shared__ __attribute__((aligned(16))) BlockGroups<NG> Gs[kWaves][2];

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = blockIdx.x % a.row_tiles, share = blockIdx.x / a.row_tiles;
    const int bh = share / a.splits, split = share - bh * a.splits;
    const int b = bh / a.H;
    const int rows = a.G * a.Lq;
    const Kv4Mask mask = sequence_mask(a.key_len, a.q_len, b, a.L, a.Lq, a.causal);

    // blocks begin + w, + kWaves, ... are the wave's; its first one's words
    const size_t head = (size_t)bh * a.Lp;
    const uint32_t *kw = a.kw + head * (D / 8), *vw = a.vw + head / 8 * D;
    const uint32_t *kp = a.kp + head * NG, *vp = a.vp + head * NG;
    const int begin = split * a.chunk, mine = begin + w, last = a.Lp / 32 - 1;
    Kv4Keys<D> k0, k1;
    Kv4Values<D> v0, v1;
    Kv4GroupWords<NG> g0, g1;
    k0.load(kw, min(mine, last), c, g);
    v0.load(vw, min(mine, last), c, g);
    g0.load(kp, vp, min(mine, last), lane);

    const int r = kRows * tile + c;
    const bool in = r < rows;
    const RowAt at = row_at(in ? r : rows - 1, bh, a.G, a.Lq);
    Kv4Query<D, NP> q;
    // (rows behind the sequence's, whatever they hold, are taken as zeros)
    q.load(static_cast<const T *>(a.Q) + at.at * D, in && at.i < mask.rows, g,
           a.scale_log2 < 0.f);
    const auto factors = Kv4Sweep<D, NP>::factors(q, a.scale_log2, lane);

    // the tokens that the tile's last and its first row see
    if (32 * begin >= mask.n && begin > 0) return;   // kv4_join knows
    const int first_i = kRows * tile / a.G;
    const int last_i = min((min(rows, kRows * (tile + 1)) - 1) / a.G, mask.rows - 1);
    const int end = first_i < mask.rows ? max(mask.limit(last_i), 0) : 0;
    const int all = mask.limit(first_i);   // below: every row sees the token
    const int limit = mask.limit(at.i);
    const int stop = min((end + 31) / 32, begin + a.chunk);

    Kv4Sweep<D, NP> sweep;
    auto step = [&](int block, const Kv4Keys<D> &key, const Kv4Values<D> &val,
                    Kv4GroupWords<NG> &words, BlockGroups<NG> &groups) {
        sweep.step(block, q, factors, limit, all, mask.n, key, val, words, groups, lane,
                   [&](const f32x4(&s)[2]) {
            if (a.score == nullptr || !in) return;
            float *to = a.score + ((size_t)bh * rows + r) * a.Lp + 32 * block + 8 * g;
            *reinterpret_cast<f32x4 *>(to) = s[0] * factors.factor;
            *reinterpret_cast<f32x4 *>(to + 4) = s[1] * factors.factor;
        });
    };

    // the next block's words load while one is worked on (past the end the last
    // block again)
    for (int block = mine; block < stop; block += 2 * kWaves) {
        const int b1 = min(block + kWaves, stop - 1), b2 = min(block + 2 * kWaves, stop - 1);
        k1.load(kw, b1, c, g);
        v1.load(vw, b1, c, g);
        g1.load(kp, vp, b1, lane);
        step(block, k0, v0, g0, Gs[w][0]);
        if (block + kWaves >= stop) break;
        k0.load(kw, b2, c, g);
        v0.load(vw, b2, c, g);
        g0.load(kp, vp, b2, lane);
        step(block + kWaves, k1, v1, g1, Gs[w][1]);
    }

    // the waves' shares through LDS
    sweep.finish();
#pragma unroll
    for (int cb = 0; cb < NB; ++cb)
        *reinterpret_cast<f32x4 *>(&Os[w][c][16 * cb + 4 * g]) = sweep.o[cb];
    if (g == 0) {
        Ms[w][c] = sweep.m;
        Ls[w][c] = sweep.l;
    }
    __syncthreads();

    constexpr int N = D / 16;   // channels a thread writes
    const int row = tid >> 4, d0 = N * (tid & 15);
    const int rr = kRows * tile + row;
    if (rr >= rows) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = fmaxf(top, Ms[k][row]);
    float sum = 0.f, x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const float f = top == -INFINITY ? 1.f : exp2_fast(Ms[k][row] - top);
        sum = fmaf(f, Ls[k][row], sum);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(f, Os[k][row][d0 + i], x[i]);
    }
    const RowAt to = row_at(rr, bh, a.G, a.Lq);
    const bool valid = to.i < mask.rows;
    if (a.splits > 1) {
        const size_t slot = ((size_t)bh * a.splits + split) * rows + rr;
        float *p = a.part + slot * D + d0;
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = valid ? x[i] : 0.f;
        if (d0 == 0) {
            a.stat[2 * slot] = valid ? top : -INFINITY;
            a.stat[2 * slot + 1] = valid ? sum : 0.f;
        }
        return;
    }
    if (!valid) sum = 0.f;
    const float inv = 1.f / sum;
    T *out = static_cast<T *>(a.O) + to.at * D + d0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float y = sum == 0.f ? 0.f : x[i] * inv;
        if constexpr (sizeof(T) == 2) out[i] = to_bf16(y);
        else out[i] = y;
    }
    if (d0 == 0) a.LSE[to.at] = sum != sum ? sum : row_lse(top, sum);
}

// ------------------------------------------------------------------- joining --
struct JoinArgs {
    void *O;
    float *LSE, *weight;
    const float *part, *stat, *score;
    const int32_t *key_len, *q_len;
    int H, G, Lq, L, Lp, causal, splits, chunk, heads, out_groups;   // chunk: blocks, or 0
};
constexpr int kJoinKeys = 4 * kThreads;   // tokens of a weights workgroup

// A row's splits (at most 64), one a lane: maximum, sum, and the lane's factor.
// Splits whose chunk lies behind the sequence's n tokens wrote nothing.
struct Joined {
    float top, sum, factor;
};
__device__ __forceinline__ int written_splits(const JoinArgs &a, int n) {
    return a.chunk == 0 ? a.splits : max(1, min(a.splits, (n + 32 * a.chunk - 1) / (32 * a.chunk)));
}
__device__ __forceinline__ Joined join_stats(f32x2 stat, int count, int lane) {
    const float m = lane < count ? stat[0] : -INFINITY, l = lane < count ? stat[1] : 0.f;
    const float top = max_of_wave(m);
    // without a score above -inf the sums are 0, or NaN where a score is
    const float factor = top == -INFINITY ? 1.f : exp2_fast(m - top);
    return {top, sum_of_wave(factor * l), factor};
}
__device__ __forceinline__ f32x2 load_stat(const float *stat, size_t first, int stride, int splits,
                                           int lane) {
    return *reinterpret_cast<const f32x2 *>(stat +
                                            2 * (first + (size_t)min(lane, splits - 1) * stride));
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads)
void kv4_join(JoinArgs a) {
    const int rows = a.G * a.Lq;
    if ((int)blockIdx.x < a.out_groups) {
        // a wave joins a row
        const int id = blockIdx.x * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
        const int bh = id / rows, r = id - bh * rows;
        if (bh >= a.heads) return;
        const size_t first = (size_t)bh * a.splits * rows + r;
        // lanes in teams of D / 4, four channels each, take splits in turn, four
        // reads at a time (the first ones do not wait for length or maxima; past
        // the end the last split again, unused)
        constexpr int TEAMS = 256 / D;
        const int team = lane / (D / 4), d0 = 4 * (lane % (D / 4));
        auto part_at = [&](int k) {
            return *reinterpret_cast<const f32x4 *>(
                a.part + (first + (size_t)min(k, a.splits - 1) * rows) * D + d0);
        };
        const f32x2 stat = load_stat(a.stat, first, rows, a.splits, lane);
        const int n = optional_len(a.key_len, bh / a.H, a.L);
        f32x4 y[4], x = zero4();
#pragma unroll
        for (int u = 0; u < 4; ++u) y[u] = part_at(u * TEAMS + team);
        const int count = written_splits(a, n);
        const Joined j = join_stats(stat, count, lane);
        for (int k0 = 0; k0 < count; k0 += 4 * TEAMS)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int k = k0 + u * TEAMS + team;
                const float f = __shfl(j.factor, k & 63, 64);
                if (k < count) x += f * y[u];
                if (k0 + 4 * TEAMS < count) y[u] = part_at(k + 4 * TEAMS);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (TEAMS >= 2) x[i] = sum_xor32(x[i]);
            if (TEAMS >= 4) x[i] = sum_xor16(x[i]);
            if (TEAMS >= 8) x[i] += xor_lanes(x[i], 8);
        }
        const RowAt to = row_at(r, bh, a.G, a.Lq);
        if (team == 0) {
            const float inv = 1.f / j.sum;
            T *out = static_cast<T *>(a.O) + to.at * D + d0;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = j.sum == 0.f ? 0.f : x[i] * inv;
            store_row(out, y);
        }
        if (lane == 0) a.LSE[to.at] = j.sum != j.sum ? j.sum : row_lse(j.top, j.sum);
        return;
    }
    // weights: a thread adds the rows' probabilities of four tokens
    __shared__ float lse2[kRows];
    const int per = (a.Lp + kJoinKeys - 1) / kJoinKeys;
    const int id = blockIdx.x - a.out_groups, bh = id / per;
    const int j0 = (id - bh * per) * kJoinKeys + 4 * threadIdx.x;
    const int b = bh / a.H;
    const Kv4Mask mask = sequence_mask(a.key_len, a.q_len, b, a.L, a.Lq, a.causal);
    if ((id - bh * per) * kJoinKeys >= mask.n) return;
    // a row without sight adds nothing
    for (int r = threadIdx.x >> 6; r < rows; r += kWaves) {
        const RowAt at = row_at(r, bh, a.G, a.Lq);
        const int lane = threadIdx.x & 63;
        float v;
        if (a.splits > 1) {
            const f32x2 stat =
                load_stat(a.stat, (size_t)bh * a.splits * rows + r, rows, a.splits, lane);
            const Joined j = join_stats(stat, written_splits(a, mask.n), lane);
            v = j.sum == 0.f ? INFINITY : j.top + log2f(j.sum);
        } else {
            v = a.LSE[at.at] * kLog2e;
            if (v == -INFINITY) v = INFINITY;
        }
        if (lane == 0) lse2[r] = at.i < mask.rows ? v : INFINITY;
    }
    __syncthreads();
    if (j0 >= mask.n) return;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < rows; ++r) {
        const float z = lse2[r];
        if (z == INFINITY) continue;
        const RowAt at = row_at(r, bh, a.G, a.Lq);
        const int limit = mask.limit(at.i);
        // scores of blocks behind the row tile's last token were not written
        const f32x4 s = *reinterpret_cast<const f32x4 *>(a.score + ((size_t)bh * rows + r) * a.Lp +
                                                         j0);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j0 + k < limit) w[k] += exp2_fast(s[k] - z);
    }
    float *to = a.weight + (size_t)bh * a.L + j0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (j0 + k < mask.n) to[k] += w[k];
}

template <typename T, int D, int NP>
hipError_t rows(const Kv4Attn &p, const Kv4Plan &plan, const void *Q,
                const Kv4Cache<const uint32_t> &c, void *O, float *LSE, char *ws, hipStream_t s) {
    const int tiles = (int)((kv4_rows(p) + kRows - 1) / kRows);
    const RowsArgs a = {Q, c.k, c.v, c.kp, c.vp, O, LSE, (float *)(ws + plan.part),
                        (float *)(ws + plan.stat),
                        plan.scores ? (float *)(ws + plan.score) : nullptr, p.key_len, p.q_len,
                        p.H, p.G, p.Lq, p.L, kv4_padded(p.L), p.causal, p.scale * kLog2e,
                        plan.splits, plan.chunk, tiles};
    kv4_rows<T, D, NP><<<(unsigned)((int64_t)p.B * p.H * plan.splits * tiles), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t join(const Kv4Attn &p, const Kv4Plan &plan, void *O, float *LSE, float *weight,
                const char *ws, hipStream_t s) {
    const int64_t heads = (int64_t)p.B * p.H;
    const int64_t outs = plan.splits > 1 ? (heads * kv4_rows(p) + kWaves - 1) / kWaves : 0;
    const int64_t keys = plan.scores ? heads * cdiv(kv4_padded(p.L), kJoinKeys) : 0;
    const JoinArgs a = {O, LSE, weight, (const float *)(ws + plan.part),
                        (const float *)(ws + plan.stat), (const float *)(ws + plan.score),
                        p.key_len, p.q_len, p.H, p.G, p.Lq, p.L, kv4_padded(p.L), p.causal,
                        plan.splits, plan.rows == kRows ? plan.chunk : 0, (int)heads, (int)outs};
    kv4_join<T, D><<<(unsigned)(outs + keys), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_rows(const Kv4Attn &p, const Kv4Plan &plan, const void *Q, bool bf16,
                           const Kv4Cache<const uint32_t> &c, void *O, float *LSE, void *ws,
                           hipStream_t s) {
    char *w = static_cast<char *>(ws);
    if (bf16)
        return p.d == 32 ? rows<uint16_t, 32, 1>(p, plan, Q, c, O, LSE, w, s)
             : p.d == 64 ? rows<uint16_t, 64, 1>(p, plan, Q, c, O, LSE, w, s)
                         : rows<uint16_t, 128, 1>(p, plan, Q, c, O, LSE, w, s);
    return p.d == 32 ? rows<float, 32, 2>(p, plan, Q, c, O, LSE, w, s)
         : p.d == 64 ? rows<float, 64, 2>(p, plan, Q, c, O, LSE, w, s)
                     : rows<float, 128, 2>(p, plan, Q, c, O, LSE, w, s);
}

hipError_t launch_kv4_join(const Kv4Attn &p, const Kv4Plan &plan, bool bf16, void *O, float *LSE,
                           float *weight, const void *ws, hipStream_t s) {
    const char *w = static_cast<const char *>(ws);
    if (bf16)
        return p.d == 32 ? join<uint16_t, 32>(p, plan, O, LSE, weight, w, s)
             : p.d == 64 ? join<uint16_t, 64>(p, plan, O, LSE, weight, w, s)
                         : join<uint16_t, 128>(p, plan, O, LSE, weight, w, s);
    return p.d == 32 ? join<float, 32>(p, plan, O, LSE, weight, w, s)
         : p.d == 64 ? join<float, 64>(p, plan, O, LSE, weight, w, s)
                     : join<float, 128>(p, plan, O, LSE, weight, w, s);
}

}  // namespace mg
