// kv4_weights.hip -- the attention probabilities that more than a few rows give
// each cached token, from Q, K and LSE: weight_j += sum over rows of
// exp(S_ij - LSE_i).
//
// Tokens stay, rows stream: a wave keeps the codes (strict: less 8, as the forward that
// made LSE does) of 32 tokens in registers and takes rows 32 at a time (32x32x16
// products, S^T as in kv4_many.hip) from LDS, where its workgroup's eight waves prepare
// them once: scaled f16 operands, group sums, exponents, LSE and limits.  Sums stay in
// the lanes until the end.  Where token tiles are too few for the GPU, the rows are
// shared out too, and shares of a weight are added in order by a second kernel.
//
// 16 heads of 16,384 causal rows over 4,096 tokens of 128 channels: 274 us, half of
// it vector instructions (about 200 for 32 x 32 probabilities, 16 of them
// exponentials), a quarter matrix products.  Two workgroups a compute unit need at
// most 128 registers, so scales come from LDS (with them in registers: 416 us where this made 286).
#include "cdiv.h"
#include "kv4_launch.h"
#include "kv4_tile.h"

namespace mg {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kUnits = 256;          // compute units
constexpr int kTile = 32 * kWaves;   // tokens of a workgroup

struct WeightArgs {
    const void *Q;
    const uint32_t *kw, *kp;
    const float *LSE;
    float *weight, *part;   // part [share][B*H][Lp], or null: add to weight
    const int32_t *key_len, *q_len;
    int H, G, Lq, L, Lp, causal, tiles, shares, heads;
    float scale_log2;
};

template <typename T, int D, int NP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4, 8)))
void kv4_weights(WeightArgs a) {
    constexpr int NG = Kv4Dim<D>::kGroups, NS = D / 16, KR = D / 8;
    constexpr int PER = KR;   // threads that prepare a row, 8 channels each
    __shared__ __attribute__((aligned(16))) f16x8 Qs[2][NP][32 * (KR + 1)];
    __shared__ float Sum[2][2][32], Lse[2][32];
    __shared__ int Exponent[2][32], Limit[2][32];
    __shared__ __attribute__((aligned(16))) float Scale[kWaves][NG][32];

    const int tid = threadIdx.x, lane = tid & 63, c = lane & 31, h = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the first tiles, which causal rows see the most, first; where a compute unit
    // gets two workgroups and no more, its second is the lighter the heavier the
    // first is
    const int all = gridDim.x, order = blockIdx.x;
    const int item = all <= 2 * kUnits && order >= kUnits ? all - 1 - (order - kUnits) : order;
    const int tile = item / (a.heads * a.shares), rest = item - tile * a.heads * a.shares;
    const int bh = rest / a.shares, share = rest - bh * a.shares;
    const Kv4Mask mask = sequence_mask(a.key_len, a.q_len, bh / a.H, a.L, a.Lq, a.causal);
    const int j0 = kTile * tile;
    if (j0 >= mask.n) return;

    // rows that see the tile's first token, 32 at a time, this share's
    const int rows = mask.rows * a.G;
    const int first = a.causal ? max(0, j0 - (mask.n - mask.rows)) * a.G / 32 : 0;
    const int blocks = (rows + 31) / 32 - first, each = (blocks + a.shares - 1) / a.shares;
    const int begin = first + share * each, stop = first + min(blocks, (share + 1) * each);

    // the wave's tokens: row i of a product is token_of(i); behind the padded
    // end (where none counts) the last block again
    const size_t head = (size_t)bh * a.Lp;
    const int mine = j0 + 32 * w, base = min(mine, a.Lp - 32);
    const uint32_t *kw = a.kw + (head + base) * KR, *kp = a.kp + (head + base) * NG;
    f16x8 code[NS];
    const int tok = token_of(c);
#pragma unroll
    for (int s = 0; s < NS; ++s)   // channels 16s + 8h + e: word 2s + h of the row
        code[s] = operand_of<NP>(kw[tok * KR + k_word<D>(2 * s + h)]);
    // Scales and bases are taken over 2^size, the largest of the wave's tokens (those
    // that are there and finite), and factors times it, so that products stay in range.
    const uint32_t own = kp[c * NG + (NG == 2 ? h : 0)];
    const float most = fmaxf(0x1p-4f * fabsf(group_min(own)), group_scale(own));
    const int size = 4 + __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(
        max_of_wave(base + c < mask.n && most < INFINITY ? most : 0.f)));
    if (h < NG) Scale[w][h][c] = ldexpf(group_scale(own), -size);   // read by the wave itself
    const float low =
        NG == 2 || h == 0 ? ldexpf(base_of<NP>(kp[tok * NG + (NG == 2 ? h : 0)]), -size) : 0.f;

    // preparing rows: thread r * PER + k takes channels 8k..8k+7 of row r
    const int pr = tid / PER, pk = tid % PER;
    const bool prepares = tid < 32 * PER;
    float x[8];
    float lse = 0.f;
    int limit = 0;
    // its query row i and head g in the next block, a block's step of both
    int i = (32 * begin + pr) / a.G, g = 32 * begin + pr - i * a.G;
    const int step_i = 32 / a.G, step_g = 32 - step_i * a.G;
    const T *qs = static_cast<const T *>(a.Q) + (size_t)bh * a.G * a.Lq * D + 8 * pk;
    const float *lses = a.LSE + (size_t)bh * a.G * a.Lq;
    auto fetch = [&](int block) {   // called for one block after the other
        if (!prepares) return;
        const bool in = i < mask.rows && block < stop;
        const int at = in ? g * a.Lq + i : 0;
        load_row(x, qs + (size_t)at * D);
        lse = lses[at];
        // nothing from rows without sight (LSE -inf)
        limit = in && lse != -INFINITY ? mask.limit(i) : 0;
        g += step_g;
        i += step_i + (g >= a.G ? 1 : 0);
        g -= g >= a.G ? a.G : 0;
    };
    auto put = [&](int buf) {
        if (!prepares) return;
        float top = 0.f, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
        top = max_of<PER>(top);
        const int exponent = __builtin_amdgcn_frexp_expf(top);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = ldexpf(x[e], 15 - exponent);
            sum += x[e];
        }
        sum = sum_of<PER / NG>(sum);
        f16x8 part[NP];
        split_operand<NP>(part, x);
#pragma unroll
        for (int p = 0; p < NP; ++p) Qs[buf][p][piece<KR>(pr, pk)] = part[p];
        if (pk % (PER / NG) == 0) Sum[buf][pk / (PER / NG)][pr] = sum * 0x1p-9f;
        if (pk == 0) {
            if (NG == 1) Sum[buf][1][pr] = 0.f;
            Exponent[buf][pr] = top > 0.f ? exponent - 6 : kNoSize;   // (zeros: scores of 0)
            Lse[buf][pr] = lse * kLog2e;
            Limit[buf][pr] = limit;
        }
    };

    float sum[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[v] = 0.f;
    if (begin < stop) {
        fetch(begin);
        put(0);
        fetch(begin + 1);
        __syncthreads();
        for (int block = begin; block < stop; ++block) {
            const int buf = (block - begin) & 1;
            f32x16 s = mfma32x32x2(low, Sum[buf][h][c], zero16());
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                f32x16 part = zero16();
#pragma unroll
                for (int k = g * (NS / NG); k < (g + 1) * (NS / NG); ++k)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        part = mfma32x32x16f16(code[k], Qs[buf][p][piece<KR>(c, 2 * k + h)], part);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const f32x4 scale = *reinterpret_cast<const f32x4 *>(
                        &Scale[w][g][16 * (u >> 1) + 8 * h + 4 * (u & 1)]);
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s[4 * u + v] = fmaf(part[4 * u + v], scale[v], s[4 * u + v]);
                }
            }
            const float factor = ldexpf(a.scale_log2, Exponent[buf][c] + size);
            const float off = Lse[buf][c];
            const int left = Limit[buf][c] - mine - 8 * h;
            if (__all(left > 23)) {   // every row sees every token
#pragma unroll
                for (int v = 0; v < 16; ++v) sum[v] += exp2_fast(fmaf(s[v], factor, -off));
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float p = exp2_fast(fmaf(s[v], factor, -off));
                    sum[v] += 16 * (v >> 3) + (v & 7) < left ? p : 0.f;
                }
            }
            // first of all, as every wave waits for it (286 us without, 273)
            __builtin_amdgcn_s_setprio(1);
            put(buf ^ 1);
            fetch(block + 2);
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();
        }
    }
    // over the rows; lane 32h + v keeps register v's token
    float mine_sum = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        float t = sum[v];
#pragma unroll
        for (int m = 1; m < 32; m *= 2) t += xor_lanes(t, m);
        mine_sum = c == v ? t : mine_sum;
    }
    const int j = mine + 16 * (c >> 3) + 8 * h + (c & 7);
    if (c < 16 && j < mask.n) {
        if (a.part != nullptr)
            a.part[((size_t)share * a.heads + bh) * a.Lp + j] = mine_sum;
        else
            a.weight[(size_t)bh * a.L + j] += mine_sum;
    }
}

// A thread adds a token's shares, in order.
__global__ __launch_bounds__(256)
void kv4_weight_shares(const float *__restrict__ part, float *__restrict__ weight,
                       const int32_t *key_len, int H, int L, int Lp, int shares, int heads,
                       int groups) {
    const int bh = blockIdx.x / groups, j = (blockIdx.x - bh * groups) * 256 + threadIdx.x;
    if (j >= optional_len(key_len, bh / H, L)) return;
    float sum = 0.f;
    for (int k = 0; k < shares; ++k) sum += part[((size_t)k * heads + bh) * Lp + j];
    weight[(size_t)bh * L + j] += sum;
}

template <typename T, int D, int NP>
hipError_t weights(const Kv4Attn &p, const Kv4Plan &plan, const void *Q,
                   const Kv4Cache<const uint32_t> &c, const float *LSE, float *weight, char *ws,
                   hipStream_t s) {
    const int tiles = cdiv(kv4_padded(p.L), kTile), heads = p.B * p.H;
    const WeightArgs a = {Q, c.k, c.kp, LSE, weight,
                          plan.shares > 1 ? (float *)(ws + plan.sums) : nullptr, p.key_len,
                          p.q_len, p.H, p.G, p.Lq, p.L, kv4_padded(p.L), p.causal, tiles,
                          plan.shares, heads, p.scale * kLog2e};
    kv4_weights<T, D, NP><<<(unsigned)((int64_t)heads * tiles * plan.shares), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_weights(const Kv4Attn &p, const Kv4Plan &plan, const void *Q, bool bf16,
                              const Kv4Cache<const uint32_t> &c, const float *LSE, float *weight,
                              void *ws, hipStream_t s) {
    char *w = static_cast<char *>(ws);
    if (bf16)
        return p.d == 32 ? weights<uint16_t, 32, 1>(p, plan, Q, c, LSE, weight, w, s)
             : p.d == 64 ? weights<uint16_t, 64, 1>(p, plan, Q, c, LSE, weight, w, s)
                         : weights<uint16_t, 128, 1>(p, plan, Q, c, LSE, weight, w, s);
    return p.d == 32 ? weights<float, 32, 2>(p, plan, Q, c, LSE, weight, w, s)
         : p.d == 64 ? weights<float, 64, 2>(p, plan, Q, c, LSE, weight, w, s)
                     : weights<float, 128, 2>(p, plan, Q, c, LSE, weight, w, s);
}

hipError_t launch_kv4_weight_shares(const Kv4Attn &p, const Kv4Plan &plan, float *weight,
                                    const void *ws, hipStream_t s) {
    const int groups = cdiv(p.L, 256), heads = p.B * p.H;
    kv4_weight_shares<<<(unsigned)((int64_t)heads * groups), 256, 0, s>>>(
        (const float *)(static_cast<const char *>(ws) + plan.sums), weight, p.key_len, p.H, p.L,
        kv4_padded(p.L), plan.shares, heads, groups);
    return hipGetLastError();
}

}  // namespace mg
