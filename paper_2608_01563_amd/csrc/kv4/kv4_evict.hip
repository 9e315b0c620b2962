// kv4_evict.hip -- the tokens of least accumulated weight leave the 4-bit cache.
//
// kv4_select: a workgroup a head finds the weight of rank keep - recent among
// the older tokens by radix selection (11 + 11 + 10 bits of a key whose order is
// the weights', LDS histograms of whole-number counts, so the result does not
// depend on the order of the counting), then writes the indices of what stays
// in order: each wave counts its share, one scan over the waves places it.  Of
// the tokens that equal the last weight, the first ones stay.
//
// kv4_compact: moves rows to where select's indices put them.  A workgroup owns
// a column of the cache (16 bytes of the K rows, 64 bytes of the V octets, or
// the group words and weights).  index[p] >= p, so going through p upwards,
// reading a stretch before any of it is written, is safe in place; into another
// cache, stretches are shared out over workgroups.
#include "cdiv.h"
#include "kv4_device.h"
#include "kv4_launch.h"

namespace mg {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;

// Order-preserving whole number of a weight; NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kThreads)
void kv4_select(const float *__restrict__ weight, int32_t *__restrict__ index,
                const int32_t *key_len, int H, int L, int keep, int recent) {
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t above[kWaves], equal[kWaves];
    __shared__ uint32_t found[2];   // digit, and how many of its bin stay
    const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = optional_len(key_len, bh / H, L);
    const float *w = weight + (size_t)bh * L;
    int32_t *to = index + (size_t)bh * keep;
    if (n <= keep) {
        for (int p = tid; p < keep; p += kThreads) to[p] = p < n ? p : -1;
        return;
    }
    const int old = n - recent;
    uint32_t want = keep - recent;   // of the old tokens; old > want
    for (int p = tid; p < recent; p += kThreads) to[want + p] = old + p;
    if (want == 0) return;

    // the key of rank `want` from the top, digit by digit
    uint32_t prefix = 0;
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : 11, below = shift - bits;
        for (int k = tid; k < kBins; k += kThreads) hist[k] = 0;
        __syncthreads();
        for (int j = tid; j < old; j += kThreads) {
            const uint32_t key = weight_key(w[j]);
            if (shift == 32 || key >> shift == prefix >> shift)
                atomicAdd(&hist[(key >> below) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            // lanes take bins from the top, 32 each
            uint32_t mine = 0;
            const int hi = kBins - 1 - 32 * lane;
            for (int k = 0; k < 32; ++k) mine += hist[hi - k];
            uint32_t before = mine;
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                const uint32_t v = __shfl_up((int)before, m, 64);
                if (lane >= m) before += v;
            }
            before -= mine;
            if (before < want && before + mine >= want) {
                uint32_t left = want - before;
                for (int k = 0; k < 32; ++k) {
                    const uint32_t h = hist[hi - k];
                    if (left <= h) {
                        found[0] = hi - k;
                        found[1] = left;
                        break;
                    }
                    left -= h;
                }
            }
        }
        __syncthreads();
        prefix |= found[0] << below;
        want = found[1];
        shift = below;
    }

    // every key above prefix stays, and the first `want` that equal it
    const int share = (old + kWaves - 1) / kWaves, j0 = wave * share, j1 = min(old, j0 + share);
    uint32_t up = 0, same = 0;
    for (int j = j0; j < j1; j += 64) {
        const uint32_t key = j + lane < j1 ? weight_key(w[j + lane]) : 0;
        up += __popcll(__ballot(j + lane < j1 && key > prefix));
        same += __popcll(__ballot(j + lane < j1 && key == prefix));
    }
    if (lane == 0) {
        above[wave] = up;
        equal[wave] = same;
    }
    __syncthreads();
    up = same = 0;
    for (int k = 0; k < wave; ++k) {
        up += above[k];
        same += equal[k];
    }
    const uint64_t lower = (1ull << lane) - 1;
    for (int j = j0; j < j1; j += 64) {
        const bool in = j + lane < j1;
        const uint32_t key = in ? weight_key(w[j + lane]) : 0;
        const uint64_t gt = __ballot(in && key > prefix), eq = __ballot(in && key == prefix);
        const uint32_t u = up + __popcll(gt & lower), s = same + __popcll(eq & lower);
        if (in && (key > prefix || (key == prefix && s < want))) to[u + min(s, want)] = j + lane;
        up += __popcll(gt);
        same += __popcll(eq);
    }
}

struct CompactArgs {
    Kv4Cache<const uint32_t> in;
    Kv4Cache<uint32_t> out;
    const float *weight;
    float *out_weight;
    const int32_t *index, *key_len;
    int32_t *new_len;
    int H, L, Lp, keep, in_place;
};

// One pass takes kRowsPass tokens of a K column or the side words, or
// kOctetsPass octets of a V column.
constexpr int kCompactThreads = 512;

template <int D>
__global__ __launch_bounds__(kCompactThreads)
void kv4_compact(CompactArgs a) {
    constexpr int NG = Kv4Dim<D>::kGroups;
    constexpr int KC = D / 32, VC = D / 16;   // 16-byte K columns, 64-byte V columns
    const int bh = blockIdx.x / (KC + VC + 1), col = blockIdx.x - bh * (KC + VC + 1);
    const int b = bh / a.H, tid = threadIdx.x;
    const int n = min(optional_len(a.key_len, b, a.L), a.keep);
    const int32_t *index = a.index + (size_t)bh * a.keep;
    if (a.new_len != nullptr && bh % a.H == 0 && col == 0 && blockIdx.y == 0 && tid == 0)
        a.new_len[b] = n;
    const size_t head = (size_t)bh * a.Lp;

    if (col < KC) {
        const u32x4 *in = reinterpret_cast<const u32x4 *>(a.in.k + head * (D / 8)) + col;
        u32x4 *out = reinterpret_cast<u32x4 *>(a.out.k + head * (D / 8)) + col;
        for (int p0 = blockIdx.y * kCompactThreads; p0 < n; p0 += gridDim.y * kCompactThreads) {
            const int p = p0 + tid;
            u32x4 v;
            if (p < n) v = in[(size_t)index[p] * KC];
            if (a.in_place) __syncthreads();
            if (p < n) out[(size_t)p * KC] = v;
        }
    } else if (col < KC + VC) {
        // a thread makes four words of an octet: eight nibbles from eight rows
        const int q = 4 * (col - KC) + (tid & 3);   // of D / 4
        const u32x4 *in = reinterpret_cast<const u32x4 *>(a.in.v + head / 8 * D) + q;
        u32x4 *out = reinterpret_cast<u32x4 *>(a.out.v + head / 8 * D) + q;
        const int octets = (n + 7) / 8;
        constexpr int PASS = kCompactThreads / 4;
        for (int o0 = blockIdx.y * PASS; o0 < octets; o0 += gridDim.y * PASS) {
            const int o = o0 + (tid >> 2);
            u32x4 v = {0u, 0u, 0u, 0u};
            if (o < octets) {
                uint32_t mask = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * o + e < n) {
                        const int j = index[8 * o + e];
                        v |= ((in[(size_t)(j >> 3) * (D / 4)] >> (uint32_t)(4 * (j & 7))) & 15u)
                             << (uint32_t)(4 * e);
                        mask |= 15u << (4 * e);
                    }
                if (mask != 0xffffffffu) v |= out[(size_t)o * (D / 4)] & ~mask;
            }
            if (a.in_place) __syncthreads();
            if (o < octets) out[(size_t)o * (D / 4)] = v;
        }
    } else {
        const uint32_t *ik = a.in.kp + head * NG, *iv = a.in.vp + head * NG;
        uint32_t *ok = a.out.kp + head * NG, *ov = a.out.vp + head * NG;
        const float *iw = a.weight + (size_t)bh * a.L;
        float *ow = a.out_weight + (size_t)bh * a.L;
        for (int p0 = blockIdx.y * kCompactThreads; p0 < n; p0 += gridDim.y * kCompactThreads) {
            const int p = p0 + tid;
            uint32_t k[NG], v[NG];
            float w = 0.f;
            if (p < n) {
                const int j = index[p];
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    k[i] = ik[(size_t)j * NG + i];
                    v[i] = iv[(size_t)j * NG + i];
                }
                w = iw[j];
            }
            if (a.in_place) __syncthreads();
            if (p < n) {
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    ok[(size_t)p * NG + i] = k[i];
                    ov[(size_t)p * NG + i] = v[i];
                }
                ow[p] = w;
            }
        }
    }
}

template <int D>
hipError_t compact(const Kv4Evict &p, const CompactArgs &a, hipStream_t s) {
    const int cols = D / 32 + D / 16 + 1;
    const dim3 grid((unsigned)(p.B * p.H * cols),
                    a.in_place ? 1u : (unsigned)cdiv(p.keep, kCompactThreads));
    kv4_compact<D><<<grid, kCompactThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_select(const Kv4Evict &p, const float *weight, int32_t *index,
                             hipStream_t s) {
    kv4_select<<<(unsigned)(p.B * p.H), kThreads, 0, s>>>(weight, index, p.key_len, p.H, p.L,
                                                          p.keep, p.recent);
    return hipGetLastError();
}

hipError_t launch_kv4_compact(const Kv4Evict &p, const Kv4Cache<const uint32_t> &c,
                              const float *weight, const Kv4Cache<uint32_t> &out,
                              float *out_weight, const int32_t *index, int32_t *new_len,
                              bool in_place, hipStream_t s) {
    const CompactArgs a = {c, out, weight, out_weight, index, p.key_len, new_len, p.H, p.L,
                           kv4_padded(p.L), p.keep, in_place ? 1 : 0};
    return p.d == 32 ? compact<32>(p, a, s) : p.d == 64 ? compact<64>(p, a, s)
                                                        : compact<128>(p, a, s);
}

}  // namespace mg
