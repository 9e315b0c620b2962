// kv4_evict.hip -- the tokens of least accumulated weight leave the 4-bit cache.
//
// kv4_select: a workgroup a head finds the weight of rank keep - recent among
// the older tokens by radix selection (11 + 11 + 10 bits of a key whose order is
// the weights', LDS histograms of whole-number counts, so the result does not
// depend on the order of the counting), then writes the indices of what stays
// in order: counts of every 64 tokens, one scan over them, places.  Of the tokens
// that equal the last weight, the first ones stay.  Weights are read once and kept
// in registers for sequences up to 32,768 tokens.  Many tokens share a digit, so
// LDS additions meet: from 4,097 tokens on first digits are counted in four places
// (16 heads of 32,768: 24 us, 26 without), else a wave adds its first lane's digit
// once for all that share it (37 us with plain additions, 27 so).  Registers are
// laid out for 4, 12 or 32 times 1,024 tokens, unused ones costing their part of the
// passes (16 heads of 5,000 to 12,000 tokens: 14.5 us with 12, 25 with 32).  Beyond, or
// without them, weights are read in every pass: 33 us at 16,384 tokens where registers
// take 25, 60 at 32,768 (25), 73 at 40,000, 222 at 131,072.
//
// kv4_compact: moves rows to where select's indices put them.  A workgroup owns
// whole 128-byte columns of the cache (the K rows, 128 bytes of the V octets, or the
// group words and weights).  index[p] >= p, so going through p upwards, reading a
// stretch of tokens before any of it is written, is safe in place; into
// another cache, stretches are shared out over workgroups.
//
// 64 heads cut from 4,096 to 1,024 tokens of 128 channels: 9 us to select, 10 to
// move; 16 heads from up to 32,768 to 8,192: 24 and 17.  Selection is bound by the
// vector and LDS work of the one compute unit a head has (5 us to load and turn
// into keys), moving by the latency of rows that follow their index.
#include "cdiv.h"
#include "kv4_device.h"
#include "kv4_launch.h"

namespace mg {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;
constexpr int kList = 4 * kBins;   // keys

// Order-preserving whole number of a weight; NaN lowest, -0 as 0.  No weight has 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 1;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ uint32_t scan_wave(uint32_t v, int lane) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint32_t x = __shfl_up((int)v, m, 64);
        if (lane >= m) v += x;
    }
    return v;
}
// Inclusive sum over the workgroup's threads; sums: kWaves words of LDS.
__device__ __forceinline__ uint32_t scan_group(uint32_t v, uint32_t *sums, int lane, int wave) {
    v = scan_wave(v, lane);
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) before += k < wave ? sums[k] : 0u;
    __syncthreads();
    return v + before;
}

// SLABS: 1,024 tokens each, the most a sequence has; 0: any number, not kept in
// registers.
template <int SLABS>
__global__ __launch_bounds__(kThreads)
void kv4_select(const float *__restrict__ weight, int32_t *__restrict__ index,
                const int32_t *key_len, int H, int L, int keep, int recent) {
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t sums[kWaves];
    __shared__ uint32_t found[3];   // digit, how many of its bin stay, how many it has
    __shared__ uint32_t counts[SLABS > 0 ? SLABS * kWaves : 1];
    constexpr bool LISTS = SLABS > 4;   // (4,096 tokens: 9.7 us with a list, 8.9 without)
    __shared__ uint32_t list[LISTS ? kList : 1];
    const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *w = weight + (size_t)bh * L;
    int32_t *to = index + (size_t)bh * keep;
    constexpr int KEYS = SLABS > 0 ? SLABS : 1;
    float raw[KEYS];
    if (SLABS > 0) {   // asked for before the length is known
#pragma unroll
        for (int i = 0; i < KEYS; ++i) raw[i] = w[min(kThreads * i + tid, L - 1)];
    }
    const int n = optional_len(key_len, bh / H, L);
    if (n <= keep) {
        for (int p = tid; p < keep; p += kThreads) to[p] = p < n ? p : -1;
        return;
    }
    const int old = n - recent;
    uint32_t want = keep - recent;   // of the old tokens; old > want
    for (int p = tid; p < recent; p += kThreads) to[want + p] = old + p;
    if (want == 0) return;
    // the keys of the thread's turns; 0 behind the old tokens
    const int turns = (old + kThreads - 1) / kThreads;
    auto key_of = [&](int i, float x) {
        return kThreads * i + tid < old ? weight_key(x) : 0u;
    };
    uint32_t kept[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i) kept[i] = SLABS > 0 ? key_of(i, raw[i]) : 0u;
    auto each = [&](auto &&f) {
        if (SLABS > 0) {
#pragma unroll
            for (int i = 0; i < KEYS; ++i) f(kept[i]);
        } else {
            for (int i = 0; i < turns; ++i) f(key_of(i, w[min(kThreads * i + tid, L - 1)]));
        }
    };

    // The key of rank `want` from the top, digit by digit.  The first digit of most
    // weights is one of few; the keys that share the one found go to a list, if they
    // fit, for the other two passes.
    uint32_t prefix = 0;
    int shift = 32, listed = -1;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : 11, below = shift - bits;
        const uint32_t mask = (1u << bits) - 1;
        const bool apart = LISTS && pass == 0;   // counted in four places, lane by lane
        for (int k = tid; k < kBins; k += kThreads) hist[k] = 0;
        if (apart)
            for (int k = tid; k < 4 * kBins; k += kThreads) list[k] = 0;
        __syncthreads();
        auto count = [&](uint32_t key) {
            const bool in = pass == 0 || (key ^ prefix) >> shift == 0;
            const uint64_t votes = __ballot(in);
            if (votes == 0) return;
            const uint32_t digit = (key >> below) & mask;
            const uint32_t first = __builtin_amdgcn_readlane(digit, __builtin_ctzll(votes));
            const uint64_t same = __ballot(in && digit == first);
            if (in && digit != first) atomicAdd(&hist[digit], 1u);
            if (lane == 0) atomicAdd(&hist[first], (uint32_t)__popcll(same));
        };
        if (apart)
            each([&](uint32_t key) { atomicAdd(&list[(key >> 21) * 4 + (lane & 3)], 1u); });
        else if (listed < 0)
            each(count);
        else   // (0, which is behind the list, shares no digit with what is sought but 0)
            for (int k = 0; k < listed; k += kThreads) {
                const bool there = k + tid < listed;
                count(there ? list[k + tid] : 0u);
            }
        __syncthreads();
        // threads take bins from the top, two each
        const int bin = kBins - 1 - 2 * tid;
        uint32_t h0 = hist[bin], h1 = hist[bin - 1];
        if (apart)
            for (int k = 0; k < 4; ++k) {
                h0 += list[4 * bin + k];
                h1 += list[4 * (bin - 1) + k];
            }
        const uint32_t upto = scan_group(h0 + h1, sums, lane, wave), before = upto - h0 - h1;
        if (before < want && upto >= want) {
            const bool second = before + h0 < want;
            found[0] = second ? bin - 1 : bin;
            found[1] = want - before - (second ? h0 : 0u);
            found[2] = second ? h1 : h0;
        }
        __syncthreads();
        prefix |= found[0] << below;
        want = found[1];
        shift = below;
        if (LISTS && pass == 0 && found[2] <= kList) {
            uint32_t n_in = 0;
            each([&](uint32_t key) { n_in += key >> 21 == prefix >> 21 ? 1u : 0u; });
            uint32_t at = scan_group(n_in, sums, lane, wave) - n_in;
            each([&](uint32_t key) {
                if (key >> 21 == prefix >> 21) list[at++] = key;
            });
            listed = (int)found[2];   // all of them; the next barrier is before they are read
        }
    }

    // Every key above prefix stays, and the first `want` that equal it: all of them,
    // most often, and then one comparison does.
    if (found[2] == want) {
        prefix -= 1;
        want = 0;
    }
    const uint64_t lower = (1ull << lane) - 1;
    auto place = [&](int i, uint32_t key, uint64_t gt, uint64_t eq, uint32_t up, uint32_t same) {
        const uint32_t u = up + __popcll(gt & lower), s = same + __popcll(eq & lower);
        if (key > prefix || (key == prefix && s < want))
            to[u + min(s, want)] = kThreads * i + tid;
    };
    if constexpr (SLABS > 0) {
        // counts of each 64 tokens: above in the upper half, equal in the lower
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            uint32_t n_in = __popcll(__ballot(kept[i] > prefix)) << 16;
            if (want > 0) n_in |= __popcll(__ballot(kept[i] == prefix));
            if (lane == 0) counts[kWaves * i + wave] = n_in;
        }
        __syncthreads();
        const uint32_t mine = tid < SLABS * kWaves ? counts[tid] : 0u;
        const uint32_t upto = scan_group(mine, sums, lane, wave);
        if (tid < SLABS * kWaves) counts[tid] = upto - mine;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const uint32_t at = counts[kWaves * i + wave];
            const uint64_t gt = __ballot(kept[i] > prefix);
            if (want == 0) {
                if (kept[i] > prefix) to[(at >> 16) + __popcll(gt & lower)] = kThreads * i + tid;
            } else {
                place(i, kept[i], gt, __ballot(kept[i] == prefix), at >> 16, at & 0xffffu);
            }
        }
    } else {
        // the same, a slab at a time
        uint32_t up = 0, same = 0;
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
            const uint32_t key = key_of(i, w[min(kThreads * i + tid, L - 1)]);
            const uint64_t gt = __ballot(key > prefix), eq = __ballot(key == prefix);
            if (lane == 0) sums[wave] = (uint32_t)__popcll(gt) << 16 | (uint32_t)__popcll(eq);
            __syncthreads();
            uint32_t here = 0, all = 0;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                here += k < wave ? sums[k] : 0u;
                all += sums[k];
            }
            place(i, key, gt, eq, up + (here >> 16), same + (here & 0xffffu));
            up += all >> 16;
            same += all & 0xffffu;
            __syncthreads();
        }
    }
}

struct CompactArgs {
    Kv4Cache<const uint32_t> in;
    Kv4Cache<uint32_t> out;
    const float *weight;
    float *out_weight;
    const int32_t *index, *key_len;
    int32_t *new_len;
    int H, L, Lp, keep;
};

// Tokens read before any is written, and threads: in place one workgroup goes through
// a column, else several share it, evened out better the smaller they are (64 heads,
// 1,024 kept tokens: 36.0 us with 1,024, 33.8 with 512, 34.2 with 256).
constexpr int stretch(bool in_place) { return in_place ? 1024 : 512; }

template <int D, bool IN_PLACE>
__global__ __launch_bounds__(stretch(IN_PLACE))
void kv4_compact(CompactArgs a) {
    constexpr int S = stretch(IN_PLACE);
    constexpr int NG = Kv4Dim<D>::kGroups;
    constexpr int VC = D / 32, COLS = VC + 2;   // V's columns, K, the rest
    const int bh = blockIdx.x / COLS, col = blockIdx.x - bh * COLS;
    const int b = bh / a.H, tid = threadIdx.x;
    const int n = min(optional_len(a.key_len, b, a.L), a.keep);
    const int32_t *index = a.index + (size_t)bh * a.keep;
    if (bh % a.H == 0 && col == 0 && blockIdx.y == 0 && tid == 0) a.new_len[b] = n;
    const size_t head = (size_t)bh * a.Lp;

    for (int p0 = blockIdx.y * S; p0 < n; p0 += gridDim.y * S) {
        if (col < VC) {
            // a thread makes four words of an octet: eight nibbles from eight rows
            const int q = 8 * col + (tid & 7);   // of D / 4
            const u32x4 *in = reinterpret_cast<const u32x4 *>(a.in.v + head / 8 * D) + q;
            u32x4 *out = reinterpret_cast<u32x4 *>(a.out.v + head / 8 * D) + q;
            const int o = p0 / 8 + (tid >> 3);
            u32x4 v = {0u, 0u, 0u, 0u};
            if (8 * o < n) {
                uint32_t mask = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool there = 8 * o + e < n;
                    const int j = index[there ? 8 * o + e : 8 * o];
                    const u32x4 x = in[(size_t)(j >> 3) * (D / 4)] >> (uint32_t)(4 * (j & 7));
                    mask |= there ? 15u << (4 * e) : 0u;
                    v |= (x & (there ? 15u : 0u)) << (uint32_t)(4 * e);
                }
                if (mask != 0xffffffffu) v |= out[(size_t)o * (D / 4)] & ~mask;
            }
            if (IN_PLACE) __syncthreads();
            if (8 * o < n) out[(size_t)o * (D / 4)] = v;
        } else if (col == VC) {
            // D / 2 bytes a token, 16 a thread
            constexpr int T = D / 32;
            const u32x4 *in = reinterpret_cast<const u32x4 *>(a.in.k + head * (D / 8));
            u32x4 *out = reinterpret_cast<u32x4 *>(a.out.k + head * (D / 8));
            u32x4 v[T];
#pragma unroll
            for (int u = 0; u < T; ++u) {
                const int p = p0 + (u * S + tid) / T;
                v[u] = in[(size_t)index[min(p, n - 1)] * T + tid % T];
            }
            if (IN_PLACE) __syncthreads();
#pragma unroll
            for (int u = 0; u < T; ++u) {
                const int p = p0 + (u * S + tid) / T;
                if (p < n) out[(size_t)p * T + tid % T] = v[u];
            }
        } else {
            const int p = p0 + tid, j = index[min(p, n - 1)];
            const uint32_t *ik = a.in.kp + (head + j) * NG, *iv = a.in.vp + (head + j) * NG;
            uint32_t k[NG], v[NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                k[i] = ik[i];
                v[i] = iv[i];
            }
            const float w = a.weight[(size_t)bh * a.L + j];
            if (IN_PLACE) __syncthreads();
            if (p < n) {
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    a.out.kp[(head + p) * NG + i] = k[i];
                    a.out.vp[(head + p) * NG + i] = v[i];
                }
                a.out_weight[(size_t)bh * a.L + p] = w;
            }
        }
    }
}

template <int D>
hipError_t compact(const Kv4Evict &p, const CompactArgs &a, bool in_place, hipStream_t s) {
    const unsigned columns = (unsigned)(p.B * p.H * (D / 32 + 2));
    if (in_place)
        kv4_compact<D, true><<<columns, stretch(true), 0, s>>>(a);
    else
        kv4_compact<D, false><<<dim3(columns, (unsigned)cdiv(p.keep, stretch(false))),
                                stretch(false), 0, s>>>(a);
    return hipGetLastError();
}

template <int SLABS>
hipError_t select(const Kv4Evict &p, const float *weight, int32_t *index, hipStream_t s) {
    kv4_select<SLABS><<<(unsigned)(p.B * p.H), kThreads, 0, s>>>(weight, index, p.key_len, p.H,
                                                                 p.L, p.keep, p.recent);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_select(const Kv4Evict &p, const float *weight, int32_t *index,
                             hipStream_t s) {
    const int slabs = cdiv(p.L, kThreads);
    return slabs <= 4 ? select<4>(p, weight, index, s) : slabs <= 12 ? select<12>(p, weight, index, s)
         : slabs <= 32 ? select<32>(p, weight, index, s) : select<0>(p, weight, index, s);
}

hipError_t launch_kv4_compact(const Kv4Evict &p, const Kv4Cache<const uint32_t> &c,
                              const float *weight, const Kv4Cache<uint32_t> &out,
                              float *out_weight, const int32_t *index, int32_t *new_len,
                              bool in_place, hipStream_t s) {
    const CompactArgs a = {c, out, weight, out_weight, index, p.key_len, new_len, p.H, p.L,
                           kv4_padded(p.L), p.keep};
    return p.d == 32 ? compact<32>(p, a, in_place, s) : p.d == 64 ? compact<64>(p, a, in_place, s)
                                                      : compact<128>(p, a, in_place, s);
}

}  // namespace mg
