// paged_append.hip -- rows of K and V into their slots, and the bounds of the
// pages they go to.
//
// A wave takes R rows of one head, 16 bytes a lane, and keeps their K.  Rows, one behind
// the other, whose slots rise inside a page are a run; the wave in whose rows a run
// begins owns it, reads on to the run's end where that lies behind its rows, and
// writes its bounds: every page has one writer, and no order of waves matters.  A
// run of one row (a decode step) needs no reduction over lanes and costs nothing
// beside its row.
#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct AppendArgs {
    const char *K, *V;
    char *Kp, *Vp, *bounds;
    const int32_t *slot;
    int T, H, shift, N;
    int64_t waves;
};

template <typename T>
struct Piece {   // the elements of 16 bytes
    static constexpr int kN = 16 / sizeof(T);
    // the largest finite value
    static constexpr float kMost = sizeof(T) == 2 ? 0x1.fep127f : 0x1.fffffep127f;
    float x[kN];

    __device__ __forceinline__ static Piece of(u32x4 v) {
        Piece p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                p.x[2 * e] = __uint_as_float(v[e] << 16);
                p.x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
            } else {
                p.x[e] = __uint_as_float(v[e]);
            }
        }
        return p;
    }
    __device__ __forceinline__ void store(char *to) const {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2)
                v[e] = to_bf16(x[2 * e]) | (uint32_t)to_bf16(x[2 * e + 1]) << 16;
            else
                v[e] = __float_as_uint(x[e]);
        }
        *reinterpret_cast<u32x4 *>(to) = v;
    }
};

// Smallest and largest (fminf and fmaxf leave NaN out).
template <typename T>
struct Bounds {
    Piece<T> lo, hi;

    __device__ __forceinline__ Bounds() {
#pragma unroll
        for (int e = 0; e < Piece<T>::kN; ++e) lo.x[e] = Piece<T>::kMost, hi.x[e] = -Piece<T>::kMost;
    }
    __device__ __forceinline__ void join(const Piece<T> &l, const Piece<T> &h) {
#pragma unroll
        for (int e = 0; e < Piece<T>::kN; ++e) {
            lo.x[e] = fminf(lo.x[e], l.x[e]);
            hi.x[e] = fmaxf(hi.x[e], h.x[e]);
        }
    }
    __device__ __forceinline__ void add(const Piece<T> &p) { join(p, p); }
    // Over the lanes whose numbers differ by multiples of RL.
    template <int RL>
    __device__ __forceinline__ void join_lanes() {
#pragma unroll
        for (int e = 0; e < Piece<T>::kN; ++e) {
            float h = hi.x[e], l = -lo.x[e];   // (the largest of both)
            if (RL <= 4) h = fmaxf(h, rotated<0x124>(h)), l = fmaxf(l, rotated<0x124>(l));
            if (RL <= 8) h = fmaxf(h, rotated<0x128>(h)), l = fmaxf(l, rotated<0x128>(l));
            if (RL <= 16) h = max_xor16(h), l = max_xor16(l);
            hi.x[e] = max_xor32(h);
            lo.x[e] = -max_xor32(l);
        }
    }
    // The value of the lane so many before in a row of 16.
    template <int CONTROL>
    __device__ __forceinline__ static float rotated(float v) {
        return __int_as_float(
            __builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 0xf, 0xf, true));
    }
    // With what the page's bounds were, unless the run begins it.
    __device__ __forceinline__ void write(char *at, int row_bytes, bool begun) {
        if (begun)
            join(Piece<T>::of(*reinterpret_cast<const u32x4 *>(at)),
                 Piece<T>::of(*reinterpret_cast<const u32x4 *>(at + row_bytes)));
#pragma unroll
        for (int e = 0; e < Piece<T>::kN; ++e) {
            lo.x[e] = fmaxf(lo.x[e], -Piece<T>::kMost);   // infinities
            hi.x[e] = fminf(hi.x[e], Piece<T>::kMost);
        }
        lo.store(at);
        hi.store(at + row_bytes);
    }
};

template <typename T, int D, int NI, bool OWN, bool PAST>
__global__ __launch_bounds__(kThreads)
void paged_append(AppendArgs a) {
    constexpr int RB = D * (int)sizeof(T), RL = RB / 16;   // lanes a row
    constexpr int RPI = 64 / RL, R = RPI * NI;             // rows a read, rows at a time
    static_assert(R < 64, "a lane for every row's slot and the next one's");
    const int lane = threadIdx.x & 63, sub = lane / RL;
    const int64_t wave = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (wave >= a.waves) return;
    const int h = (int)(wave % a.H), t0 = __builtin_amdgcn_readfirstlane((int)(wave / a.H) * R);
    const int page = 1 << a.shift;
    const uint32_t slots = (uint32_t)a.N << a.shift;
    const size_t piece = (size_t)16 * (lane % RL);
    const uint64_t mine = (1ull << R) - 1;

    const auto slot_of = [&](int t) { return t < a.T ? a.slot[t] : -1; };
    const auto row_at = [&](const char *rows, int t) {
        return reinterpret_cast<const u32x4 *>(rows + ((size_t)t * a.H + h) * RB + piece);
    };
    // lane j: the slot of row t0 + j, whether it goes on with the one before
    const int slot = slot_of(t0 + lane);
    const int first = t0 > 0 ? a.slot[t0 - 1] : -1;
    const int shifted = __shfl_up(slot, 1, 64), before = lane == 0 ? first : shifted;
    const bool good = (uint32_t)slot < slots;
    const bool on = good && before < slot && before >> a.shift == slot >> a.shift;
    const uint64_t goods = __ballot(good), ons = __ballot(on), starts = goods & ~ons & mine;
    const uint64_t singles = starts & ~(ons >> 1);
    const auto end_of = [&](int from) {   // of the run that begins there, as far as is known
        const uint64_t rest = ~ons >> from >> 1;
        return from + 1 + (rest == 0 ? 64 : __builtin_ctzll(rest));
    };
    // a head's rows in the pools, and its bounds
    const auto head_of = [&](int s) { return (size_t)(s >> a.shift) * a.H + h; };
    const auto bounds_of = [&](int s) { return a.bounds + head_of(s) * 2 * RB + piece; };

    // The rows that the wave moves.  Of many rows, those without a slot are not read (few
    // do not wait for their slots).  Where pages have at most R rows, a wave moves the
    // runs that begin among its rows, whole: no row is read twice.  In two parts where
    // they are more than R, the last of them by itself.
    int base = 0, count = R, second = -1;
    if constexpr (OWN) {
        if (starts == 0) return;
        base = __builtin_ctzll(starts);
        second = 63 - __builtin_clzll(starts);
        count = end_of(second) - base;
        if (count <= R) second = -1;
        else count = second - base;
    } else if (NI > 1 && (goods & mine) == 0) {
        return;
    }
    for (;;) {
        u32x4 k[NI], v[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int t = min(t0 + base + min(i * RPI + sub, count - 1), a.T - 1);
            if constexpr (PAST) k[i] = __builtin_nontemporal_load(row_at(a.K, t));
            else k[i] = *row_at(a.K, t);
            v[i] = __builtin_nontemporal_load(row_at(a.V, t));
        }
        // the rows of the last run behind the wave's own, as far as slots are known: the
        // first of them come with the own rows
        const int behind =
            !OWN && a.bounds != nullptr && starts != 0 ? __builtin_ctzll(~(ons >> R)) : 0;
        constexpr int NX = OWN ? 1 : 4;
        u32x4 x[NX];
        if (behind > 0)
#pragma unroll
            for (int i = 0; i < NX; ++i)
                x[i] = *row_at(a.K, t0 + R + min(i * RPI + sub, behind - 1));

#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int j = base + i * RPI + sub, s = __shfl(slot, j, 64);
            if (j >= base + count || (uint32_t)s >= slots) continue;
            const size_t to = ((head_of(s) << a.shift) + (s & (page - 1))) * RB + piece;
            *reinterpret_cast<u32x4 *>(a.Kp + to) = k[i];
            *reinterpret_cast<u32x4 *>(a.Vp + to) = v[i];
            if (a.bounds != nullptr && (singles >> j & 1)) {
                Bounds<T> b;
                b.add(Piece<T>::of(k[i]));
                b.write(bounds_of(s), RB, (s & (page - 1)) != 0);
            }
        }
        if (a.bounds == nullptr) return;
        const uint64_t here = (count == 64 ? ~0ull : (1ull << count) - 1) << base;
        for (uint64_t left = starts & ~singles & here; left != 0; left &= left - 1) {
            const int from = __builtin_ctzll(left), end = end_of(from);
            const int s = __builtin_amdgcn_readlane(slot, from);
            Bounds<T> b;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                if (base + i * RPI >= end || base + (i + 1) * RPI <= from) continue;   // (uniform)
                const int j = base + i * RPI + sub;
                if (j >= from && j < end) b.add(Piece<T>::of(k[i]));
            }
            if (!OWN && end > R) {
#pragma unroll
                for (int i = 0; i < NX; ++i) b.add(Piece<T>::of(x[i]));
                // what is left of a long page
                for (int done = min(behind, NX * RPI), known = behind;;) {
                    if (done == known) {
                        // how many of the next 64 rows are the run's
                        if (R + known < 64) break;
                        const int t = t0 + R + done + lane, next = slot_of(t);
                        const bool same = next >> a.shift == s >> a.shift && slot_of(t - 1) < next;
                        const uint64_t other = ~__ballot(same);
                        const int more = other == 0 ? 64 : __builtin_ctzll(other);
                        if (more == 0) break;
                        known += more;
                    }
                    constexpr int AT_ONCE = 8;
                    u32x4 y[AT_ONCE];
#pragma unroll
                    for (int e = 0; e < AT_ONCE; ++e)   // (past the end the last row again)
                        y[e] = *row_at(a.K, t0 + R + min(done + e * RPI + sub, known - 1));
#pragma unroll
                    for (int e = 0; e < AT_ONCE; ++e) b.add(Piece<T>::of(y[e]));
                    done = min(done + AT_ONCE * RPI, known);
                }
            }
            b.template join_lanes<RL>();
            if (sub == 0) b.write(bounds_of(s), RB, (s & (page - 1)) != 0);
        }
        if (!OWN || second < 0) return;
        base = second;
        count = end_of(second) - second;
        second = -1;
    }
}

template <typename T, int D, int NI, bool OWN, bool PAST>
hipError_t append(const PagedAppend &p, AppendArgs a, hipStream_t s) {
    constexpr int R = 64 / (D * (int)sizeof(T) / 16) * NI;
    a.waves = (int64_t)((p.T + R - 1) / R) * p.H;
    paged_append<T, D, NI, OWN, PAST>
        <<<(unsigned)((a.waves + kWaves - 1) / kWaves), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

// Few rows: one read a wave, so that all compute units have some.  Many: pages of 16
// and 32 by waves of as many rows, which move whole runs (20,480 rows of 8 heads of 128
// bf16 channels into pages of 16: 33 us; 37 where a run's owner reads on behind its
// rows); longer ones by waves of 16 rows (40 us for pages of 64; a wave of 32 has
// registers for fewer waves: 43).  Rows are read past the caches (30 us instead of 36
// without bounds), but K of long pages, of which most rows are read a second time (40
// instead of 45).
template <typename T, int D>
hipError_t append(const PagedAppend &p, const AppendArgs &a, hipStream_t s) {
    constexpr int RPI = 64 / (D * (int)sizeof(T) / 16);
    constexpr int NI = 16 / RPI > 4 ? 4 : 16 / RPI > 1 ? 16 / RPI : 2;
    if ((int64_t)p.T * p.H <= 16384) return append<T, D, 1, false, false>(p, a, s);
    if (a.bounds == nullptr) return append<T, D, NI, false, true>(p, a, s);
    if (p.shift == 4) return append<T, D, 16 / RPI, true, true>(p, a, s);
    if (p.shift == 5) return append<T, D, 32 / RPI, true, true>(p, a, s);
    return append<T, D, NI, false, false>(p, a, s);
}

}  // namespace

hipError_t launch_paged_append(const PagedAppend &p, const void *K, const void *V, void *Kp,
                               void *Vp, void *bounds, bool bf16, hipStream_t s) {
    const AppendArgs a = {static_cast<const char *>(K), static_cast<const char *>(V),
                          static_cast<char *>(Kp), static_cast<char *>(Vp),
                          static_cast<char *>(bounds), p.slot, p.T, p.H, p.shift, p.N, 0};
    if (bf16)
        return p.d == 32 ? append<uint16_t, 32>(p, a, s) : p.d == 64 ? append<uint16_t, 64>(p, a, s)
                                                                     : append<uint16_t, 128>(p, a, s);
    return p.d == 32 ? append<float, 32>(p, a, s) : p.d == 64 ? append<float, 64>(p, a, s)
                                                              : append<float, 128>(p, a, s);
}

}  // namespace mg
