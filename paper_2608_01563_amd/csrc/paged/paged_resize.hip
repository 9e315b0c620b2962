// paged_resize.hip -- block tables and slots from the sequences' lengths.
//
// Sums over the sequences say everything: rows before a sequence's, pages given
// back before its own, pages taken before its own.  paged_resize (one workgroup)
// makes them and a record of each sequence; every page given back and every row's
// slot then follows from a search in those sums, in the same workgroup where that
// is little, in the grid of paged_slots otherwise.  A page that is taken is read
// from the stack or, where it was given back in the same call, from the table of
// the sequence that lost it, so that nothing waits for what is written.
//
// Latency bounds it: one read of the lengths, two scans (what a sequence needs
// counts only if its rows fit), a search, one read of table or stack.
#include <type_traits>

#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kSlotThreads = 256;
constexpr int kHeld = 1024;   // sequences whose sums fit the LDS

// What the second part has to know of the sequences.
struct Records {
    int32_t *row_end;    // rows up to and with it, T at most
    int32_t *back_end;   // pages given back up to and with it
    int32_t *base;       // pages taken before its own; -1: no rows, or none granted
    int32_t *len;
    int32_t *left;       // pages it keeps of those it had
    int32_t *sums;       // kCount, kBack, kAvailable
};
enum { kCount, kBack, kAvailable, kSums };

// The first b with end[b] > x[e] (x below end[B - 1]), for all e at a time: a search
// waits for each of its reads, so several wait together.
template <int M>
__device__ __forceinline__ void find(const int32_t *end, int B, const int (&x)[M], int (&b)[M]) {
#pragma unroll
    for (int e = 0; e < M; ++e) b[e] = 0;
    for (int half = B > 1 ? 1 << (31 - __builtin_clz(B - 1)) : 0; half > 0; half /= 2)
#pragma unroll
        for (int e = 0; e < M; ++e)
            if (b[e] + half < B && end[b[e] + half - 1] <= x[e]) b[e] += half;
}

// Slots and pages given back (M at a time), by threads first, first + step, ...;
// r.row_end and r.back_end may be copies in LDS.
template <int M>
__device__ __forceinline__ void pages_and_slots(const PagedResize &p, const Records &r, int first,
                                                int step) {
    const int count = r.sums[kCount], back = r.sums[kBack], available = r.sums[kAvailable];
    // the k-th page given back, the k-th page taken
    const auto entry_of = [&](int b, int k) {
        return (size_t)b * p.P + r.left[b] + k - (b > 0 ? r.back_end[b - 1] : 0);
    };
    const auto given = [&](int k) {
        const int x[1] = {k};
        int b[1];
        find(r.back_end, p.B, x, b);
        return p.table[entry_of(b[0], k)];
    };
    const auto taken = [&](int k) {
        const int at = available - 1 - k;
        return at < count ? p.free_pages[at] : given(at - count);
    };
    // pages given back: the first M are on their way while slots are found
    const int pushed = min(back, p.N - count);
    int x[M], b[M], id[M];
    const auto read = [&](int k) {
#pragma unroll
        for (int e = 0; e < M; ++e) x[e] = min(k + e * step, pushed - 1);
        find(r.back_end, p.B, x, b);
#pragma unroll
        for (int e = 0; e < M; ++e) id[e] = p.table[entry_of(b[e], x[e])];
    };
    if (first < pushed) read(first);

    const int rows = r.row_end[p.B - 1], page = 1 << p.shift;
    for (int t = first; t < p.T; t += step) {
        int slot = -1;
        if (t < rows) {
            const int at_row[1] = {t};
            int found[1];
            find(r.row_end, p.B, at_row, found);
            const int b = found[0], base = r.base[b];
            if (base >= 0) {
                const int len = r.len[b], have = (len + page - 1) >> p.shift;
                const int pos = len + t - (b > 0 ? r.row_end[b - 1] : 0), at = pos >> p.shift;
                int32_t *entry = p.table + (size_t)b * p.P + at;
                const int id = at < have ? *entry : taken(base + at - have);
                const int row = pos & (page - 1);
                if (at >= have && row == 0) *entry = id;
                if ((uint32_t)id < (uint32_t)p.N) slot = (id << p.shift) + row;
            }
        }
        p.slot[t] = slot;
    }
    for (int k = first; k < pushed; k += M * step) {
        if (k > first) read(k);
#pragma unroll
        for (int e = 0; e < M; ++e)
            if (k + e * step < pushed) p.free_pages[count + k + e * step] = id[e];
    }
}

// Sums over the threads up to and with each one, and over all, of two values at a
// time.  `part` may be written again behind another barrier.
template <int THREADS, typename A, typename B>
__device__ __forceinline__ void block_scan(A &a, B &b, A &all_a, B &all_b, A *part_a, B *part_b) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    a = wave_scan(a);
    b = wave_scan(b);
    if (lane == 63) {
        part_a[w] = a;
        part_b[w] = b;
    }
    __syncthreads();
    all_a = 0;
    all_b = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        const A x = part_a[k];
        const B y = part_b[k];
        if (k < w) {
            a += x;
            b += y;
        }
        all_a += x;
        all_b += y;
    }
}

// ALONE: at most THREADS sequences, records in LDS, and the second part follows.
template <int THREADS, bool ALONE>
__global__ __launch_bounds__(THREADS)
void paged_resize(PagedResize p, Records r) {
    constexpr int W = THREADS / 64;
    using Rows = std::conditional_t<ALONE, int32_t, int64_t>;   // T and THREADS are small: clamped
    __shared__ Rows wide[W];
    __shared__ int32_t part[3][W], sums[kSums];
    __shared__ int32_t records[5][ALONE ? THREADS : 1];
    if constexpr (ALONE)
        r = {records[0], records[1], records[2], records[3], records[4], sums};
    const int tid = threadIdx.x, page = 1 << p.shift, capacity = p.P << p.shift;
    const auto pages = [&](int n) { return (int)(((int64_t)n + page - 1) >> p.shift); };
    const int count = min(max(p.free_count[0], 0), p.N);
    struct Sequence {
        int len, goal;
    };
    const auto sequence = [&](int b) {
        if (b >= p.B) return Sequence{0, 0};
        return Sequence{min(max(p.key_len[b], 0), capacity), max(p.want[b], 0)};
    };
    const auto back_of = [&](Sequence q) { return max(pages(q.len) - pages(q.goal), 0); };

    // pages given back by all come first: they may be taken by any
    int back_total = 0;
    if (p.B > THREADS) {
        int none = 0, nothing;
        for (int b = tid; b < p.B; b += THREADS) none += back_of(sequence(b));
        int same = 0;
        block_scan<THREADS>(none, same, back_total, nothing, part[1], part[2]);
    }
    Rows rows_before = 0;
    int need_before = 0, back_before = 0, took_before = 0;
    for (int b0 = 0; b0 < p.B; b0 += THREADS) {
        const int b = b0 + tid;
        const Sequence q = sequence(b);
        const int add = max(q.goal - q.len, 0);
        Rows row_end = min(add, p.T + 1), rows;   // (one row too many is as bad as more)
        int back_end = back_of(q), backs;
        block_scan<THREADS>(row_end, back_end, rows, backs, wide, part[0]);
        row_end += rows_before;
        if (p.B <= THREADS) back_total = backs;
        const int available = (int)min((int64_t)count + back_total, (int64_t)p.N);
        const bool fits = add > 0 && q.goal <= capacity && row_end <= p.T;
        const int need = fits ? pages(q.goal) - pages(q.len) : 0;
        // whether a sequence is granted its pages hangs on those before it only: they
        // are, if it is
        int need_end = need, all, unused = 0, none;
        block_scan<THREADS>(need_end, unused, all, none, part[1], part[2]);
        need_end += need_before;
        const bool granted = fits && (need == 0 || need_end <= available);
        if (granted && need > 0) took_before = need_end;
        if (b < p.B) {
            const int upto = (int)min(row_end, (Rows)p.T);
            r.row_end[b] = upto;
            r.back_end[b] = back_before + back_end;
            r.base[b] = granted ? need_end - need : -1;
            r.len[b] = q.len;
            r.left[b] = pages(q.goal);
            p.offset[b + 1] = upto;
            if (b == 0) p.offset[0] = 0;
            p.new_len[b] = add == 0 || granted ? q.goal : q.len;
        }
        rows_before += rows;
        back_before += backs;
        need_before += all;
    }
    // pages taken: up to the last granted sequence's (part[0] was read before the last
    // scan's barrier; part[1] and part[2] are read behind it)
#pragma unroll
    for (int m = 1; m < 64; m *= 2) took_before = max(took_before, __shfl_xor(took_before, m, 64));
    if ((tid & 63) == 0) part[0][tid >> 6] = took_before;
    const int available = (int)min((int64_t)count + back_total, (int64_t)p.N);
    if (tid == 0) {
        r.sums[kCount] = count;
        r.sums[kBack] = back_total;
        r.sums[kAvailable] = available;
    }
    __syncthreads();
    if (tid == 0) {
        int took = 0;
        for (int k = 0; k < W; ++k) took = max(took, part[0][k]);
        p.new_count[0] = available - took;
    }
    if constexpr (ALONE) pages_and_slots<4>(p, r, tid, THREADS);
}

__global__ __launch_bounds__(kSlotThreads)
void paged_slots(PagedResize p, Records r) {
    __shared__ int32_t ends[2][kHeld];
    if (p.B <= kHeld) {
        for (int b = threadIdx.x; b < p.B; b += kSlotThreads) {
            ends[0][b] = r.row_end[b];
            ends[1][b] = r.back_end[b];
        }
        __syncthreads();
        r.row_end = ends[0];
        r.back_end = ends[1];
    }
    pages_and_slots<1>(p, r, blockIdx.x * kSlotThreads + threadIdx.x, gridDim.x * kSlotThreads);
}

Records records_of(const PagedResize &p, void *ws) {
    int32_t *w = static_cast<int32_t *>(ws);
    const size_t B = p.B;
    return {w + kSums, w + kSums + B, w + kSums + 2 * B, w + kSums + 3 * B, w + kSums + 4 * B, w};
}

}  // namespace

// (Pages given back do not count here: some 10,000 cost nothing, 65,536 take 25 us where
// the grid needs 8.)
bool paged_resize_alone(int B, int T) { return B <= 1024 && T <= 2048; }

size_t paged_resize_bytes(int B, int T) {
    return paged_resize_alone(B, T) ? 0 : ((size_t)5 * B + kSums) * 4;
}

hipError_t launch_paged_resize(const PagedResize &p, void *ws, hipStream_t s) {
    if (!paged_resize_alone(p.B, p.T))
        paged_resize<1024, false><<<1, 1024, 0, s>>>(p, records_of(p, ws));
    else
        paged_resize<1024, true><<<1, 1024, 0, s>>>(p, Records{});
    return hipGetLastError();
}

hipError_t launch_paged_slots(const PagedResize &p, const void *ws, hipStream_t s) {
    const int groups = (p.T + kSlotThreads - 1) / kSlotThreads;
    paged_slots<<<groups < 2048 ? (groups < 64 ? 64 : groups) : 2048, kSlotThreads, 0, s>>>(
        p, records_of(p, const_cast<void *>(ws)));
    return hipGetLastError();
}

}  // namespace mg
