// paged_resize.hip -- block tables and slots from the sequences' lengths.
//
// Sums over the sequences say everything: rows before a sequence's, pages given
// back before its own, pages taken before its own.  paged_resize (one workgroup)
// makes them and a record of each sequence; every page given back and every row's
// slot then follows from a search in those sums, in the same workgroup where that
// is little, in the grid of paged_slots otherwise.  A page that is taken is read
// from the stack or, where it was given back in the same call, from the table of
// the sequence that lost it, so that nothing waits for what is written.
#include "paged_device.h"
#include "paged_launch.h"

namespace mg {
namespace {

constexpr int kThreads = 1024;
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

// The first b with end[b] > x (x below end[B - 1]).
__device__ __forceinline__ int find(const int32_t *end, int B, int x) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (end[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Pages given back and slots, by threads first, first + step, ...; r.row_end and
// r.back_end may be copies in LDS.
__device__ __forceinline__ void pages_and_slots(const PagedResize &p, const Records &r, int first,
                                                int step) {
    const int count = r.sums[kCount], back = r.sums[kBack], available = r.sums[kAvailable];
    // the k-th page given back, the k-th page taken
    const auto given = [&](int k) {
        const int b = find(r.back_end, p.B, k);
        return p.table[(size_t)b * p.P + r.left[b] + k - (b > 0 ? r.back_end[b - 1] : 0)];
    };
    const auto taken = [&](int k) {
        const int at = available - 1 - k;
        return at < count ? p.free_pages[at] : given(at - count);
    };
    for (int k = first; k < back && k < p.N - count; k += step) p.free_pages[count + k] = given(k);
    const int rows = r.row_end[p.B - 1], page = 1 << p.shift;
    for (int t = first; t < p.T; t += step) {
        int slot = -1;
        if (t < rows) {
            const int b = find(r.row_end, p.B, t), base = r.base[b];
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
}

// Sum over the threads before, and with, each one; `total` over all.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T *part, T &total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const T upto = wave_scan(v, lane);
    __syncthreads();   // the last scan's parts have been read
    if (lane == 63) part[w] = upto;
    __syncthreads();
    T before = 0;
    total = 0;
    for (int k = 0; k < kThreads / 64; ++k) {
        if (k < w) before += part[k];
        total += part[k];
    }
    return before + upto;
}

// ALONE: at most kHeld sequences, records in LDS, and the second part follows.
template <bool ALONE>
__global__ __launch_bounds__(kThreads)
void paged_resize(PagedResize p, Records r) {
    __shared__ int64_t wide[kThreads / 64];
    __shared__ int32_t part[kThreads / 64];
    __shared__ int32_t kept, sums[kSums];
    __shared__ int32_t records[5][ALONE ? kHeld : 1];
    if constexpr (ALONE) {
        r = {records[0], records[1], records[2], records[3], records[4], sums};
    }
    const int tid = threadIdx.x, page = 1 << p.shift, capacity = p.P << p.shift;
    const auto pages = [&](int n) { return (int)(((int64_t)n + page - 1) >> p.shift); };
    const int count = min(max(p.free_count[0], 0), p.N);
    if (tid == 0) kept = 0;

    int back_total = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        int back = 0;
        if (b < p.B) {
            const int len = min(max(p.key_len[b], 0), capacity), goal = max(p.want[b], 0);
            back = max(pages(len) - pages(goal), 0);
        }
        int total;
        const int end = back_total + block_scan(back, part, total);
        if (b < p.B) r.back_end[b] = end;
        back_total += total;
    }
    const int available = (int)min((int64_t)count + back_total, (int64_t)p.N);

    int64_t rows_before = 0;
    int need_before = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        int len = 0, goal = 0;
        if (b < p.B) {
            len = min(max(p.key_len[b], 0), capacity);
            goal = max(p.want[b], 0);
        }
        const int add = max(goal - len, 0);
        int64_t rows;
        const int64_t row_end = rows_before + block_scan((int64_t)add, wide, rows);
        const bool fits = add > 0 && goal <= capacity && row_end <= p.T;
        const int need = fits ? pages(goal) - pages(len) : 0;
        int all;
        const int end = need_before + block_scan(need, part, all);
        const bool granted = fits && (need == 0 || end <= available);
        if (granted && need > 0) atomicAdd(&kept, need);
        if (b < p.B) {
            const int upto = (int)min(row_end, (int64_t)p.T);
            r.row_end[b] = upto;
            r.base[b] = granted ? end - need : -1;
            r.len[b] = len;
            r.left[b] = pages(goal);
            p.offset[b + 1] = upto;
            if (b == 0) p.offset[0] = 0;
            p.new_len[b] = add == 0 || granted ? goal : len;
        }
        rows_before += rows;
        need_before += all;
    }
    if (tid == 0) {
        r.sums[kCount] = count;
        r.sums[kBack] = back_total;
        r.sums[kAvailable] = available;
    }
    __syncthreads();
    if (tid == 0) p.new_count[0] = available - kept;
    if constexpr (ALONE) pages_and_slots(p, r, tid, kThreads);
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
    pages_and_slots(p, r, blockIdx.x * kSlotThreads + threadIdx.x, gridDim.x * kSlotThreads);
}

Records records_of(const PagedResize &p, void *ws) {
    int32_t *w = static_cast<int32_t *>(ws);
    const size_t B = p.B;
    return {w + kSums, w + kSums + B, w + kSums + 2 * B, w + kSums + 3 * B, w + kSums + 4 * B, w};
}

}  // namespace

bool paged_resize_alone(int B, int T) { return B <= kHeld && T <= 2048; }

size_t paged_resize_bytes(int B, int T) {
    return paged_resize_alone(B, T) ? 0 : ((size_t)5 * B + kSums) * 4;
}

hipError_t launch_paged_resize(const PagedResize &p, void *ws, hipStream_t s) {
    if (paged_resize_alone(p.B, p.T))
        paged_resize<true><<<1, kThreads, 0, s>>>(p, Records{});
    else
        paged_resize<false><<<1, kThreads, 0, s>>>(p, records_of(p, ws));
    return hipGetLastError();
}

hipError_t launch_paged_slots(const PagedResize &p, const void *ws, hipStream_t s) {
    const int groups = (p.T + kSlotThreads - 1) / kSlotThreads;
    paged_slots<<<groups < 2048 ? (groups < 64 ? 64 : groups) : 2048, kSlotThreads, 0, s>>>(
        p, records_of(p, const_cast<void *>(ws)));
    return hipGetLastError();
}

}  // namespace mg
