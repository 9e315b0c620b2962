// paged_launch.h -- host-side launchers of the paged cache's kernels (internal;
// arguments are validated in mg_paged.cpp).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace mg {

struct PagedResize {
    int B, shift, P, N, T;   // page = 1 << shift
    const int32_t *key_len, *want;
    int32_t *table, *free_pages;
    const int32_t *free_count;
    int32_t *new_len, *new_count, *slot, *offset;
};
// Whether one workgroup does it all; otherwise records of the sequences go
// through the workspace.
bool paged_resize_alone(int B, int T);
size_t paged_resize_bytes(int B, int T);
hipError_t launch_paged_resize(const PagedResize &p, void *ws, hipStream_t s);
hipError_t launch_paged_slots(const PagedResize &p, const void *ws, hipStream_t s);

struct PagedAppend {
    int T, H, d, shift, N;
    const int32_t *slot;
};
hipError_t launch_paged_append(const PagedAppend &p, const void *K, const void *V, void *Kp,
                               void *Vp, void *bounds, bool bf16, hipStream_t s);

// Query rows over the pages; index: nullptr, or the pages that each row sees.
struct PagedAttn {
    int B, H, G, Lq, d;   // G query heads a cache head
    int shift, P, N, causal, keep;
    bool half;   // bf16, else f32
    float scale;
    const int32_t *table, *index, *key_len, *q_len;
};
// The query rows that a unit's workgroups work on, and of how many units' kind
// there is one: sequences, or (sparse) their rows.
inline int64_t paged_rows(const PagedAttn &p, bool sparse) {
    return sparse ? p.G : (int64_t)p.G * p.Lq;
}

constexpr int kPagedScanned = 256;   // sequences whose lengths every wave can scan

// How one call runs: every sequence (sparse: every query row) is cut into units
// of the same number of blocks of 32 tokens, each a workgroup for every cache
// head and so many of the rows that share it.
struct PagedPlan {
    int units;     // of the grid, enough for any lengths
    int splits;    // units of every sequence; 0: as many as its length asks for
    int chunk;     // blocks of a unit (splits 0: at least)
    int share;     // splits 0: units that all lengths together are cut into
    int round, round_most;   // splits 0: units of one round, two or three a compute unit
    int rows;      // of a workgroup: 16, 32, 64 or 128
    int groups;    // workgroups of a unit and cache head
    bool once;     // K and V are read past the caches
    int most;      // units a sequence has at most
    int join_waves;   // that join a row: 1 or 4
    bool lengths;     // the units are found by a kernel of their own
    size_t part, stat, info, map, bytes;   // workspace: offsets of the parts, size
};
PagedPlan paged_plan(const PagedAttn &p, bool sparse);

hipError_t launch_paged_cut(const PagedAttn &p, const PagedPlan &plan, void *ws, hipStream_t s);
hipError_t launch_paged_attn(const PagedAttn &p, const PagedPlan &plan, const void *Q,
                             const void *Kp, const void *Vp, void *O, float *LSE, void *ws,
                             hipStream_t s);
hipError_t launch_paged_join(const PagedAttn &p, const PagedPlan &plan, void *O, float *LSE,
                             const void *ws, hipStream_t s);

struct PagedSelect {
    int B, H, G, Lq, d, shift, P, N, causal, keep, first, recent;
    const int32_t *table, *key_len, *q_len;
};
hipError_t launch_paged_scores(const PagedSelect &p, const void *Q, const void *bounds, bool bf16,
                               float *score, hipStream_t s);
hipError_t launch_paged_select(const PagedSelect &p, const float *score, int32_t *index,
                               hipStream_t s);

}  // namespace mg
