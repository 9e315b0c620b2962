// kv4_launch.h -- host-side launchers of the 4-bit cache's kernels (internal;
// arguments are validated in mg_kv4.cpp).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "kv4_layout.h"

namespace mg {

struct Kv4Move {          // rows of K and V into the cache, or back
    int B, H, n, L, d;
    const int32_t *start, *count;   // device [B] or nullptr
};
hipError_t launch_kv4_append(const Kv4Move &p, const void *K, const void *V, bool bf16,
                             const Kv4Cache<uint32_t> &c, float *weight, hipStream_t s);
hipError_t launch_kv4_read(const Kv4Move &p, const Kv4Cache<const uint32_t> &c, void *K, void *V,
                           bool bf16, hipStream_t s);

struct Kv4Attn {
    int B, H, G, Lq, L, d;   // G query heads a cache head
    int causal;
    float scale;
    const int32_t *key_len, *q_len;   // device [B] or nullptr
};
// Query rows that share a cache head, r = i * G + g (row i of the group's head g).
inline int64_t kv4_rows(const Kv4Attn &p) { return (int64_t)p.G * p.Lq; }

// How one call runs.
struct Kv4Plan {
    int rows;          // of a workgroup: 16 (kv4_rows) or 256 (kv4_many)
    int splits;        // workgroups that share a row tile's tokens
    int chunk;         // kv4_rows: blocks of 32 tokens of each
    bool scores;       // weights come from scores the forward keeps
    int shares;        // of the rows, where weights come from Q, K and LSE (else 0)
    size_t part, stat, score, sums, bytes;   // workspace: offsets of the parts, size
};
Kv4Plan kv4_plan(const Kv4Attn &p, bool weights, bool bf16);

hipError_t launch_kv4_rows(const Kv4Attn &p, const Kv4Plan &plan, const void *Q, bool bf16,
                           const Kv4Cache<const uint32_t> &c, void *O, float *LSE, void *ws,
                           hipStream_t s);
hipError_t launch_kv4_many(const Kv4Attn &p, const Kv4Plan &plan, const void *Q,
                           const Kv4Cache<const uint32_t> &c, void *O, float *LSE, void *ws,
                           hipStream_t s);   // bf16
// Joins the splits' outputs and adds the kept scores' probabilities to the
// weights, whichever of the two there is.
hipError_t launch_kv4_join(const Kv4Attn &p, const Kv4Plan &plan, bool bf16, void *O, float *LSE,
                           float *weight, const void *ws, hipStream_t s);
// Every row's probabilities from Q, K and LSE, added to the weights or, with
// several shares, kept for launch_kv4_weight_shares to add.
hipError_t launch_kv4_weights(const Kv4Attn &p, const Kv4Plan &plan, const void *Q, bool bf16,
                              const Kv4Cache<const uint32_t> &c, const float *LSE, float *weight,
                              void *ws, hipStream_t s);
hipError_t launch_kv4_weight_shares(const Kv4Attn &p, const Kv4Plan &plan, float *weight,
                                    const void *ws, hipStream_t s);

struct Kv4Evict {
    int B, H, L, d, keep, recent;
    const int32_t *key_len;   // device [B] or nullptr
};
hipError_t launch_kv4_select(const Kv4Evict &p, const float *weight, int32_t *index,
                             hipStream_t s);
hipError_t launch_kv4_compact(const Kv4Evict &p, const Kv4Cache<const uint32_t> &c,
                              const float *weight, const Kv4Cache<uint32_t> &out,
                              float *out_weight, const int32_t *index, int32_t *new_len,
                              bool in_place, hipStream_t s);

}  // namespace mg
