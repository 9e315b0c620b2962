// paged_device.h -- device helpers shared by the paged cache's kernels.
#pragma once

#include "device_common.h"
#include "kv4/kv4_device.h"

namespace mg {

// What a sequence's rows see: row i the first limit(i) of its n tokens.
struct PagedMask {
    int n, rows, causal;

    __device__ __forceinline__ int limit(int i) const {
        if (i >= rows) return 0;
        return max(causal ? min(n, i + 1 + n - rows) : n, 0);
    }
};
__device__ __forceinline__ PagedMask paged_mask(const int32_t *key_len, const int32_t *q_len,
                                                int b, int capacity, int Lq, int causal) {
    return {optional_len(key_len, b, capacity), optional_len(q_len, b, Lq), causal};
}

// Sums over a wave: of all lanes, and of the lanes up to each one.
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
    return v;
}
template <typename T>
__device__ __forceinline__ T wave_scan(T v, int lane) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const T x = __shfl_up(v, m, 64);
        if (lane >= m) v += x;
    }
    return v;
}

}  // namespace mg
