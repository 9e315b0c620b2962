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

// Sums over a wave: of the lanes up to each one, and of all.  32-bit values go
// through the register file: 1, 2, 4 and 8 lanes down a row of 16, then a row's last
// lane to the next row (mask 0xa) and the second row's to the upper half (0xc).
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint32_t add_from(uint32_t v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CONTROL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = add_from<0x111, 0xf>(v);
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v);
    return add_from<0x143, 0xc>(v);
}
__device__ __forceinline__ int32_t wave_scan(int32_t v) { return (int32_t)wave_scan((uint32_t)v); }
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int64_t x = __shfl_up(v, m, 64);
        if (lane >= m) v += x;
    }
    return v;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
    return __builtin_amdgcn_readlane(wave_scan(v), 63);
}

}  // namespace mg
