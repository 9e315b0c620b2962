// kv4_device.h -- device helpers shared by the 4-bit cache's kernels.
#pragma once

#include "device_common.h"

namespace mg {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int D>
struct Kv4Dim {
    static constexpr int kGroups = D <= 64 ? 1 : D / 64;
    static constexpr int kBlocks = D / 16;                  // 16-channel blocks
    static constexpr int kWide = kBlocks < 4 ? kBlocks : 4;   // V words a lane reads at once
    static constexpr int kSteps = D / 32;                   // 32-channel products
};

// Place of channel word d/8 in a token's K row, of channel c in an octet's V row.
template <int D>
__device__ __forceinline__ int k_word(int w) { return (w & 3) * Kv4Dim<D>::kSteps + (w >> 2); }
template <int D>
__device__ __forceinline__ int v_word(int c) {
    constexpr int W = Kv4Dim<D>::kWide;
    const int b = c >> 4;
    return 16 * W * (b / W) + W * (c & 15) + b % W;
}

// A group's word: scale in the upper half, minimum in the lower.
__device__ __forceinline__ float group_scale(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float group_min(uint32_t w) { return __uint_as_float(w << 16); }

// An optional length of batch b, clamped to [0, full].
__device__ __forceinline__ int optional_len(const int32_t *len, int b, int full) {
    return key_limit(len, b, full);
}

// bf16 bits, nearest even (one conversion instruction for a pair).
__device__ __forceinline__ uint16_t to_bf16(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// The value of another lane, one step of a reduction over aligned lanes: neighbour,
// other pair of four, mirror image in eight, mirror image in sixteen.
template <int STEP>
__device__ __forceinline__ float other_lane(float v) {
    constexpr int CONTROL = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(v), CONTROL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float max_of(float v) {
    if (LANES >= 2) v = fmaxf(v, other_lane<0>(v));
    if (LANES >= 4) v = fmaxf(v, other_lane<1>(v));
    if (LANES >= 8) v = fmaxf(v, other_lane<2>(v));
    if (LANES >= 16) v = fmaxf(v, other_lane<3>(v));
    return v;
}
template <int LANES>
__device__ __forceinline__ float sum_of(float v) {
    if (LANES >= 2) v += other_lane<0>(v);
    if (LANES >= 4) v += other_lane<1>(v);
    if (LANES >= 8) v += other_lane<2>(v);
    if (LANES >= 16) v += other_lane<3>(v);
    return v;
}

// N consecutive elements as f32, N * sizeof(T) a multiple of 8 bytes.
template <int N>
__device__ __forceinline__ void load_row(float (&x)[N], const float *p) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i + k] = v[k];
    }
}
template <int N>
__device__ __forceinline__ void load_row(float (&x)[N], const uint16_t *p) {
    constexpr int W = N < 8 ? N : 8;
    typedef uint32_t words __attribute__((ext_vector_type(W / 2)));
#pragma unroll
    for (int i = 0; i < N; i += W) {
        const words v = *reinterpret_cast<const words *>(p + i);
#pragma unroll
        for (int k = 0; k < W / 2; ++k) {
            x[i + 2 * k] = __uint_as_float(v[k] << 16);
            x[i + 2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
        }
    }
}
template <int N>
__device__ __forceinline__ void store_row(float *p, const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
        *reinterpret_cast<f32x4 *>(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
}
template <int N>
__device__ __forceinline__ void store_row(uint16_t *p, const float (&x)[N]) {
    constexpr int W = N < 8 ? N : 8;
    typedef uint32_t words __attribute__((ext_vector_type(W / 2)));
#pragma unroll
    for (int i = 0; i < N; i += W) {
        words v;
#pragma unroll
        for (int k = 0; k < W / 2; ++k)
            v[k] = to_bf16(x[i + 2 * k]) | (uint32_t)to_bf16(x[i + 2 * k + 1]) << 16;
        *reinterpret_cast<words *>(p + i) = v;
    }
}

}  // namespace mg
