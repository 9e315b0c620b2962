// kv4_layout.h -- where the parts of a 4-bit key/value cache lie (host and
// device; the layout itself is described in mg_kv4.h).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "mg_attn.h"

namespace mg {

constexpr int kKv4Block = 32;   // tokens are padded to a multiple of this

inline int kv4_groups(int d) { return d <= 64 ? 1 : d / 64; }
inline int kv4_padded(int L) { return (L + kKv4Block - 1) / kKv4Block * kKv4Block; }

// Byte offsets of the regions after K's words, and the cache's size.
struct Kv4Regions {
    size_t v, kp, vp, bytes;
};
inline Kv4Regions kv4_regions(int B, int H, int L, int d) {
    const size_t rows = (size_t)B * H * kv4_padded(L);
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t words = up(rows * (d / 2)), params = up(rows * kv4_groups(d) * 4);
    return {words, 2 * words, 2 * words + params, 2 * words + 2 * params};
}

// A cache's regions as pointers; C is uint32_t or const uint32_t.
template <typename C>
struct Kv4Cache {
    C *k, *v, *kp, *vp;
};
template <typename C, typename P>
inline Kv4Cache<C> kv4_cache(P *base, int B, int H, int L, int d) {
    const Kv4Regions r = kv4_regions(B, H, L, d);
    auto *c = reinterpret_cast<C *>(base);
    return {c, c + r.v / 4, c + r.kp / 4, c + r.vp / 4};
}

}  // namespace mg
