// kv4_host_check.cpp -- the 4-bit cache's host code under AddressSanitizer and
// UndefinedBehaviorSanitizer, built by tests/test_kv4_sanitized_cpu.py with
// launchers that must not be reached: every call here is refused on the host or
// only asks for sizes.  Pointers are never dereferenced.
#include <climits>
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "kv4_launch.h"
#include "mg_kv4.h"

namespace {
int g_failures = 0;
void expect(bool ok, const char *what, int line) {
    if (!ok) {
        std::fprintf(stderr, "FAIL line %d: %s (detail: %s)\n", line, what,
                     mg_last_error_detail());
        ++g_failures;
    }
}
#define EXPECT(cond) expect((cond), #cond, __LINE__)
hipError_t reached() {
    EXPECT(!"a launcher was reached");
    return hipErrorUnknown;
}
void *fake(uintptr_t a) { return reinterpret_cast<void *>(a); }
}  // namespace

namespace mg {
hipError_t launch_kv4_append(const Kv4Move &, const void *, const void *, bool,
                             const Kv4Cache<uint32_t> &, float *, hipStream_t) { return reached(); }
hipError_t launch_kv4_read(const Kv4Move &, const Kv4Cache<const uint32_t> &, void *, void *, bool,
                           hipStream_t) { return reached(); }
hipError_t launch_kv4_rows(const Kv4Attn &, const Kv4Plan &, const void *, bool,
                           const Kv4Cache<const uint32_t> &, void *, float *, void *,
                           hipStream_t) { return reached(); }
hipError_t launch_kv4_many(const Kv4Attn &, const Kv4Plan &, const void *,
                           const Kv4Cache<const uint32_t> &, void *, float *, void *,
                           hipStream_t) { return reached(); }
hipError_t launch_kv4_join(const Kv4Attn &, const Kv4Plan &, bool, void *, float *, float *,
                           const void *, hipStream_t) { return reached(); }
hipError_t launch_kv4_weights(const Kv4Attn &, const Kv4Plan &, const void *, bool,
                              const Kv4Cache<const uint32_t> &, const float *, float *, void *,
                              hipStream_t) { return reached(); }
hipError_t launch_kv4_weight_shares(const Kv4Attn &, const Kv4Plan &, float *, const void *,
                                    hipStream_t) { return reached(); }
hipError_t launch_kv4_select(const Kv4Evict &, const float *, int32_t *, hipStream_t) {
    return reached();
}
hipError_t launch_kv4_compact(const Kv4Evict &, const Kv4Cache<const uint32_t> &, const float *,
                              const Kv4Cache<uint32_t> &, float *, const int32_t *, int32_t *,
                              bool, hipStream_t) { return reached(); }
}  // namespace mg

int main() {
    const int big[] = {INT_MIN, -1, 0, 1, 3, 1 << 12, 1 << 19, 1 << 24, (1 << 24) + 1, INT_MAX};
    const mg_contract_t fast = MG_CONTRACT_FAST_BF16;
    void *p = fake(0x1000);
    float *f = static_cast<float *>(p);
    int32_t *n32 = static_cast<int32_t *>(p);
    // sizes of every magnitude: refused, or refused for the pointers, which are nobody's
    for (int B : big)
        for (int H : big)
            for (int L : big) {
                const size_t bytes = mg_kv4_cache_bytes(B, H, L, 64);
                const bool good = B > 0 && H > 0 && L > 0 && (int64_t)B * H <= 1 << 19 &&
                                  L <= 1 << 24 &&
                                  (int64_t)B * H * ((L + 31LL) / 32 * 32) <= 1 << 30;
                EXPECT((bytes > 0) == good);
                for (int n : big) {
                    EXPECT(mg_kv4_append(p, p, p, f, n32, n32, B, H, n, L, 64, fast, nullptr) != MG_OK);
                    EXPECT(mg_kv4_read(p, p, p, n32, n32, B, H, n, L, 64, fast, nullptr) != MG_OK);
                    EXPECT(mg_kv4_evict(p, f, p, f, n32, n32, n32, B, H, L, 64, n, 1, nullptr) != MG_OK);
                    EXPECT(mg_attn_fwd_kv4(p, p, p, f, f, n32, n32, B, n, H, n, L, 64, 1, 1.f, fast,
                                           nullptr, 0, nullptr) != MG_OK);
                    (void)mg_attn_fwd_kv4_workspace_bytes(B, n, H, n, L, 64, 1, fast);
                }
            }
    // the plan: parts inside the workspace, every token and row covered
    for (int heads : {1, 8, 513, 1 << 19})
        for (int G : {1, 4, 128})
            for (int Lq : {1, 5, 127, 2048, 1 << 20})
                for (int L : {1, 33, 1000, 1 << 15, 1 << 24})
                    for (int weights = 0; weights < 2; ++weights)
                        for (int bf16 = 0; bf16 < 2; ++bf16) {
                            if ((int64_t)heads * ((L + 31) / 32 * 32) > 1 << 30 ||
                                (int64_t)heads * G * Lq * 32 > INT_MAX)
                                continue;
                            const mg::Kv4Attn a = {heads, 1, G, Lq, L, 32, 1, 1.f, nullptr, nullptr};
                            const mg::Kv4Plan q = mg::kv4_plan(a, weights != 0, bf16 != 0);
                            const int64_t rows = mg::kv4_rows(a), Lp = mg::kv4_padded(L);
                            EXPECT(q.rows == 16 || (bf16 && q.rows == 256));
                            EXPECT(q.splits >= 1 && (int64_t)q.splits * q.chunk * 32 >= Lp);
                            const int64_t tiles = heads * ((rows + q.rows - 1) / q.rows);
                            EXPECT(tiles * q.splits * 512 < 1LL << 32);
                            size_t at = 0;
                            if (q.splits > 1) {
                                EXPECT(q.part == at && q.stat >= at + heads * q.splits * rows * 32 * 4);
                                at = q.stat + heads * q.splits * rows * 8;
                            }
                            if (q.scores) {
                                EXPECT(weights && rows <= 16 && q.score >= at);
                                at = q.score + heads * rows * Lp * 4;
                            }
                            if (q.shares > 1) {
                                EXPECT(q.sums >= at);
                                at = q.sums + q.shares * heads * Lp * 4;
                            }
                            EXPECT(q.shares == 0 || weights);
                            EXPECT(heads * ((L + 255) / 256) * (int64_t)q.shares * 512 < 1LL << 32);
                            EXPECT(q.bytes >= at);
                        }
    EXPECT(mg_attn_fwd_kv4(p, p, p, f, f, n32, n32, 1, 4, 2, 1, 64, 64, 1, std::nanf(""), fast,
                           nullptr, 0, nullptr) == MG_ERR_INVALID_ARGUMENT);
    if (g_failures == 0) std::printf("kv4 host checks passed\n");
    return g_failures != 0;
}
