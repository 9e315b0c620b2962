// paged_host_check.cpp -- the paged cache's host code under AddressSanitizer and
// UndefinedBehaviorSanitizer, built by tests/test_paged_sanitized_cpu.py with
// launchers that must not be reached: every call here is refused on the host or
// only asks for sizes.  Pointers are never dereferenced.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <initializer_list>

#include "mg_paged.h"
#include "paged_launch.h"

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
bool paged_resize_alone(int B, int T) { return B <= 1024 && T <= 2048; }
size_t paged_resize_bytes(int B, int T) { return paged_resize_alone(B, T) ? 0 : (size_t)20 * B + 12; }
hipError_t launch_paged_resize(const PagedResize &, void *, hipStream_t) { return reached(); }
hipError_t launch_paged_slots(const PagedResize &, const void *, hipStream_t) { return reached(); }
hipError_t launch_paged_append(const PagedAppend &, const void *, const void *, void *, void *, void *,
                               bool, hipStream_t) { return reached(); }
hipError_t launch_paged_cut(const PagedAttn &, const PagedPlan &, void *, hipStream_t) {
    return reached();
}
hipError_t launch_paged_attn(const PagedAttn &, const PagedPlan &, const void *, const void *,
                             const void *, void *, float *, void *, hipStream_t) { return reached(); }
hipError_t launch_paged_join(const PagedAttn &, const PagedPlan &, void *, float *, const void *,
                             hipStream_t) { return reached(); }
hipError_t launch_paged_scores(const PagedSelect &, const void *, const void *, bool, float *,
                               hipStream_t) { return reached(); }
hipError_t launch_paged_select(const PagedSelect &, const float *, int32_t *, hipStream_t) {
    return reached();
}
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
            for (int P : big) {
                (void)mg_paged_resize_workspace_bytes(B, P);
                for (int n : big) {
                    EXPECT(mg_paged_resize(n32, n32, n32, n32, n32, n32, n32, n32, n32, B, 16, P, H, n,
                                           nullptr, 0, nullptr) != MG_OK);
                    EXPECT(mg_paged_append(p, p, p, p, p, n32, B, H, 64, 32, n, fast, nullptr) != MG_OK);
                    EXPECT(mg_attn_fwd_paged(p, p, p, p, f, n32, n32, n32, B, n, H, n, 64, 16, P, 9, 1,
                                             1.f, fast, nullptr, 0, nullptr) != MG_OK);
                    EXPECT(mg_attn_fwd_paged_sparse(p, p, p, p, f, n32, n32, n32, n32, B, H, H, 1, 64,
                                                    256, P, 9, 1, n, 1.f, fast, nullptr, 0,
                                                    nullptr) != MG_OK);
                    EXPECT(mg_paged_select(p, p, n32, n32, n32, n32, B, H, H, 1, 64, 16, P, 9, 1, n, n,
                                           n, fast, nullptr, 0, nullptr) != MG_OK);
                    (void)mg_attn_fwd_paged_workspace_bytes(B, n, H, n, 128, 16, P, fast);
                    (void)mg_attn_fwd_paged_sparse_workspace_bytes(B, n, H, n, 128, 64, P, fast);
                    (void)mg_paged_select_workspace_bytes(B, n, H, n, 32, 256, P, fast);
                }
            }
    // the plan: units for any lengths, parts inside the workspace, short chains
    for (int B : {1, 7, 64, 1000, 1 << 16})
        for (int H : {1, 8, 100})
            for (int G : {1, 4, 40})
                for (int Lq : {1, 7, 2048})
                    for (int shift : {4, 6, 8})
                        for (int P : {1, 33, 1000, 1 << 16})
                            for (int sparse = 0; sparse < 2; ++sparse) {
                                if ((int64_t)P << shift > 1 << 24 || (int64_t)B * H * Lq > 1 << 19 ||
                                    (int64_t)B * H * G * Lq * 32 > INT_MAX ||
                                    (int64_t)B * P << shift > 1LL << 35)
                                    continue;
                                const mg::PagedAttn a = {B, H, G, Lq, 32, shift, P, 9, 1, P, true, 1.f,
                                                         nullptr, nullptr, nullptr, nullptr};
                                const mg::PagedPlan q = mg::paged_plan(a, sparse != 0);
                                const int64_t rows = mg::paged_rows(a, sparse != 0);
                                const int64_t blocks = (((int64_t)P << shift) + 31) / 32;
                                EXPECT(q.rows * (int64_t)q.groups >= rows);
                                EXPECT(q.rows == 16 || q.rows == 32 || q.rows == 64 || q.rows == 128);
                                EXPECT(q.chunk >= 4 && q.chunk <= 1 << 13);
                                const int64_t seqs = (int64_t)B * (sparse ? Lq : 1);
                                if (q.splits > 0) {
                                    EXPECT((int64_t)q.splits * q.chunk >= blocks);
                                    EXPECT(q.most == q.splits && q.units == seqs * q.splits);
                                    EXPECT(!sparse || q.chunk * 32 <= 64 << shift);
                                } else {
                                    // as the kernel cuts them, whatever the lengths
                                    EXPECT(!sparse && q.share >= 1 && q.round >= 1 &&
                                           q.round <= q.round_most && q.round_most <= q.share);
                                    for (int64_t n : {(int64_t)0, (int64_t)1, blocks / 3, blocks}) {
                                        const int64_t total = n * B;
                                        for (int64_t share : {q.share, q.round}) {
                                            int64_t chunk = (total + share - 1) / share;
                                            chunk = std::min<int64_t>(
                                                std::max<int64_t>(chunk, q.chunk), 1 << 13);
                                            const int64_t parts =
                                                std::max<int64_t>((n + chunk - 1) / chunk, 1);
                                            EXPECT(parts * B <= q.units && parts <= q.most);
                                        }
                                    }
                                }
                                size_t at = 0;
                                if (q.most > 1) {
                                    if (!sparse) {
                                        EXPECT(q.info == 0);
                                        at = (size_t)B * 8;
                                    }
                                    EXPECT(q.lengths == (q.splits == 0 && B > mg::kPagedScanned));
                                    EXPECT(q.splits != 0 || q.most > 1);
                                    if (q.lengths) {
                                        EXPECT(q.map >= at);
                                        at = q.map + (size_t)q.units * 4;
                                    }
                                    const size_t slots = (size_t)q.units * H * rows;
                                    EXPECT(q.part >= at && q.stat >= q.part + slots * 32 * 4 &&
                                           q.bytes >= q.stat + slots * 8);
                                }
                                EXPECT(q.most > 1 || (q.bytes == 0 && !q.lengths && q.splits == 1));
                            }
    EXPECT(mg_attn_fwd_paged(p, p, p, p, f, n32, n32, n32, 1, 4, 2, 1, 64, 16, 4, 9, 1, std::nanf(""),
                             fast, nullptr, 0, nullptr) == MG_ERR_INVALID_ARGUMENT);
    if (g_failures == 0) std::printf("paged host checks passed\n");
    return g_failures != 0;
}
