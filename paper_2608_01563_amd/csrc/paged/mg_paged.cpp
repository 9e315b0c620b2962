// mg_paged.cpp -- C ABI of the paged key/value cache: argument validation,
// workspace sizing and launches on the caller's stream.  Validation runs on the
// host before anything is enqueued.
#include "mg_paged.h"

#include <algorithm>
#include <cmath>
#include <tuple>

#include "cdiv.h"
#include "host_runtime.h"
#include "paged_launch.h"

namespace mg {

namespace {
// (Measured at d = 128, where a compute unit runs three workgroups of 16 rows or two of 32.
// Smaller heads fit more, d = 32 bf16 six and five, d = 64 four and three, and are cut
// alike: 4.8 to 4.9 TB/s over 8 long caches, 5.3 with d = 128.)
constexpr int kWant = 1536;       // workgroups of 16 rows that a call is cut into: six a
                                  // compute unit
constexpr int kWantMore = 1024;   // of more rows: four
constexpr int kRound = 512;       // of a short call
constexpr int kLeast = 4;         // blocks of a unit: one a wave (2 sequences of 1,020 tokens, 8
                                  // heads: 10.6 us with 4, 12.1 with 8, 13.6 with 32, f32 11.5,
                                  // 15.0, 30.8)
// Bytes that caches may hold from call to call; by the room in tables, not the lengths.
// (4 to 130 MB held in roomy tables: 0 to 5 % slower past the caches.  Shared pages: 16
// sequences over the same 8,192 tokens 57 us, 47 through the caches.)
constexpr int64_t kCached = 64 << 20;
constexpr int kLongest = 1 << 13; // blocks of a unit (2^18 tokens)

void paged_workspace(PagedPlan &plan, const PagedAttn &p, int64_t rows) {
    plan.join_waves = plan.most <= 16 ? 1 : 4;   // (by the room in tables, not the lengths)
    if (plan.most <= 1) return;
    const size_t slots = (size_t)plan.units * p.H * rows;
    plan.part = plan.bytes;
    plan.bytes += host::round256(slots * p.d * 4);
    plan.stat = plan.bytes;
    plan.bytes += host::round256(slots * 8);
}
}  // namespace

PagedPlan paged_plan(const PagedAttn &p, bool sparse) {
    PagedPlan plan = {};
    const int64_t rows = paged_rows(p, sparse);
    plan.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    plan.groups = (int)((rows + plan.rows - 1) / plan.rows);
    const int64_t groups = (int64_t)p.H * plan.groups;   // workgroups of a unit
    const int64_t cut = std::max<int64_t>(1, (plan.rows == 16 ? kWant : kWantMore) / groups);
    const int64_t round = std::max<int64_t>(1, kRound / groups);
    const int64_t pages = std::min<int64_t>(
        p.N, (int64_t)p.B * (sparse ? (int64_t)p.Lq * p.keep : p.P));
    plan.once = (pages << p.shift) * p.H * p.d * (p.half ? 4 : 8) > kCached;
    // what is no more than two (f32) or four blocks a wave is one unit, which needs no
    // joining (500 tokens: 8.8 us instead of 10.7; f32 16.4 instead of 10.8)
    const int64_t held = (int64_t)(sparse ? p.keep : p.P) << p.shift;
    const int tokens = p.half ? 512 : p.d == 128 ? 128 : 256;
    const int blocks = (int)((held + 31) / 32);
    const int least = held <= tokens ? tokens / 32 : kLeast;
    if (sparse) {
        // lists are short of their `keep` pages only where sequences are: units are all
        // alike, and one round of them will do.
        // A unit has at most 64 pages, whose entries a wave holds.
        const int64_t seqs = (int64_t)p.B * p.Lq;
        const int64_t want = std::max<int64_t>(
            1, std::min<int64_t>(round / seqs, cdiv(blocks, least)));
        plan.chunk = (cdiv(blocks, (int)want) + 3) / 4 * 4;
        plan.chunk = std::min(plan.chunk, 2 << p.shift);
        plan.splits = cdiv(blocks, plan.chunk);
        plan.units = (int)std::min<int64_t>(seqs * plan.splits, INT32_MAX);
        plan.most = plan.splits;
        paged_workspace(plan, p, rows);
        return plan;
    }
    const int full = cdiv(blocks, least), longest = cdiv(blocks, kLongest);
    plan.chunk = least;
    plan.most = std::max(std::min(full, (int)cut), longest);   // a cut sequence's units
    if (plan.most == 1) {
        plan.splits = 1;
        plan.chunk = std::max(blocks, least);
        plan.units = p.B;
    } else if ((int64_t)p.B * full <= round) {
        plan.splits = plan.most = full;
        plan.units = p.B * full;
    } else {
        plan.share = (int)cut;
        plan.round = (int)round;
        plan.round_most = (int)(plan.rows == 16 ? round + round / 2 : round);
        plan.units = (int)std::max<int64_t>(cut + p.B, (int64_t)p.B * longest);
        plan.lengths = p.B > kPagedScanned;
    }
    if (plan.most > 1) {
        plan.info = plan.bytes;
        plan.bytes += host::round256((size_t)p.B * 8);
    }
    if (plan.lengths) {
        plan.map = plan.bytes;
        plan.bytes += host::round256((size_t)plan.units * 4);
    }
    paged_workspace(plan, p, rows);
    return plan;
}

}  // namespace mg

namespace {

using mg::host::fail;
using mg::host::ok;
using mg::host::run_kernel;

// Grids stay below 2^32 threads.
constexpr int kMaxTokens = 1 << 24, kMaxSequences = 1 << 16, kMaxHeads = 1 << 19;
constexpr int kMaxRows = 1 << 28;
constexpr int64_t kMaxGroups = (1LL << 24) - 1;   // of 256 threads
constexpr float kLog2e = 1.4426950408889634f;     // as the kernels take it

mg_status_t check_contract(mg_contract_t c) {
    if (c != MG_CONTRACT_STRICT_F32 && c != MG_CONTRACT_FAST_BF16 && c != MG_CONTRACT_ACCELERATED)
        return fail(MG_ERR_INVALID_ARGUMENT, "unknown contract %d", (int)c);
    return MG_OK;
}

int shift_of(int page) {
    for (int s = 4; s <= 8; ++s)
        if (page == 1 << s) return s;
    return -1;
}

mg_status_t check_page(int page) {
    if (shift_of(page) < 0)
        return fail(MG_ERR_UNSUPPORTED, "pages of %d tokens: not 16, 32, 64, 128 or 256", page);
    return MG_OK;
}

mg_status_t check_tables(int B, int page, int P) {
    if (B < 1 || P < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (B=%d P=%d)", B, P);
    MG_TRY(check_page(page));
    if (B > kMaxSequences || (int64_t)P * page > kMaxTokens ||
        (int64_t)B * P * page > 1LL << 35 || (int64_t)B * P > INT32_MAX)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "the tables are too large (B=%d P=%d page=%d): B at most 2^16, P*page at most "
                    "2^24, B*P*page at most 2^35, B*P below 2^31", B, P, page);
    return MG_OK;
}

mg_status_t check_pool(int N, int H, int page, int d) {
    if (N < 1 || H < 1 || d < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (N=%d H=%d d=%d)", N, H, d);
    MG_TRY(check_page(page));
    if ((int64_t)N * page > INT32_MAX || (int64_t)H * page * d >= 1 << 28)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "the pools are too large (N=%d H=%d page=%d d=%d): N*page below 2^31, H*page*d "
                    "below 2^28", N, H, page, d);
    if (d != 32 && d != 64 && d != 128)
        return fail(MG_ERR_UNSUPPORTED, "head dimension %d is not 32, 64 or 128", d);
    return MG_OK;
}

mg_status_t check_rows(int B, int Hq, int H, int Lq, int d) {
    if (Hq < 1 || Lq < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (Hq=%d Lq=%d)", Hq, Lq);
    if (Hq % H != 0)
        return fail(MG_ERR_INVALID_ARGUMENT, "%d query heads over %d cache heads", Hq, H);
    if ((int64_t)B * Hq > INT32_MAX || (int64_t)B * Hq * Lq > INT32_MAX ||
        (int64_t)B * Hq * Lq * d > INT32_MAX || (int64_t)B * H * Lq > kMaxHeads)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "too many query rows (B=%d Hq=%d H=%d Lq=%d d=%d): B*Hq*Lq*d below 2^31, B*H*Lq "
                    "at most 2^19", B, Hq, H, Lq, d);
    return MG_OK;
}

// Required pointers of 16- and of 4-byte alignment and optional ones: what needs no
// look at the device comes first.
using Ptrs = std::initializer_list<mg::host::NamedPtr>;
mg_status_t check_ptrs(Ptrs wide, Ptrs narrow, Ptrs optional, int optional_align) {
    for (const auto &[list, align, needed] :
         {std::tuple<Ptrs, int, bool>{wide, 16, true}, {narrow, 4, true},
          {optional, optional_align, false}})
        for (const mg::host::NamedPtr &p : list) {
            if (p.ptr == nullptr && needed)
                return fail(MG_ERR_INVALID_ARGUMENT, "%s is NULL", p.name);
            if (reinterpret_cast<uintptr_t>(p.ptr) % align != 0)
                return fail(MG_ERR_MISALIGNED, "%s is not %d-byte aligned", p.name, align);
        }
    MG_TRY(mg::host::check_device_ptrs(wide, 16));
    MG_TRY(mg::host::check_device_ptrs(narrow, 4));
    for (const mg::host::NamedPtr &p : optional)
        MG_TRY(mg::host::check_optional_device_ptr(p.ptr, p.name, optional_align));
    return MG_OK;
}

mg_status_t check_attn(const mg::PagedAttn &p, int Hq, int page, bool sparse,
                       mg_contract_t contract, mg::PagedPlan *plan) {
    MG_TRY(check_contract(contract));
    MG_TRY(check_pool(p.N, p.H, page, p.d));
    MG_TRY(check_tables(p.B, page, p.P));
    MG_TRY(check_rows(p.B, Hq, p.H, p.Lq, p.d));
    if (sparse && (p.keep < 1 || (int64_t)p.keep * page > kMaxTokens))
        return fail(MG_ERR_INVALID_ARGUMENT, "keep must be >= 1 and keep*page at most 2^24 (got %d)",
                    p.keep);
    if (!std::isfinite(p.scale * kLog2e))
        return fail(MG_ERR_INVALID_ARGUMENT, "scale log2 e is not finite (scale %g)", p.scale);
    *plan = mg::paged_plan(p, sparse);
    const int64_t joins = (int64_t)p.B * Hq * p.Lq * plan->join_waves / 4;
    if ((int64_t)plan->units * p.H * plan->groups > kMaxGroups ||
        (plan->most > 1 && joins >= kMaxGroups))
        return fail(MG_ERR_INVALID_ARGUMENT, "too much work for one call (B=%d H=%d Lq=%d P=%d)",
                    p.B, p.H, p.Lq, p.P);
    return MG_OK;
}

mg::PagedAttn attn_of(int B, int Hq, int H, int Lq, int d, int page, int P, int N, int causal,
                      int keep, float scale, const int32_t *table, const int32_t *index,
                      const int32_t *key_len, const int32_t *q_len, mg_contract_t contract) {
    return {B, H, H > 0 ? Hq / H : 0, Lq, d, shift_of(page), P, N, causal != 0, keep,
            contract == MG_CONTRACT_FAST_BF16, scale, table, index, key_len, q_len};
}

mg_status_t attn_call(const mg::PagedAttn &p, int Hq, int page, bool sparse, const void *Q,
                      const void *Kp, const void *Vp, void *O, float *LSE, mg_contract_t contract,
                      void *workspace, size_t workspace_bytes, hipStream_t stream) {
    mg::PagedPlan plan;
    MG_TRY(check_attn(p, Hq, page, sparse, contract, &plan));
    if (plan.bytes > 0 && (workspace == nullptr || workspace_bytes < plan.bytes))
        return fail(MG_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed",
                    workspace ? workspace_bytes : (size_t)0, plan.bytes);
    const void *ws = plan.bytes > 0 ? workspace : nullptr;
    if (reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return fail(MG_ERR_MISALIGNED, "workspace is not 16-byte aligned");
    if (sparse && p.index == nullptr) return fail(MG_ERR_INVALID_ARGUMENT, "index is NULL");
    MG_TRY(check_ptrs({{Q, "Q"}, {Kp, "Kp"}, {Vp, "Vp"}, {O, "O"}, {LSE, "LSE"}},
                      {{p.table, "table"}, {p.key_len, "key_len"}},
                      {{p.q_len, "q_len"}, {sparse ? p.index : nullptr, "index"},
                       {ws, "workspace"}}, 4));
    if (plan.lengths)
        MG_TRY(run_kernel("paged_cut", stream, [&] {
            return mg::launch_paged_cut(p, plan, workspace, stream);
        }));
    MG_TRY(run_kernel("paged_attn", stream, [&] {
        return mg::launch_paged_attn(p, plan, Q, Kp, Vp, O, LSE, workspace, stream);
    }));
    if (plan.most > 1)
        MG_TRY(run_kernel("paged_join", stream, [&] {
            return mg::launch_paged_join(p, plan, O, LSE, workspace, stream);
        }));
    return ok();
}

mg_status_t check_resize(int B, int page, int P, int N, int T) {
    MG_TRY(check_tables(B, page, P));
    if (N < 1 || T < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (N=%d T=%d)", N, T);
    if ((int64_t)N * page > INT32_MAX || T > kMaxRows)
        return fail(MG_ERR_INVALID_ARGUMENT, "N*page must be below 2^31, T at most 2^28 (N=%d T=%d)",
                    N, T);
    return MG_OK;
}

mg_status_t check_select(const mg::PagedSelect &p, int Hq, int page, mg_contract_t contract) {
    MG_TRY(check_contract(contract));
    MG_TRY(check_pool(p.N, p.H, page, p.d));
    MG_TRY(check_tables(p.B, page, p.P));
    MG_TRY(check_rows(p.B, Hq, p.H, p.Lq, p.d));
    if (p.keep < 1 || p.first < 0 || p.recent < 0 || (int64_t)p.first + p.recent > p.keep)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "keep must be >= 1, first and recent >= 0 and together at most keep (keep=%d "
                    "first=%d recent=%d)", p.keep, p.first, p.recent);
    if ((int64_t)p.B * p.H * p.Lq * std::max(p.P, p.keep) > 1 << 29)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "too many scores (B=%d H=%d Lq=%d P=%d keep=%d): B*H*Lq*P and B*H*Lq*keep at "
                    "most 2^29", p.B, p.H, p.Lq, p.P, p.keep);
    return MG_OK;
}

size_t scores_bytes(const mg::PagedSelect &p) {
    return mg::host::round256((size_t)p.B * p.H * p.Lq * p.P * 4);
}

// The size a query asks for: 0 where `check` refuses, with the last detail kept.
template <typename F>
size_t asked(F &&check) {
    const std::string saved = mg::host::saved_detail();
    const size_t bytes = check();
    mg::host::restore_detail(saved);
    return bytes;
}

}  // namespace

extern "C" {

size_t mg_paged_resize_workspace_bytes(int B, int T) {
    if (B < 1 || B > kMaxSequences || T < 1 || T > kMaxRows) return 0;
    return mg::host::round256(mg::paged_resize_bytes(B, T));
}

mg_status_t mg_paged_resize(const int32_t *key_len, const int32_t *want, int32_t *table,
                            int32_t *free_pages, const int32_t *free_count, int32_t *new_len,
                            int32_t *new_count, int32_t *slot, int32_t *offset, int B, int page,
                            int P, int N, int T, void *workspace, size_t workspace_bytes,
                            hipStream_t stream) {
    MG_TRY(check_resize(B, page, P, N, T));
    const size_t need = mg_paged_resize_workspace_bytes(B, T);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need))
        return fail(MG_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed",
                    workspace ? workspace_bytes : (size_t)0, need);
    MG_TRY(check_ptrs({}, {{key_len, "key_len"}, {want, "want"}, {table, "table"},
                           {free_pages, "free_pages"}, {free_count, "free_count"},
                           {new_len, "new_len"}, {new_count, "new_count"}, {slot, "slot"},
                           {offset, "offset"}},
                      {{need > 0 ? workspace : nullptr, "workspace"}}, 16));
    const mg::PagedResize p = {B, shift_of(page), P, N, T, key_len, want, table, free_pages,
                               free_count, new_len, new_count, slot, offset};
    MG_TRY(run_kernel("paged_resize", stream, [&] {
        return mg::launch_paged_resize(p, workspace, stream);
    }));
    if (!mg::paged_resize_alone(B, T))
        MG_TRY(run_kernel("paged_slots", stream, [&] {
            return mg::launch_paged_slots(p, workspace, stream);
        }));
    return ok();
}

mg_status_t mg_paged_append(const void *K, const void *V, void *Kp, void *Vp, void *bounds,
                            const int32_t *slot, int T, int H, int d, int page, int N,
                            mg_contract_t contract, hipStream_t stream) {
    MG_TRY(check_contract(contract));
    MG_TRY(check_pool(N, H, page, d));
    if (T < 1) return fail(MG_ERR_INVALID_ARGUMENT, "T must be >= 1 (got %d)", T);
    if ((int64_t)T * H > kMaxRows)
        return fail(MG_ERR_INVALID_ARGUMENT, "too many rows (T=%d H=%d): T*H at most 2^28", T, H);
    MG_TRY(check_ptrs({{K, "K"}, {V, "V"}, {Kp, "Kp"}, {Vp, "Vp"}}, {{slot, "slot"}},
                      {{bounds, "bounds"}}, 16));
    const mg::PagedAppend p = {T, H, d, shift_of(page), N, slot};
    MG_TRY(run_kernel("paged_append", stream, [&] {
        return mg::launch_paged_append(p, K, V, Kp, Vp, bounds, contract == MG_CONTRACT_FAST_BF16,
                                       stream);
    }));
    return ok();
}

size_t mg_attn_fwd_paged_workspace_bytes(int B, int Hq, int H, int Lq, int d, int page, int P,
                                         mg_contract_t contract) {
    return asked([&]() -> size_t {
        mg::PagedPlan plan;
        const mg::PagedAttn p = attn_of(B, Hq, H, Lq, d, page, P, 1, 1, 0, 1.f, nullptr, nullptr,
                                        nullptr, nullptr, contract);
        return check_attn(p, Hq, page, false, contract, &plan) == MG_OK ? plan.bytes : 0;
    });
}

mg_status_t mg_attn_fwd_paged(const void *Q, const void *Kp, const void *Vp, void *O, float *LSE,
                              const int32_t *table, const int32_t *key_len, const int32_t *q_len,
                              int B, int Hq, int H, int Lq, int d, int page, int P, int N,
                              int causal, float scale, mg_contract_t contract, void *workspace,
                              size_t workspace_bytes, hipStream_t stream) {
    const mg::PagedAttn p = attn_of(B, Hq, H, Lq, d, page, P, N, causal, 0, scale, table, nullptr,
                                    key_len, q_len, contract);
    return attn_call(p, Hq, page, false, Q, Kp, Vp, O, LSE, contract, workspace, workspace_bytes,
                     stream);
}

size_t mg_attn_fwd_paged_sparse_workspace_bytes(int B, int Hq, int H, int Lq, int d, int page,
                                                int keep, mg_contract_t contract) {
    return asked([&]() -> size_t {
        mg::PagedPlan plan;
        const mg::PagedAttn p = attn_of(B, Hq, H, Lq, d, page, 1, 1, 1, keep, 1.f, nullptr, nullptr,
                                        nullptr, nullptr, contract);
        return check_attn(p, Hq, page, true, contract, &plan) == MG_OK ? plan.bytes : 0;
    });
}

mg_status_t mg_attn_fwd_paged_sparse(const void *Q, const void *Kp, const void *Vp, void *O,
                                     float *LSE, const int32_t *table, const int32_t *index,
                                     const int32_t *key_len, const int32_t *q_len, int B, int Hq,
                                     int H, int Lq, int d, int page, int P, int N, int causal,
                                     int keep, float scale, mg_contract_t contract,
                                     void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const mg::PagedAttn p = attn_of(B, Hq, H, Lq, d, page, P, N, causal, keep, scale, table, index,
                                    key_len, q_len, contract);
    return attn_call(p, Hq, page, true, Q, Kp, Vp, O, LSE, contract, workspace, workspace_bytes,
                     stream);
}

size_t mg_paged_select_workspace_bytes(int B, int Hq, int H, int Lq, int d, int page, int P,
                                       mg_contract_t contract) {
    return asked([&]() -> size_t {
        const mg::PagedSelect p = {B, H, H > 0 ? Hq / H : 0, Lq, d, shift_of(page), P, 1, 1, 1, 0,
                                   0, nullptr, nullptr, nullptr};
        return check_select(p, Hq, page, contract) == MG_OK ? scores_bytes(p) : 0;
    });
}

mg_status_t mg_paged_select(const void *Q, const void *bounds, const int32_t *table,
                            const int32_t *key_len, const int32_t *q_len, int32_t *index, int B,
                            int Hq, int H, int Lq, int d, int page, int P, int N, int causal,
                            int keep, int first, int recent, mg_contract_t contract,
                            void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const mg::PagedSelect p = {B, H, H > 0 ? Hq / H : 0, Lq, d, shift_of(page), P, N, causal != 0,
                               keep, first, recent, table, key_len, q_len};
    MG_TRY(check_select(p, Hq, page, contract));
    const size_t need = scores_bytes(p);
    if (workspace == nullptr || workspace_bytes < need)
        return fail(MG_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed",
                    workspace ? workspace_bytes : (size_t)0, need);
    MG_TRY(check_ptrs({{Q, "Q"}, {bounds, "bounds"}, {workspace, "workspace"}},
                      {{table, "table"}, {key_len, "key_len"}, {index, "index"}},
                      {{q_len, "q_len"}}, 4));
    float *score = static_cast<float *>(workspace);
    MG_TRY(run_kernel("paged_scores", stream, [&] {
        return mg::launch_paged_scores(p, Q, bounds, contract == MG_CONTRACT_FAST_BF16, score,
                                       stream);
    }));
    MG_TRY(run_kernel("paged_select", stream, [&] {
        return mg::launch_paged_select(p, score, index, stream);
    }));
    return ok();
}

}  // extern "C"
