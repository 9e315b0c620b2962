// mg_kv4.cpp -- C ABI of the 4-bit key/value cache: argument validation,
// workspace sizing and launches on the caller's stream.  Validation runs on
// the host before anything is enqueued.
#include "mg_kv4.h"

#include <algorithm>
#include <cmath>

#include "cdiv.h"
#include "host_runtime.h"
#include "kv4_launch.h"

namespace mg {

// How a call runs.  kv4_many reads a tile of tokens once for 256 rows, kv4_rows
// for 16, with a simpler start and end.  At 256 heads of 8,192 tokens, kv4_many /
// kv4_rows in us: d = 128: 211/92 with 32 rows a head, 246/266 with 96, 251/361
// with 128, 656/1034 with 512; d = 64: 200/181 with 128, 227/329 with 256.  It
// needs the work too: 43/47 at 8 heads x 512 rows x 8,192 tokens (2^25) and 41/53
// at 256 x 128 x 1,024 (the same), but 35/28 with 8 x 256 x 8,192, where its split
// form hardly fills the GPU.  One bound for every d costs a tenth at most beside it
// (96 rows of d = 128, 128 rows of d = 64).  (128-row workgroups were slower at d =
// 128: their unpacked tiles fill the LDS all the same.)  Tokens are split over
// workgroups where there are fewer than the GPU holds at once: one of kv4_many or two
// of kv4_rows a compute unit (with 1,280 workgroups drafts took 22.9 instead of 19.9
// us, a long batch 51 either way: each workgroup prepares its query rows and joins its
// waves).  A split has at least 256 tokens.  It has at most 2^18, also where the GPU
// is full: f32 sums of more drift where terms are alike (65,536 rows over 2^24 tokens of
// equal score in one split: O off by 2.8 %, LSE by 0.02; so 3e-4), unless the
// workspace would pass 8 GiB, which is seconds of work.
Kv4Plan kv4_plan(const Kv4Attn &p, bool weights, bool bf16) {
    const int64_t heads = (int64_t)p.B * p.H, rows = kv4_rows(p);
    Kv4Plan plan = {};
    const bool many = bf16 && rows >= 128 && heads * rows * p.L >= (1 << 25);
    plan.rows = many ? 256 : 16;
    const int64_t tiles = heads * ((rows + plan.rows - 1) / plan.rows);
    const int64_t want = many ? 256 : 512;
    const int blocks = kv4_padded(p.L) / 32;
    plan.splits = (int)std::max<int64_t>(
        1, std::min({(want + tiles - 1) / tiles, (int64_t)64, (int64_t)blocks / 8}));
    const int64_t room = (8LL << 30) / (heads * rows * (p.d + 2) * 4);
    plan.splits = (int)std::max<int64_t>(plan.splits, std::min<int64_t>(cdiv(blocks, 1 << 13), room));
    plan.chunk = cdiv(blocks, plan.splits);
    plan.scores = weights && rows <= 16;
    if (plan.splits > 1) {
        plan.part = plan.bytes;
        plan.bytes += host::round256((size_t)(heads * plan.splits * rows * p.d) * 4);
        plan.stat = plan.bytes;
        plan.bytes += host::round256((size_t)(heads * plan.splits * rows) * 8);
    }
    if (plan.scores) {
        plan.score = plan.bytes;
        plan.bytes += host::round256((size_t)(heads * rows) * kv4_padded(p.L) * 4);
    }
    if (weights && !plan.scores) {
        // four workgroups of 256 tokens a compute unit, which even out how much
        // causal rows see of them, each with 15 blocks of 32 rows or more (4 x 4
        // heads, 4,000 rows, 1,000 tokens of 64: 27 us with 8 shares, 34 with 16;
        // 16 heads, 16,384 rows, 4,096 tokens of 128: 419 with 2, 286 with 4 or 8)
        const int64_t groups = heads * cdiv(p.L, 256);
        plan.shares = (int)std::min<int64_t>((1024 + groups - 1) / groups,
                                             std::max<int64_t>(1, rows / 480));
        if (plan.shares > 1) {
            plan.sums = plan.bytes;
            plan.bytes += host::round256((size_t)plan.shares * heads * kv4_padded(p.L) * 4);
        }
    }
    return plan;
}

}  // namespace mg

namespace {

using mg::host::fail;
using mg::host::ok;
using mg::host::run_kernel;

// These keep every grid below 2^32 threads (six workgroups of 1,024 a head where
// sequences are cut, 64 threads an octet of tokens written, two threads a token
// where weights are gathered) and a head's regions below 4 GiB.
constexpr int kMaxTokens = 1 << 24, kMaxHeads = 1 << 19;
constexpr int64_t kMaxCache = 1 << 30, kMaxMoved = 1 << 28;
constexpr float kLog2e = 1.4426950408889634f;   // as the kernels take it

mg_status_t check_contract(mg_contract_t c) {
    if (c != MG_CONTRACT_STRICT_F32 && c != MG_CONTRACT_FAST_BF16 && c != MG_CONTRACT_ACCELERATED)
        return fail(MG_ERR_INVALID_ARGUMENT, "unknown contract %d", (int)c);
    return MG_OK;
}

// Sizes every entry point shares.
mg_status_t check_cache(int B, int H, int L, int d) {
    if (B < 1 || H < 1 || L < 1 || d < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (B=%d H=%d L=%d d=%d)", B, H, L,
                    d);
    if ((int64_t)B * H > kMaxHeads || L > kMaxTokens ||
        (int64_t)B * H * mg::kv4_padded(L) > kMaxCache)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "the cache is too large (B=%d H=%d L=%d): B*H at most 2^19, L at most 2^24, "
                    "B*H*L (L rounded up to 32) at most 2^30", B, H, L);
    if (d != 32 && d != 64 && d != 128)
        return fail(MG_ERR_UNSUPPORTED, "head dimension %d is not 32, 64 or 128", d);
    return MG_OK;
}

mg_status_t check_move(int B, int H, int n, int L, int d, mg_contract_t contract) {
    MG_TRY(check_contract(contract));
    MG_TRY(check_cache(B, H, L, d));
    if (n < 1) return fail(MG_ERR_INVALID_ARGUMENT, "n must be >= 1 (got %d)", n);
    if (n > kMaxTokens || (int64_t)B * H * n > kMaxMoved)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "too many rows (B=%d H=%d n=%d): n at most 2^24, B*H*n at most 2^28", B, H, n);
    return MG_OK;
}

mg_status_t check_arrays(std::initializer_list<mg::host::NamedPtr> ptrs) {
    for (const mg::host::NamedPtr &p : ptrs)
        MG_TRY(mg::host::check_optional_device_ptr(p.ptr, p.name, 4));
    return MG_OK;
}

mg_status_t check_attn(int B, int Hq, int H, int Lq, int L, int d, float scale,
                       mg_contract_t contract) {
    MG_TRY(check_contract(contract));
    MG_TRY(check_cache(B, H, L, d));
    if (Hq < 1 || Lq < 1)
        return fail(MG_ERR_INVALID_ARGUMENT, "sizes must be >= 1 (Hq=%d Lq=%d)", Hq, Lq);
    if (Hq % H != 0)
        return fail(MG_ERR_INVALID_ARGUMENT, "%d query heads over %d cache heads", Hq, H);
    if ((int64_t)B * Hq > INT32_MAX || (int64_t)B * Hq * Lq > INT32_MAX ||
        (int64_t)B * Hq * Lq * d > INT32_MAX)
        return fail(MG_ERR_INVALID_ARGUMENT, "B*Hq*Lq*d exceeds 2^31-1 (B=%d Hq=%d Lq=%d d=%d)",
                    B, Hq, Lq, d);
    if (!std::isfinite(scale * kLog2e))
        return fail(MG_ERR_INVALID_ARGUMENT, "scale log2 e is not finite (scale %g)", scale);
    return MG_OK;
}

}  // namespace

extern "C" {

size_t mg_kv4_cache_bytes(int B, int H, int L, int d) {
    const std::string saved = mg::host::saved_detail();
    const bool good = check_cache(B, H, L, d) == MG_OK;
    mg::host::restore_detail(saved);
    return good ? mg::kv4_regions(B, H, L, d).bytes : 0;
}

mg_status_t mg_kv4_append(const void *K, const void *V, void *cache, float *weight,
                          const int32_t *start, const int32_t *count, int B, int H, int n, int L,
                          int d, mg_contract_t contract, hipStream_t stream) {
    MG_TRY(check_move(B, H, n, L, d, contract));
    MG_TRY(mg::host::check_device_ptrs({{K, "K"}, {V, "V"}, {cache, "cache"}}, 16));
    MG_TRY(check_arrays({{weight, "weight"}, {start, "start"}, {count, "count"}}));
    const mg::Kv4Move p = {B, H, n, L, d, start, count};
    const bool bf16 = contract == MG_CONTRACT_FAST_BF16;
    MG_TRY(run_kernel("kv4_append", stream, [&] {
        return mg::launch_kv4_append(p, K, V, bf16,
                                     mg::kv4_cache<uint32_t>(cache, B, H, L, d), weight, stream);
    }));
    return ok();
}

mg_status_t mg_kv4_read(const void *cache, void *K, void *V, const int32_t *start,
                        const int32_t *count, int B, int H, int n, int L, int d,
                        mg_contract_t contract, hipStream_t stream) {
    MG_TRY(check_move(B, H, n, L, d, contract));
    MG_TRY(mg::host::check_device_ptrs({{cache, "cache"}, {K, "K"}, {V, "V"}}, 16));
    MG_TRY(check_arrays({{start, "start"}, {count, "count"}}));
    const mg::Kv4Move p = {B, H, n, L, d, start, count};
    const bool bf16 = contract == MG_CONTRACT_FAST_BF16;
    MG_TRY(run_kernel("kv4_read", stream, [&] {
        return mg::launch_kv4_read(p, mg::kv4_cache<const uint32_t>(cache, B, H, L, d), K, V,
                                   bf16, stream);
    }));
    return ok();
}

size_t mg_attn_fwd_kv4_workspace_bytes(int B, int Hq, int H, int Lq, int L, int d, int weights,
                                       mg_contract_t contract) {
    const std::string saved = mg::host::saved_detail();
    const bool good = check_attn(B, Hq, H, Lq, L, d, 1.f, contract) == MG_OK;
    mg::host::restore_detail(saved);
    if (!good) return 0;
    const mg::Kv4Attn p = {B, H, Hq / H, Lq, L, d, 0, 1.f, nullptr, nullptr};
    return mg::kv4_plan(p, weights != 0, contract == MG_CONTRACT_FAST_BF16).bytes;
}

mg_status_t mg_attn_fwd_kv4(const void *Q, const void *cache, void *O, float *LSE, float *weight,
                            const int32_t *key_len, const int32_t *q_len, int B, int Hq, int H,
                            int Lq, int L, int d, int causal, float scale,
                            mg_contract_t contract, void *workspace, size_t workspace_bytes,
                            hipStream_t stream) {
    MG_TRY(check_attn(B, Hq, H, Lq, L, d, scale, contract));
    const bool bf16 = contract == MG_CONTRACT_FAST_BF16;
    const mg::Kv4Attn p = {B, H, Hq / H, Lq, L, d, causal != 0, scale, key_len, q_len};
    const mg::Kv4Plan plan = mg::kv4_plan(p, weight != nullptr, bf16);
    if (plan.bytes > 0 && (workspace == nullptr || workspace_bytes < plan.bytes))
        return fail(MG_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed",
                    workspace ? workspace_bytes : (size_t)0, plan.bytes);
    MG_TRY(mg::host::check_device_ptrs({{Q, "Q"}, {cache, "cache"}, {O, "O"}, {LSE, "LSE"}}, 16));
    if (plan.bytes > 0) MG_TRY(mg::host::check_device_ptrs({{workspace, "workspace"}}, 16));
    MG_TRY(check_arrays({{weight, "weight"}, {key_len, "key_len"}, {q_len, "q_len"}}));
    const auto c = mg::kv4_cache<const uint32_t>(cache, B, H, L, d);
    if (plan.rows > 16)
        MG_TRY(run_kernel("kv4_many", stream, [&] {
            return mg::launch_kv4_many(p, plan, Q, c, O, LSE, workspace, stream);
        }));
    else
        MG_TRY(run_kernel("kv4_rows", stream, [&] {
            return mg::launch_kv4_rows(p, plan, Q, bf16, c, O, LSE, workspace, stream);
        }));
    if (plan.splits > 1 || plan.scores)
        MG_TRY(run_kernel("kv4_join", stream, [&] {
            return mg::launch_kv4_join(p, plan, bf16, O, LSE, weight, workspace, stream);
        }));
    if (plan.shares > 0)
        MG_TRY(run_kernel("kv4_weights", stream, [&] {
            return mg::launch_kv4_weights(p, plan, Q, bf16, c, LSE, weight, workspace, stream);
        }));
    if (plan.shares > 1)
        MG_TRY(run_kernel("kv4_weight_shares", stream, [&] {
            return mg::launch_kv4_weight_shares(p, plan, weight, workspace, stream);
        }));
    return ok();
}

mg_status_t mg_kv4_evict(const void *cache, const float *weight, void *out_cache,
                         float *out_weight, int32_t *index, int32_t *new_len,
                         const int32_t *key_len, int B, int H, int L, int d, int keep, int recent,
                         hipStream_t stream) {
    MG_TRY(check_cache(B, H, L, d));
    if (keep < 1 || keep > L || recent < 0 || recent > keep)
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "keep must be in [1, L] and recent in [0, keep] (L=%d keep=%d recent=%d)", L,
                    keep, recent);
    if ((out_cache == cache) != (out_weight == weight))
        return fail(MG_ERR_INVALID_ARGUMENT,
                    "cache and weight must both be cut in place or both go elsewhere");
    for (const void *p : {cache, (const void *)out_cache})
        if (reinterpret_cast<uintptr_t>(p) % 16 != 0)
            return fail(MG_ERR_MISALIGNED, "a cache is not 16-byte aligned");
    MG_TRY(mg::host::check_device_ptrs({{cache, "cache"}, {out_cache, "out_cache"},
                                        {weight, "weight"}, {out_weight, "out_weight"},
                                        {index, "index"}, {new_len, "new_len"}}, 4));
    MG_TRY(check_arrays({{key_len, "key_len"}}));
    const mg::Kv4Evict p = {B, H, L, d, keep, recent, key_len};
    MG_TRY(run_kernel("kv4_select", stream, [&] {
        return mg::launch_kv4_select(p, weight, index, stream);
    }));
    MG_TRY(run_kernel("kv4_compact", stream, [&] {
        return mg::launch_kv4_compact(p, mg::kv4_cache<const uint32_t>(cache, B, H, L, d), weight,
                                      mg::kv4_cache<uint32_t>(out_cache, B, H, L, d), out_weight,
                                      index, new_len, out_cache == cache, stream);
    }));
    return ok();
}

}  // extern "C"
