// Pages of the attention cache: checks of arguments, workspace sizes, launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "etf_internal.h"
#include "etf_launch.h"

using namespace etf;

namespace {

#include "etf_pages_kernels.hip.h"

inline int64_t al256(int64_t x) { return (x + 255) & ~(int64_t)255; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
// a launch has fewer than 2^32 threads
inline bool too_many(int64_t groups) { return groups > (int64_t)UINT32_MAX / 256; }

int check_shape(const etf_ctx *ctx, const etf_kv_cache *c)
{
    if (!ctx) return ETF_EINVAL;
    if (!c) return fail(ctx, ETF_EINVAL, "cache is null");
    if (c->dtype != ETF_KV_BF16 && c->dtype != ETF_KV_FP16) return fail(ctx, ETF_EINVAL, "unknown cache type %d", c->dtype);
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128)
        return fail(ctx, ETF_EINVAL, "head_dim must be 64, 96 or 128 (it is %d)", c->head_dim);
    if (c->batch < 1 || c->heads < 1 || c->max_blocks < 1 || c->pages < 1)
        return fail(ctx, ETF_EINVAL, "batch, heads, max_blocks and pages must be positive (%d, %d, %d, %d)", c->batch, c->heads, c->max_blocks, c->pages);
    if (c->max_blocks > (INT32_MAX >> 6) - 2 || (int64_t)c->batch * c->heads > INT32_MAX / c->max_blocks)
        return fail(ctx, ETF_EINVAL, "batch * heads * max_blocks must stay below 2^31, tokens of a sequence too");
    return ETF_OK;
}

int check_cache(const etf_ctx *ctx, const etf_kv_cache *c)
{
    const int rc = check_shape(ctx, c);
    if (rc != ETF_OK) return rc;
    const void *all[] = {c->k, c->v, c->bounds, c->scales, c->tail_k, c->tail_v, c->table, c->lens, c->evicted};
    for (const void *p : all)
        if (!p || !aligned16(p)) return fail(ctx, ETF_EINVAL, "an array of the cache is null or not 16-byte aligned");
    return ETF_OK;
}

int check_ws(const etf_ctx *ctx, const void *ws, int64_t bytes, int64_t need)
{
    if (!ws || ((uintptr_t)ws & 255) != 0) return fail(ctx, ETF_EINVAL, "workspace is null or not 256-byte aligned");
    if (bytes < need) return fail(ctx, ETF_ENOMEM, "workspace too small: %lld < %lld", (long long)bytes, (long long)need);
    return ETF_OK;
}

int enter_device(const etf_ctx *ctx)
{
    if (ctx->device < 0) return fail(ctx, ETF_ENOGPU, "host-only context");
    HIP_TRY(ctx, hipSetDevice(ctx->device));
    return ETF_OK;
}

PageView view_of(const etf_kv_cache *c)
{
    return PageView{(uint8_t *)c->k, (uint8_t *)c->v, (uint8_t *)c->bounds, c->scales, (uint16_t *)c->tail_k, (uint16_t *)c->tail_v,
                    c->table, c->lens, c->evicted, c->batch, c->heads, c->max_blocks, c->pages};
}

// Flags for `many` things; where they lie from `at` on, which is moved behind them
Flags plan_flags(int64_t many, char *ws, int64_t &at)
{
    Flags f{};
    f.many = many;
    f.size = (int32_t)(PAGE_CHUNK * ((many + (int64_t)PAGE_CHUNK * PAGE_CHUNKS - 1) / ((int64_t)PAGE_CHUNK * PAGE_CHUNKS)));
    f.chunks = (int32_t)((many + f.size - 1) / f.size);
    f.words = (uint64_t *)(ws + at);
    at += al256((int64_t)f.chunks * f.size / 8);
    f.counts = (int32_t *)(ws + at);
    at += al256((int64_t)f.chunks * 4);
    return f;
}

// what etf_kv_take lays into its workspace; returns its size
int64_t plan_take(const etf_kv_cache *c, int n, char *ws, TakeArgs &a)
{
    int64_t at = 0;
    a.per = (int)std::min<int64_t>(c->max_blocks, ((int64_t)n + PAGE_KB - 1) / PAGE_KB);
    const int64_t slots = (int64_t)c->batch * c->heads * a.per;
    a.free = plan_flags(c->pages, ws, at);
    a.slots = plan_flags(slots, ws, at);
    a.shared = (int32_t *)(ws + at);
    return at + al256(slots * 4);
}

int64_t plan_fork(const etf_kv_cache *c, char *ws, ForkArgs &a)
{
    const int64_t bh = (int64_t)c->batch * c->heads, open = bh * PAGE_KB * c->head_dim * 2;
    int64_t at = 0;
    a.plan = (int4 *)(ws + at);
    at += al256((int64_t)c->batch * 16);
    a.rows = (int32_t *)(ws + at);
    at += al256(bh * c->max_blocks * 4);
    a.save_k = (uint16_t *)(ws + at);
    at += al256(open);
    a.save_v = (uint16_t *)(ws + at);
    return at + al256(open);
}

int64_t plan_compact(const etf_kv_cache *c, char *ws, CompactArgs &a)
{
    int64_t at = 0;
    a.taken = plan_flags(c->pages, ws, at);
    return at;
}

}  // namespace

extern "C" int64_t etf_kv_take_workspace_bytes(const etf_ctx *ctx, const etf_kv_cache *cache, int n)
{
    const int rc = check_shape(ctx, cache);
    if (rc != ETF_OK) return rc;
    if (n < 1 || n > (1 << 24)) return fail(ctx, ETF_EINVAL, "need 1 <= n <= 2^24 (n=%d)", n);
    TakeArgs a{};
    return plan_take(cache, n, nullptr, a);
}

extern "C" int etf_kv_take(etf_ctx *ctx, const etf_kv_cache *cache, const int32_t *refs, int n, const int32_t *counts, int32_t *table_out, int32_t *refs_out,
                           int32_t *missing, void *ws, int64_t ws_bytes)
{
    int rc = check_cache(ctx, cache);
    if (rc != ETF_OK) return rc;
    if (n < 1 || n > (1 << 24)) return fail(ctx, ETF_EINVAL, "need 1 <= n <= 2^24 (n=%d)", n);
    if (!refs || !table_out || !refs_out || !missing) return fail(ctx, ETF_EINVAL, "null pointer");
    TakeArgs a{};
    if ((rc = check_ws(ctx, ws, ws_bytes, plan_take(cache, n, (char *)ws, a))) != ETF_OK) return rc;
    a.c = view_of(cache);
    a.refs = refs;
    a.counts = counts;
    a.table_out = table_out;
    a.refs_out = refs_out;
    a.missing = missing;
    a.n = n;
    const int64_t grid = (a.slots.many + 255) / 256;
    const int64_t copied = std::max<int64_t>(refs_out != refs ? cache->pages : 0, table_out != cache->table ? (int64_t)cache->batch * cache->heads * cache->max_blocks : 0);
    const int64_t copies = std::min<int64_t>(512, (copied + 1023) / 1024);
    if (too_many(grid)) return fail(ctx, ETF_EINVAL, "too many blocks for one call");
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    hipStream_t st = (hipStream_t)ctx->stream;
    hipLaunchKernelGGL(k_kv_take_flags, dim3((unsigned)(a.free.chunks + a.slots.chunks + copies)), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_take_flags");
    hipLaunchKernelGGL(k_kv_take, dim3((unsigned)grid), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_take");
    return ETF_OK;
}

extern "C" int etf_kv_free(etf_ctx *ctx, int32_t *refs, int pages, const int32_t *list, int64_t n)
{
    if (!ctx) return ETF_EINVAL;
    if (pages < 1 || n < 0) return fail(ctx, ETF_EINVAL, "pages must be positive, n not negative (%d, %lld)", pages, (long long)n);
    if (!refs || (n > 0 && !list)) return fail(ctx, ETF_EINVAL, "null pointer");
    const int64_t grid = (n + 1023) / 1024;
    if (too_many(grid)) return fail(ctx, ETF_EINVAL, "too many pages for one call");
    const int rc = enter_device(ctx);
    if (rc != ETF_OK || n == 0) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    hipLaunchKernelGGL(k_kv_free, dim3((unsigned)grid), dim3(256), 0, (hipStream_t)ctx->stream, refs, pages, list, n);
    LAUNCH_CHECK(ctx, "k_kv_free");
    return ETF_OK;
}

extern "C" int64_t etf_kv_fork_workspace_bytes(const etf_ctx *ctx, const etf_kv_cache *cache)
{
    const int rc = check_shape(ctx, cache);
    if (rc != ETF_OK) return rc;
    ForkArgs a{};
    return plan_fork(cache, nullptr, a);
}

extern "C" int etf_kv_fork(etf_ctx *ctx, const etf_kv_cache *cache, int32_t *refs, const int32_t *source, const int32_t *keep, void *ws, int64_t ws_bytes)
{
    int rc = check_cache(ctx, cache);
    if (rc != ETF_OK) return rc;
    if (!refs || !source) return fail(ctx, ETF_EINVAL, "null pointer");
    ForkArgs a{};
    if ((rc = check_ws(ctx, ws, ws_bytes, plan_fork(cache, (char *)ws, a))) != ETF_OK) return rc;
    const int64_t grid = (int64_t)cache->batch * cache->heads;
    if (too_many(3 * grid)) return fail(ctx, ETF_EINVAL, "too many rows for one call");
    a.c = view_of(cache);
    a.refs = refs;
    a.source = source;
    a.keep = keep;
    a.row = cache->head_dim;
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    hipStream_t st = (hipStream_t)ctx->stream;
    hipLaunchKernelGGL(k_kv_fork_plan, dim3((unsigned)grid), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_fork_plan");
    hipLaunchKernelGGL(k_kv_fork, dim3((unsigned)(3 * grid)), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_fork");
    return ETF_OK;
}

extern "C" int64_t etf_kv_compact_workspace_bytes(const etf_ctx *ctx, const etf_kv_cache *cache)
{
    const int rc = check_shape(ctx, cache);
    if (rc != ETF_OK) return rc;
    CompactArgs a{};
    return plan_compact(cache, nullptr, a);
}

extern "C" int etf_kv_compact(etf_ctx *ctx, const etf_kv_cache *cache, const int32_t *refs, int32_t *table_out, int32_t *refs_out, int32_t *used, void *ws,
                              int64_t ws_bytes)
{
    int rc = check_cache(ctx, cache);
    if (rc != ETF_OK) return rc;
    if (!refs || !table_out || !refs_out || !used) return fail(ctx, ETF_EINVAL, "null pointer");
    CompactArgs a{};
    if ((rc = check_ws(ctx, ws, ws_bytes, plan_compact(cache, (char *)ws, a))) != ETF_OK) return rc;
    a.c = view_of(cache);
    a.refs = refs;
    a.table_out = table_out;
    a.refs_out = refs_out;
    a.used = used;
    // no more than half of the pages can move
    const int64_t entries = (int64_t)cache->batch * cache->heads * cache->max_blocks;
    a.movers = (int)std::min<int64_t>(2048, cache->pages / 2 + 1);
    a.tables = (int)std::min<int64_t>(1024, (entries + 255) / 256);
    const int rest = (int)std::min<int64_t>(256, ((int64_t)cache->pages + 255) / 256);
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    hipStream_t st = (hipStream_t)ctx->stream;
    hipLaunchKernelGGL(k_kv_used_flags, dim3((unsigned)a.taken.chunks), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_used_flags");
    const dim3 grid((unsigned)(a.movers + a.tables + rest));
    if (cache->head_dim == 64) hipLaunchKernelGGL(k_kv_compact<64>, grid, dim3(256), 0, st, a);
    else if (cache->head_dim == 96) hipLaunchKernelGGL(k_kv_compact<96>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_kv_compact<128>, grid, dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_compact");
    return ETF_OK;
}
