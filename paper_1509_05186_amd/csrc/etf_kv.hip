// Attention over a cache in 8 bits: checks of arguments, workspace sizes, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <limits>

#include "etf_internal.h"
#include "etf_launch.h"

using namespace etf;

namespace {

#include "etf_kv_kernels.hip.h"

inline int64_t al256(int64_t x) { return (x + 255) & ~(int64_t)255; }
inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// a launch has fewer than 2^32 threads
inline bool too_many(int64_t groups, int threads = 256) { return groups > (int64_t)UINT32_MAX / threads; }
constexpr int KV_EVICT_MOST = 16384;  // blocks of a row that a workgroup of k_kv_evict holds

// arrays: the call goes to the device and reads them
int check_cache(const etf_ctx *ctx, const etf_kv_cache *c, bool arrays)
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
    if (!arrays) return ETF_OK;
    const void *all[] = {c->k, c->v, c->bounds, c->scales, c->tail_k, c->tail_v, c->table, c->lens, c->evicted};
    for (const void *p : all)
        if (!p || !aligned16(p)) return fail(ctx, ETF_EINVAL, "an array of the cache is null or not 16-byte aligned");
    return ETF_OK;
}

// strides of sequence, token and head of rows [batch][n][heads][dim]; offsets within a sequence's rows fit the kernels' arithmetic
int check_rows(const etf_ctx *ctx, const etf_kv_cache *c, const char *what, const void *p, const int64_t *strides, int64_t n, int64_t heads, int64_t (&out)[3])
{
    if (!p || !aligned16(p)) return fail(ctx, ETF_EINVAL, "%s is null or not 16-byte aligned", what);
    if (!strides) {
        out[2] = c->head_dim;
        out[1] = heads * c->head_dim;
        out[0] = n * out[1];
        return ETF_OK;
    }
    for (int i = 0; i < 3; ++i) {
        if (strides[i] < 0 || strides[i] % 8 != 0 || strides[i] > (int64_t)1 << 40)
            return fail(ctx, ETF_EINVAL, "stride %d of %s must be a multiple of 8 elements, not negative (it is %lld)", i, what, (long long)strides[i]);
        out[i] = strides[i];
    }
    return ETF_OK;
}

int check_queries(const etf_ctx *ctx, const etf_kv_cache *c, int n, int heads_q)
{
    if (n < 1 || heads_q < 1) return fail(ctx, ETF_EINVAL, "n and heads_q must be positive (%d, %d)", n, heads_q);
    if (heads_q % c->heads != 0) return fail(ctx, ETF_EINVAL, "heads_q (%d) must be a multiple of the cache's heads (%d)", heads_q, c->heads);
    if ((int64_t)n * heads_q > INT32_MAX / 16 / c->batch) return fail(ctx, ETF_EINVAL, "batch * n * heads_q must stay below 2^27");
    return ETF_OK;
}

KvView view_of(const etf_kv_cache *c)
{
    return KvView{(uint8_t *)c->k, (uint8_t *)c->v, (uint8_t *)c->bounds, c->scales, (uint16_t *)c->tail_k, (uint16_t *)c->tail_v,
                  c->table, c->lens, c->evicted, c->batch, c->heads, c->max_blocks, c->pages};
}

// calls f(type, dimensions) with the cache's as constants
template <typename F>
int with_shape(const etf_kv_cache *c, F f)
{
    auto dims = [&](auto t) {
        switch (c->head_dim) {
            case 64: return f(t, std::integral_constant<int, 64>());
            case 96: return f(t, std::integral_constant<int, 96>());
            default: return f(t, std::integral_constant<int, 128>());
        }
    };
    return c->dtype == ETF_KV_BF16 ? dims(TBf()) : dims(THf());
}

int enter_device(const etf_ctx *ctx)
{
    if (ctx->device < 0) return fail(ctx, ETF_ENOGPU, "host-only context");
    HIP_TRY(ctx, hipSetDevice(ctx->device));
    return ETF_OK;
}

// How an attention call is cut up, and where its workspace's arrays lie.
struct AttendPlan {
    bool many = false;  // tiles of 128 rows instead of 16
    bool solo = false;  // listed blocks: a wave to a unit
    int tiles = 0, splits = 1, rows = 16;
    bool split = false;  // whole caches: into ranges
    int64_t units = 0, grid = 0, o_ml = 0, o_plan = 0, o_row = 0, o_block = 0, total = 0;
};

AttendPlan plan_attend(const etf_kv_cache *c, int n, int heads_q, int w, bool mass)
{
    AttendPlan p;
    const int g = heads_q / c->heads;
    const int64_t rows = (int64_t)n * g;
    if (w > 0) {
        p.tiles = (g + 15) / 16;
        p.units = (int64_t)c->batch * n * c->heads * p.tiles;
        // enough workgroups for the card, none with less than a block to a wave
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>((w + 1) / KV_LEAST, 512 / std::max<int64_t>(1, p.units)));
        p.solo = p.units >= 2048;
        p.grid = p.solo ? (p.units / c->heads + 3) / 4 * c->heads : p.units * p.splits;
    } else {
        p.many = rows > 64;
        p.rows = p.many ? 128 : 16;
        p.tiles = (int)((rows + p.rows - 1) / p.rows);
        p.units = (int64_t)p.tiles * c->heads;
        // up to KV_ROUNDS rounds of workgroups (kv_plan) and one for each unit of a sequence; a card full of workgroups from the tiles of prompts alone
        // needs no ranges
        const int64_t units = c->batch * p.units;
        // Short tables are hardly faster in ranges, whose join is a launch of its own; the host knows the table's columns but not the
        // lengths, so a short sequence in a wide table is cut all the same.  Single tokens, 8 heads of 128 dimensions, not cut and cut: one sequence of 500
        // tokens 8.9 and 11.5 us, 1000 tokens 11.5 and 11.2, 2000 tokens 17.0 and 11.6; 16 sequences of 1000 tokens 14.2 and 18.8, 2000 tokens
        // 19.8 and 23.3, 4000 tokens 30.5 and 32.0, but ragged ones 28.7 and 14.9 (one of 4000, the others of 500) and 29.9 and 23.8 (500 to 4000 evenly),
        // so that the limit for many units stays below what equal lengths would allow.
        p.split = p.many ? units < 1024 : c->max_blocks > (units >= 128 ? 32 : 16);
        p.grid = (p.split ? KV_ROUNDS * KV_ROUND : 0) + units;
    }
    const bool parts = w > 0 ? p.splits > 1 : p.split;
    const int64_t slots = parts ? p.grid * p.rows : 0;
    p.o_ml = al256(slots * c->head_dim * 4);
    p.o_plan = p.o_ml + al256(slots * 2 * 4);
    p.o_row = p.o_plan + (p.split ? al256((int64_t)c->batch * 16) : 0);
    const int64_t all_rows = mass ? (int64_t)c->batch * c->heads * rows : 0;
    p.o_block = p.o_row + al256(all_rows * 4);
    p.total = std::max<int64_t>(256, p.o_block + al256(all_rows * (c->max_blocks + 1) * 4));
    return p;
}

template <typename T, int D, bool LIST, bool MASS>
int launch_attend(etf_ctx *ctx, const KvAttendArgs &a, const AttendPlan &p)
{
    hipStream_t st = (hipStream_t)ctx->stream;
    ProfScope prof(ctx, ETF_K_KV);
    if constexpr (!LIST) {
        if (p.many) {
            hipLaunchKernelGGL((k_kv_tile<T, D, MASS>), dim3((unsigned)p.grid), dim3(256), 0, st, a);
            LAUNCH_CHECK(ctx, "k_kv_tile");
            if (p.split) {
                hipLaunchKernelGGL((k_kv_join<T, D, 128, false, MASS>), dim3((unsigned)(a.c.batch * p.units * 16)), dim3(256), 0, st, a);
                LAUNCH_CHECK(ctx, "k_kv_join");
            }
            return ETF_OK;
        }
    }
    if constexpr (LIST) {
        if (p.solo) {
            hipLaunchKernelGGL((k_kv_attend<T, D, true, false, true>), dim3((unsigned)p.grid), dim3(256), 0, st, a);
            LAUNCH_CHECK(ctx, "k_kv_attend");
            return ETF_OK;
        }
    }
    hipLaunchKernelGGL((k_kv_attend<T, D, LIST, MASS, false>), dim3((unsigned)p.grid), dim3(256), 0, st, a);
    LAUNCH_CHECK(ctx, "k_kv_attend");
    if (LIST ? p.splits > 1 : p.split) {
        const int64_t units = LIST ? p.units : a.c.batch * p.units;
        hipLaunchKernelGGL((k_kv_join<T, D, 16, LIST, MASS>), dim3((unsigned)units * 2), dim3(256), 0, st, a);
        LAUNCH_CHECK(ctx, "k_kv_join");
    }
    return ETF_OK;
}

}  // namespace

extern "C" int etf_kv_append(etf_ctx *ctx, const etf_kv_cache *cache, const void *k, const int64_t *k_strides, const void *v,
                             const int64_t *v_strides, int n, const int32_t *counts)
{
    int rc = check_cache(ctx, cache, true);
    if (rc != ETF_OK) return rc;
    if (n < 1 || n > (1 << 24)) return fail(ctx, ETF_EINVAL, "need 1 <= n <= 2^24 (n=%d)", n);
    KvAppendArgs a{};
    a.c = view_of(cache);
    if ((rc = check_rows(ctx, cache, "k", k, k_strides, n, cache->heads, a.ks)) != ETF_OK) return rc;
    if ((rc = check_rows(ctx, cache, "v", v, v_strides, n, cache->heads, a.vs)) != ETF_OK) return rc;
    a.k = (const uint16_t *)k;
    a.v = (const uint16_t *)v;
    a.counts = counts;
    a.n = n;
    const int64_t most = std::max(1, (KB - 1 + n) / KB);  // blocks that n tokens can complete
    a.per = (int)most;
    const int64_t grid = (int64_t)cache->batch * cache->heads * most;
    if (too_many(grid)) return fail(ctx, ETF_EINVAL, "too many blocks for one call");
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    return with_shape(cache, [&](auto t, auto dim) {
        ProfScope prof(ctx, ETF_K_KV);
        hipLaunchKernelGGL((k_kv_append<decltype(t), decltype(dim)::value>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)ctx->stream, a);
        LAUNCH_CHECK(ctx, "k_kv_append");
        return (int)ETF_OK;
    });
}

extern "C" int64_t etf_kv_attend_workspace_bytes(const etf_ctx *ctx, const etf_kv_cache *cache, int n, int heads_q, int w, int mass)
{
    int rc = check_cache(ctx, cache, false);
    if (rc != ETF_OK) return rc;
    if ((rc = check_queries(ctx, cache, n, heads_q)) != ETF_OK) return rc;
    if (w < 0 || w > ETF_KV_MAX_LIST) return fail(ctx, ETF_EINVAL, "need 0 <= w <= %d (w=%d)", ETF_KV_MAX_LIST, w);
    if (w > 0 && mass) return fail(ctx, ETF_EINVAL, "weights of blocks are not gathered over lists");
    return plan_attend(cache, n, heads_q, w, mass != 0).total;
}

extern "C" int etf_kv_attend(etf_ctx *ctx, const etf_kv_cache *cache, const void *q, const int64_t *q_strides, int n, int heads_q, float scale,
                             const int32_t *counts, const int32_t *lists, int w, void *out, float *lse, const float *mass_in, float *mass_out,
                             void *ws, int64_t ws_bytes)
{
    int rc = check_cache(ctx, cache, true);
    if (rc != ETF_OK) return rc;
    if ((rc = check_queries(ctx, cache, n, heads_q)) != ETF_OK) return rc;
    if (lists ? w < 1 || w > ETF_KV_MAX_LIST : w != 0) return fail(ctx, ETF_EINVAL, "need 1 <= w <= %d with lists, 0 without (w=%d)", ETF_KV_MAX_LIST, w);
    if (lists && mass_out) return fail(ctx, ETF_EINVAL, "weights of blocks are not gathered over lists");
    if (mass_in && !mass_out) return fail(ctx, ETF_EINVAL, "mass_in without mass_out");
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(ctx, ETF_EINVAL, "scale must be positive and finite");
    if (!out || !aligned16(out)) return fail(ctx, ETF_EINVAL, "out is null or not 16-byte aligned");
    if (!ws || ((uintptr_t)ws & 255) != 0) return fail(ctx, ETF_EINVAL, "workspace is null or not 256-byte aligned");
    const AttendPlan p = plan_attend(cache, n, heads_q, w, mass_out != nullptr);
    if (ws_bytes < p.total) return fail(ctx, ETF_ENOMEM, "workspace too small: %lld < %lld", (long long)ws_bytes, (long long)p.total);
    KvAttendArgs a{};
    a.c = view_of(cache);
    if ((rc = check_rows(ctx, cache, "q", q, q_strides, n, heads_q, a.qs)) != ETF_OK) return rc;
    // lanes of a block's weight (k_kv_mass)
    int width = 1;
    while (width < 256 && width < n * (heads_q / cache->heads)) width *= 2;
    const int64_t blocks = (int64_t)cache->batch * cache->heads * cache->max_blocks, mass_grid = (blocks + 256 / width - 1) / (256 / width);
    const int64_t joins = lists ? p.splits > 1 ? 2 * p.units : 0 : p.split ? cache->batch * p.units * (p.rows / 8) : 0;
    if (too_many(p.grid) || too_many(joins) || (mass_out && too_many(mass_grid))) return fail(ctx, ETF_EINVAL, "too many rows for one call");
    char *base = (char *)ws;
    a.q = (const uint16_t *)q;
    a.counts = counts;
    a.lists = lists;
    a.out = (uint16_t *)out;
    a.lse = lse;
    a.part_o = (float *)base;
    a.part_ml = (float *)(base + p.o_ml);
    a.plan = (int4 *)(base + p.o_plan);
    a.row_lse = (float *)(base + p.o_row);
    a.block_lse = (float *)(base + p.o_block);
    a.scale2 = std::min(scale * 1.4426950408889634f, std::numeric_limits<float>::max());
    a.n = n;
    a.g = heads_q / cache->heads;
    a.w = w;
    a.splits = p.splits;
    a.tiles = p.tiles;
    a.units = p.units;
    a.split = p.split;
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    rc = with_shape(cache, [&](auto t, auto dim) {
        using T = decltype(t);
        constexpr int D = decltype(dim)::value;
        if (lists) return launch_attend<T, D, true, false>(ctx, a, p);
        return mass_out ? launch_attend<T, D, false, true>(ctx, a, p) : launch_attend<T, D, false, false>(ctx, a, p);
    });
    if (rc != ETF_OK || !mass_out) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    hipLaunchKernelGGL(k_kv_mass, dim3((unsigned)mass_grid), dim3(256), 0, (hipStream_t)ctx->stream, a.c, a.row_lse, a.block_lse, n * a.g, width, mass_in, mass_out);
    LAUNCH_CHECK(ctx, "k_kv_mass");
    return ETF_OK;
}

extern "C" int64_t etf_kv_select_workspace_bytes(const etf_ctx *ctx, const etf_kv_cache *cache, int n, int heads_q, int w)
{
    int rc = check_cache(ctx, cache, false);
    if (rc != ETF_OK) return rc;
    if ((rc = check_queries(ctx, cache, n, heads_q)) != ETF_OK) return rc;
    if (w < 1 || w > ETF_KV_MAX_LIST) return fail(ctx, ETF_EINVAL, "need 1 <= w <= %d (w=%d)", ETF_KV_MAX_LIST, w);
    return al256((int64_t)cache->batch * n * cache->heads * cache->max_blocks * 8);
}

extern "C" int etf_kv_select(etf_ctx *ctx, const etf_kv_cache *cache, const void *q, const int64_t *q_strides, int n, int heads_q,
                             const int32_t *counts, int w, int sink, int recent, int32_t *lists, void *ws, int64_t ws_bytes)
{
    int rc = check_cache(ctx, cache, true);
    if (rc != ETF_OK) return rc;
    if ((rc = check_queries(ctx, cache, n, heads_q)) != ETF_OK) return rc;
    if (w < 1 || w > ETF_KV_MAX_LIST) return fail(ctx, ETF_EINVAL, "need 1 <= w <= %d (w=%d)", ETF_KV_MAX_LIST, w);
    if (sink < 0 || recent < 0 || sink > w || recent > w - sink) return fail(ctx, ETF_EINVAL, "need sink + recent <= w (%d, %d, %d)", sink, recent, w);
    if (!lists) return fail(ctx, ETF_EINVAL, "lists is null");
    if (!ws || ((uintptr_t)ws & 255) != 0) return fail(ctx, ETF_EINVAL, "workspace is null or not 256-byte aligned");
    const int64_t rows = (int64_t)cache->batch * n * cache->heads, need = al256(rows * cache->max_blocks * 8);
    if (ws_bytes < need) return fail(ctx, ETF_ENOMEM, "workspace too small: %lld < %lld", (long long)ws_bytes, (long long)need);
    KvSelectArgs a{};
    a.c = view_of(cache);
    if ((rc = check_rows(ctx, cache, "q", q, q_strides, n, heads_q, a.qs)) != ETF_OK) return rc;
    a.q = (const uint16_t *)q;
    a.counts = counts;
    a.scores = (uint64_t *)ws;
    a.lists = lists;
    a.n = n;
    a.g = heads_q / cache->heads;
    a.w = w;
    a.sink = sink;
    a.recent = recent;
    a.gp = 1;
    while (a.gp < std::min(a.g, 16)) a.gp *= 2;
    a.tokens = 16 / a.gp;
    a.tiles = (n + a.tokens - 1) / a.tokens;
    const int64_t chunks = (int64_t)cache->batch * cache->heads * ((cache->max_blocks + 63) / 64);
    // a wave keeps its blocks' bounds for several tiles of tokens, as long as there are workgroups for every compute unit
    a.turns = (int)std::max<int64_t>(1, std::min<int64_t>(8, chunks * a.tiles / 1024));
    const int64_t grid = chunks * ((a.tiles + a.turns - 1) / a.turns);
    const bool many = cache->max_blocks <= 1024 ? too_many((rows + 3) / 4) : too_many(rows, cache->max_blocks <= 4096 ? 256 : 1024);
    if (too_many(grid) || many) return fail(ctx, ETF_EINVAL, "too many rows for one call");
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    return with_shape(cache, [&](auto t, auto dim) {
        using T = decltype(t);
        constexpr int D = decltype(dim)::value;
        hipStream_t st = (hipStream_t)ctx->stream;
        hipLaunchKernelGGL((k_kv_score<T, D>), dim3((unsigned)grid), dim3(256), 0, st, a);
        LAUNCH_CHECK(ctx, "k_kv_score");
        // a wave to a row as long as it holds the row's keys
        const unsigned four = (unsigned)((rows + 3) / 4), one = (unsigned)rows;
        if (cache->max_blocks <= 256)
            hipLaunchKernelGGL((k_kv_pick<T, D, 4, 1, 4>), dim3(four), dim3(256), 0, st, a);
        else if (cache->max_blocks <= 1024)
            hipLaunchKernelGGL((k_kv_pick<T, D, 4, 1, 16>), dim3(four), dim3(256), 0, st, a);
        else if (cache->max_blocks <= 4096)
            hipLaunchKernelGGL((k_kv_pick<T, D, 1, 4, 16>), dim3(one), dim3(256), 0, st, a);
        else if (cache->max_blocks <= 16384)
            hipLaunchKernelGGL((k_kv_pick<T, D, 1, 16, 16>), dim3(one), dim3(1024), 0, st, a);
        else
            hipLaunchKernelGGL((k_kv_pick<T, D, 1, 16, 0>), dim3(one), dim3(1024), 0, st, a);
        LAUNCH_CHECK(ctx, "k_kv_pick");
        return (int)ETF_OK;
    });
}

extern "C" int etf_kv_evict(etf_ctx *ctx, const etf_kv_cache *cache, const float *mass, int budget, int sink, int recent, int32_t *table_out,
                            int32_t *lens_out, int32_t *evicted_out, float *mass_out, int32_t *freed)
{
    int rc = check_cache(ctx, cache, true);
    if (rc != ETF_OK) return rc;
    if (budget < 1 || sink < 0 || recent < 0 || sink > budget || recent > budget - sink)
        return fail(ctx, ETF_EINVAL, "need sink + recent <= budget, budget >= 1 (%d, %d, %d)", sink, recent, budget);
    if (!mass || !table_out || !lens_out || !evicted_out || !mass_out || !freed) return fail(ctx, ETF_EINVAL, "null pointer");
    if (cache->max_blocks > KV_EVICT_MOST && (table_out == cache->table || mass_out == mass))
        return fail(ctx, ETF_EINVAL, "tables of more than %d blocks are not cut in place", KV_EVICT_MOST);
    const int64_t rows = (int64_t)cache->batch * cache->heads;
    if (too_many(rows, cache->max_blocks <= 256 ? 64 : cache->max_blocks <= 4096 ? 256 : 1024)) return fail(ctx, ETF_EINVAL, "too many rows for one call");
    if ((rc = enter_device(ctx)) != ETF_OK) return rc;
    ProfScope prof(ctx, ETF_K_KV);
    const KvView c = view_of(cache);
    const dim3 grid((unsigned)rows);
    hipStream_t st = (hipStream_t)ctx->stream;
    const bool apart = lens_out != cache->lens && evicted_out != cache->evicted && lens_out != cache->evicted && evicted_out != cache->lens;
    int32_t *lens = apart ? lens_out : nullptr;
    if (cache->max_blocks <= 256)
        hipLaunchKernelGGL((k_kv_evict<1, 4>), grid, dim3(64), 0, st, c, mass, budget, sink, recent, table_out, mass_out, freed, lens, evicted_out);
    else if (cache->max_blocks <= 1024)
        hipLaunchKernelGGL((k_kv_evict<4, 4>), grid, dim3(256), 0, st, c, mass, budget, sink, recent, table_out, mass_out, freed, lens, evicted_out);
    else if (cache->max_blocks <= 4096)
        hipLaunchKernelGGL((k_kv_evict<4, 16>), grid, dim3(256), 0, st, c, mass, budget, sink, recent, table_out, mass_out, freed, lens, evicted_out);
    else if (cache->max_blocks <= KV_EVICT_MOST)
        hipLaunchKernelGGL((k_kv_evict<16, 16>), grid, dim3(1024), 0, st, c, mass, budget, sink, recent, table_out, mass_out, freed, lens, evicted_out);
    else
        hipLaunchKernelGGL((k_kv_evict<16, 0>), grid, dim3(1024), 0, st, c, mass, budget, sink, recent, table_out, mass_out, freed, lens, evicted_out);
    LAUNCH_CHECK(ctx, "k_kv_evict");
    if (apart) return ETF_OK;
    hipLaunchKernelGGL(k_kv_evict_lens, dim3((unsigned)((cache->batch + 63) / 64)), dim3(64), 0, st, c, budget, lens_out, evicted_out);
    LAUNCH_CHECK(ctx, "k_kv_evict_lens");
    return ETF_OK;
}
