// Attention over whole prompts: checks of arguments, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "etf_internal.h"
#include "etf_launch.h"

using namespace etf;

namespace {

#include "etf_prompt_kernels.hip.h"

constexpr int64_t PROMPT_FEW = 768;    // (tile, head) units from which the card is full without ranges: it holds 512 workgroups of 128 dimensions at once, 768 of 64 and 96
constexpr int64_t PROMPT_LEAST = 8;    // blocks of a range, at least
constexpr int64_t PROMPT_RANGES = 16;  // ranges of a tile, at most

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// strides of token and head of rows [tokens][heads][dim]
int check_packed(const etf_ctx *ctx, const char *what, const void *p, const int64_t *strides, int64_t heads, int dim, int64_t (&out)[2])
{
    if (!p || !aligned16(p)) return fail(ctx, ETF_EINVAL, "%s is null or not 16-byte aligned", what);
    out[0] = strides ? strides[0] : heads * dim;
    out[1] = strides ? strides[1] : dim;
    for (int i = 0; i < 2; ++i)
        if (out[i] < 0 || out[i] % 8 != 0 || out[i] > (i ? (int64_t)1 << 40 : (int64_t)1 << 23))
            return fail(ctx, ETF_EINVAL, "stride %d of %s must be a multiple of 8 elements, not negative and within bounds (it is %lld)", i, what, (long long)out[i]);
    return ETF_OK;
}

inline int64_t al256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// How a call is cut up, and where its workspace's arrays lie.
struct PromptPlan {
    int64_t tiles = 0, grid = 0, o_ml = 0, total = 0;  // tiles of one head that there can be
    int ranges = 1, per = INT32_MAX;
};

int plan_prompt(const etf_ctx *ctx, int head_dim, int64_t tokens, int heads_q, int heads, int batch, PromptPlan &p)
{
    if (!ctx) return ETF_EINVAL;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128) return fail(ctx, ETF_EINVAL, "head_dim must be 64, 96 or 128 (it is %d)", head_dim);
    if (tokens < 1 || heads_q < 1 || heads < 1 || batch < 1)
        return fail(ctx, ETF_EINVAL, "tokens, heads_q, heads and batch must be positive (%lld, %d, %d, %d)", (long long)tokens, heads_q, heads, batch);
    if (heads_q % heads != 0) return fail(ctx, ETF_EINVAL, "heads_q (%d) must be a multiple of heads (%d)", heads_q, heads);
    if (tokens > INT32_MAX / heads_q || batch > (1 << 24)) return fail(ctx, ETF_EINVAL, "tokens * heads_q must stay below 2^31, batch up to 2^24");
    p.tiles = tokens * (heads_q / heads) / 128 + batch;
    // Few tiles do not fill the card, and the longest of them decides: their blocks are cut into ranges of `per`.  What that costs is the ranges' partial
    // results, written and read again, about as much as 1 / 35 of a block's time for each of them, and the launch that joins them, four blocks':
    // per blocks and units * longest / (2 per) partial results take the least together where both are sqrt(units * longest / 70).  The
    // host knows the number of tokens, not the lengths: of several prompts the longest is taken to be twice the mean (one of 8000 tokens, 1 head, beside 15 of one
    // token is left uncut, 144 us).  Measured with 128 dimensions, for all.
    // One prompt, 128 dimensions: 4096 tokens, 2 heads 79 us uncut, 38 cut; 8000 tokens, 1 head 145 and 45 to 51; 8 heads, four query heads to each:
    // 600 tokens 20 and 25, 1000 tokens 28 and 36, 2000 tokens 51 and 72, which are left uncut.
    const int64_t units = p.tiles * heads, blocks = (tokens + KB - 1) / KB, longest = batch == 1 ? blocks : std::min(blocks, 2 * ((blocks + batch - 1) / batch));
    const int64_t per = std::max<int64_t>(PROMPT_LEAST, (int64_t)std::sqrt(units * longest / 70.));
    if (units < PROMPT_FEW && 2 * per + 4 <= longest * 17 / 20) {
        p.per = (int)std::max(per, (blocks + PROMPT_RANGES - 1) / PROMPT_RANGES);
        p.ranges = (int)((blocks + p.per - 1) / p.per);
    }
    if (p.ranges == 1) p.per = INT32_MAX;
    p.grid = units * p.ranges;
    if (p.ranges > 1) {
        p.o_ml = al256(p.grid * 128 * head_dim * 4);
        p.total = p.o_ml + al256(p.grid * 128 * 2 * 4);
    }
    if (p.grid > (int64_t)UINT32_MAX / 256) return fail(ctx, ETF_EINVAL, "too many rows for one call");
    return ETF_OK;
}

template <typename T, int D>
int launch_prompt(etf_ctx *ctx, const PromptArgs &a, const PromptPlan &p)
{
    ProfScope prof(ctx, ETF_K_KV);
    hipLaunchKernelGGL((k_prompt<T, D>), dim3((unsigned)p.grid), dim3(256), 0, (hipStream_t)ctx->stream, a);
    LAUNCH_CHECK(ctx, "k_prompt");
    if (p.ranges > 1) {
        hipLaunchKernelGGL((k_prompt_join<T, D>), dim3((unsigned)(p.grid / p.ranges * 16)), dim3(256), 0, (hipStream_t)ctx->stream, a);
        LAUNCH_CHECK(ctx, "k_prompt_join");
    }
    return ETF_OK;
}
template <typename T>
int launch_prompt(etf_ctx *ctx, const PromptArgs &a, const PromptPlan &p, int head_dim)
{
    return head_dim == 64 ? launch_prompt<T, 64>(ctx, a, p) : head_dim == 96 ? launch_prompt<T, 96>(ctx, a, p) : launch_prompt<T, 128>(ctx, a, p);
}

}  // namespace

extern "C" int64_t etf_prompt_attend_workspace_bytes(const etf_ctx *ctx, int head_dim, int64_t tokens, int heads_q, int heads, int batch)
{
    PromptPlan p;
    const int rc = plan_prompt(ctx, head_dim, tokens, heads_q, heads, batch, p);
    return rc != ETF_OK ? rc : p.total;
}

extern "C" int etf_prompt_attend(etf_ctx *ctx, int dtype, int head_dim, const void *q, const int64_t *q_strides, const void *k, const int64_t *k_strides,
                                 const void *v, const int64_t *v_strides, int64_t tokens, int heads_q, int heads, const int32_t *starts, int batch, float scale,
                                 void *out, float *lse, void *ws, int64_t ws_bytes)
{
    PromptPlan p;
    int rc = plan_prompt(ctx, head_dim, tokens, heads_q, heads, batch, p);
    if (rc != ETF_OK) return rc;
    if (dtype != ETF_KV_BF16 && dtype != ETF_KV_FP16) return fail(ctx, ETF_EINVAL, "unknown type %d", dtype);
    if (!(scale > 0.f) || !std::isfinite(scale)) return fail(ctx, ETF_EINVAL, "scale must be positive and finite");
    if (!starts || !out || !aligned16(out)) return fail(ctx, ETF_EINVAL, "starts or out is null, or out not 16-byte aligned");
    if (p.total > 0 && (!ws || ((uintptr_t)ws & 255) != 0)) return fail(ctx, ETF_EINVAL, "workspace is null or not 256-byte aligned");
    if (p.total > 0 && ws_bytes < p.total) return fail(ctx, ETF_ENOMEM, "workspace too small: %lld < %lld", (long long)ws_bytes, (long long)p.total);
    PromptArgs a{};
    if ((rc = check_packed(ctx, "q", q, q_strides, heads_q, head_dim, a.qs)) != ETF_OK) return rc;
    if ((rc = check_packed(ctx, "k", k, k_strides, heads, head_dim, a.ks)) != ETF_OK) return rc;
    if ((rc = check_packed(ctx, "v", v, v_strides, heads, head_dim, a.vs)) != ETF_OK) return rc;
    a.q = (const uint16_t *)q;
    a.k = (const uint16_t *)k;
    a.v = (const uint16_t *)v;
    a.seq = Packed{starts, (int)tokens, batch};
    a.out = (uint16_t *)out;
    a.lse = lse;
    a.scale2 = std::min(scale * 1.4426950408889634f, std::numeric_limits<float>::max());
    a.heads = heads;
    a.g = heads_q / heads;
    a.ranges = p.ranges;
    a.per = p.per;
    a.part_o = (float *)ws;
    a.part_ml = (float *)((char *)ws + p.o_ml);
    if (ctx->device < 0) return fail(ctx, ETF_ENOGPU, "host-only context");
    HIP_TRY(ctx, hipSetDevice(ctx->device));
    return dtype == ETF_KV_BF16 ? launch_prompt<TBf>(ctx, a, p, head_dim) : launch_prompt<THf>(ctx, a, p, head_dim);
}
