// What the sources that launch kernels share: checks of HIP calls and launches, timing of launches.
#pragma once

#include <hip/hip_runtime.h>

#include "etf_internal.h"

#define HIP_TRY(ctx, call)                                                                            \
    do {                                                                                              \
        hipError_t e_ = (call);                                                                       \
        if (e_ != hipSuccess) return etf::fail(ctx, ETF_EHIP, "%s: %s", #call, hipGetErrorString(e_));     \
    } while (0)

#define LAUNCH_CHECK(ctx, name)                                                                       \
    do {                                                                                              \
        hipError_t e_ = hipGetLastError();                                                            \
        if (e_ != hipSuccess) return etf::fail(ctx, ETF_EHIP, "launch of %s: %s", name, hipGetErrorString(e_)); \
    } while (0)

// Brackets the launches made during its lifetime with a pair of events when profiling is on.
struct ProfScope {
    etf_ctx *ctx;
    etf_ctx::Stamp st{nullptr, nullptr, 0};
    bool live = false;
    ProfScope(etf_ctx *c, int cls) : ctx(c)
    {
        if (!c->profile_on || c->no_alloc_call) return;
        if (!c->stamp_pool.empty()) {
            st = c->stamp_pool.back();
            c->stamp_pool.pop_back();
        } else {
            hipEvent_t a, b;
            if (hipEventCreate(&a) != hipSuccess) return;
            if (hipEventCreate(&b) != hipSuccess) { (void)hipEventDestroy(a); return; }
            st.start = a;
            st.stop = b;
        }
        st.cls = cls;
        live = hipEventRecord((hipEvent_t)st.start, (hipStream_t)c->stream) == hipSuccess;
        if (!live) c->stamp_pool.push_back(st);
    }
    ~ProfScope()
    {
        if (!live) return;
        (void)hipEventRecord((hipEvent_t)st.stop, (hipStream_t)ctx->stream);
        try {
            ctx->stamps.push_back(st);
        } catch (...) {  // no memory for the record: the launch goes unmeasured
            (void)hipEventDestroy((hipEvent_t)st.start);
            (void)hipEventDestroy((hipEvent_t)st.stop);
        }
    }
};
