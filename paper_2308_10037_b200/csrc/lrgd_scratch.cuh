// What the token-gate and class-loss entry points share on the host: the scratch of a call (the context's, or a captured graph's own),
// launches that are counted, and grids.
#pragma once
#include "lrgd_ctx.cuh"

using namespace lrgd;

namespace {

// What a call works in: `words` are kGateWords counters that are zero between calls, `data` is at least what it asked for.
struct Scratch {
    unsigned char* data;
    unsigned int* words;
};

int alloc_failed(lr_ctx* ctx, cudaError_t e) {
    cudaGetLastError();
    ctx->last_cuda = int(e);
    return e == cudaErrorMemoryAllocation ? LR_ERR_NOMEM : LR_ERR_CUDA;
}

// A capture: the scratch of this graph and stream, made now if there is none that is large enough (see GraphScratch).
int captured_scratch(lr_ctx* ctx, size_t need, cudaStream_t st, unsigned long long id, cudaGraph_t graph, Scratch* out) {
    constexpr size_t kWordBytes = kGateWords * sizeof(unsigned int);
    auto use = [&](const GraphScratch* b) {
        out->words = reinterpret_cast<unsigned int*>(b->base + kGuardBytes);
        out->data = b->base + kGuardBytes + kWordBytes;
        return LR_OK;
    };
    GraphScratches& g = graph_scratches();
    const std::lock_guard<std::mutex> hold(g.mu);
    for (const GraphScratch* b : g.all)
        if (!b->dead.load() && b->owner == ctx && b->capture == id && b->stream == st && b->body >= kWordBytes + need) return use(b);
    try {
        g.all.reserve(g.all.size() + 1);
    } catch (const std::bad_alloc&) {
        return LR_ERR_NOMEM;
    }
    GraphScratch* b = new (std::nothrow) GraphScratch{ctx, ctx->device, id, st, nullptr, 0};
    if (!b) return LR_ERR_NOMEM;
    cudaError_t e = guarded_block(ctx, kWordBytes + need, &b->base, &b->body);
    if (e == cudaSuccess) e = cudaMemsetAsync(b->base + kGuardBytes, 0, kWordBytes, ctx->hstream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(ctx->hstream);
    cudaUserObject_t object = nullptr;
    if (e == cudaSuccess) e = cudaUserObjectCreate(&object, b, end_of_graph, 1, cudaUserObjectNoDestructorSync);
    if (e != cudaSuccess) {
        if (b->base) cudaFree(b->base);
        delete b;
        return alloc_failed(ctx, e);
    }
    g.all.push_back(b);
    e = cudaGraphRetainUserObject(graph, object, 1, cudaGraphUserObjectMove);
    if (e != cudaSuccess) {
        cudaUserObjectRelease(object, 1);           // marks it dead
        return alloc_failed(ctx, e);
    }
    return use(b);
}

// The scratch of a call on `st`.  Outside a capture it is the context's, between guard regions, grown (by half at least) when a call needs
// more than any before it; what it outgrew is freed.  A capture gets scratch of the graph's own.
int gate_scratch(lr_ctx* ctx, size_t need, cudaStream_t st, Scratch* out) {
    if (st != nullptr && st != cudaStreamLegacy) {              // (the legacy stream cannot be captured)
        cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
        unsigned long long id = 0;
        cudaGraph_t graph = nullptr;
        LR_CK(ctx, cudaStreamGetCaptureInfo(st, &capturing, &id, &graph));
        if (capturing == cudaStreamCaptureStatusActive) {
            const RelaxedCapture relaxed;
            return captured_scratch(ctx, need, st, id, graph, out);
        }
    }
    if (graph_scratches().dead.load() > 0) {
        const RelaxedCapture relaxed;
        free_dead_scratch();
    }
    if (ctx->scratch_bytes < need) {
        need = std::max(need, ctx->scratch_bytes + ctx->scratch_bytes / 2);
        need = (need + (size_t(1) << 20) - 1) >> 20 << 20;
        const RelaxedCapture relaxed;
        if (ctx->scratch_bytes > 0) {
            for (size_t i = 0; i < ctx->guard_bases.size(); ++i) {
                if (ctx->guard_bases[i] + kGuardBytes != ctx->d_scratch) continue;
                cudaFree(ctx->guard_bases[i]);      // waits for the calls that use it
                ctx->guard_bases.erase(ctx->guard_bases.begin() + i);
                ctx->guard_sizes.erase(ctx->guard_sizes.begin() + i);
                break;
            }
            ctx->d_scratch = nullptr;
            ctx->scratch_bytes = 0;
        }
        try {
            ctx->guard_bases.reserve(ctx->guard_bases.size() + 1);
            ctx->guard_sizes.reserve(ctx->guard_sizes.size() + 1);
        } catch (const std::bad_alloc&) {
            return LR_ERR_NOMEM;
        }
        unsigned char* fresh = nullptr;
        const cudaError_t e = guarded_alloc(ctx, &fresh, need);
        if (e != cudaSuccess) return alloc_failed(ctx, e);
        ctx->d_scratch = fresh;
        ctx->scratch_bytes = need;
    }
    out->data = ctx->d_scratch;
    out->words = ctx->d_gate_words;
    return LR_OK;
}

template <class K>
int launched(lr_ctx* ctx, K&& launch) {
    launch();
    LR_CK(ctx, cudaGetLastError());
    ctx->launches += 1;
    return LR_OK;
}

int grid_for(const lr_ctx* ctx, int64_t units, int64_t per_cta, int per_sm) {
    return int(std::max<int64_t>(1, std::min<int64_t>((units + per_cta - 1) / per_cta, int64_t(plan_sms(ctx)) * per_sm)));
}

// The same with every CTA taking equally many turns, so that the last turn is not that of a few
int even_grid(const lr_ctx* ctx, int64_t units, int64_t per_cta, int per_sm) {
    const int64_t ctas = (units + per_cta - 1) / per_cta, most = int64_t(plan_sms(ctx)) * per_sm, turns = (ctas + most - 1) / most;
    return int((ctas + turns - 1) / turns);
}

}  // namespace
