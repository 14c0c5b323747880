// The context behind every entry point, and the host helpers that the translation units of the library share: guarded
// workspaces, the device guard, error propagation and kernel launches.
#pragma once
#include "../../include/lrgd.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <new>
#include <vector>

namespace lrgd {
struct TolState;
struct FitParams;
}  // namespace lrgd

constexpr size_t kGateWords = 2048;

struct lr_ctx {
    int device = 0;
    int sm_count = 0;
    int n_max = 0;
    double* d_partial = nullptr;
    int* d_status = nullptr;                        // [0] a wait that ran out, [1] a token outside its table: neither hides the other
    lrgd::TolState* d_tol = nullptr;                // stopping-rule state of lr_fit_tol
    double* d_gbuf = nullptr;                       // [n_max+1] gradient entries for the norm
    lrgd::TolState* h_tol = nullptr;                // pinned host mirror
    int* h_words = nullptr;                         // pinned: [0] status word before a blocking call, [1] after it, [2] abort word of a persistent launch
    float* d_vel = nullptr;                         // [n_max+1] velocity of lr_fit_opt when the caller passes none
    double* d_oscr = nullptr;                       // [n_max+2] scratch of the optimiser reduction
    unsigned int* d_oticket = nullptr;
    unsigned int* d_gbar = nullptr;                 // persistent fit kernel: [0] grid-barrier counter, [1] abort flag of the launch
                                                    // (one such pair per rank when several ranks run as one launch)
    lrgd::FitParams* d_rank_params = nullptr;       // [kMaxWorld] parameters of the ranks of lr_fit_sharded_local
    int sm_limit = 0;                               // > 0: plans use at most this many SMs (lr_set_sm_limit)
    int cluster_mode = -1;                          // single-cluster fit kernel for tiny problems: -1 the library chooses, 0 never
    bool coop = false;                              // device supports cooperative launches
    int persistent_mode = -1;                       // single-launch fit kernel: -1 the library chooses, 0 never, 1 whenever the shape allows
    bool overlap = true;                            // consecutive kernels of one call are launched as programmatic dependents
    int64_t l2_keep_bytes = -1;                     // leading bytes of X fetched with an evict-last hint; -1 = per-kernel default
    int64_t l2_bytes = 0;                           // size of the device's L2
    // buffers of the host-pointer entry points (grown on demand)
    void* d_hX = nullptr; size_t hX_bytes = 0;
    void* d_hy = nullptr; size_t hy_bytes = 0;
    void* d_hw = nullptr; size_t hw_bytes = 0;      // w[n] | b | loss_hist
    void* d_hl = nullptr; size_t hl_bytes = 0;      // labels
    void* d_hXh = nullptr; size_t hXh_bytes = 0;    // bfloat16 copy of X (lr_fit_host_bf16, lr_predict_host_bf16)
    cudaStream_t hstream = nullptr;
    // One token-gate call at a time, from the look at the scratch to the call's last launch: the kernels of one call hand data to each
    // other through the scratch, so those of another host thread on the same stream must come before or after all of them.
    std::mutex gate_mu;
    // scratch of the token-gate entry points (grown on demand, between guard regions) and their zero-initialised counters
    unsigned char* d_scratch = nullptr; size_t scratch_bytes = 0;
    unsigned int* d_gate_words = nullptr;           // [kGateWords] zero between calls
    // profiling
    bool prof = false;
    std::vector<cudaEvent_t> ev;                    // pairs: start, stop
    int prof_used = 0;
    int64_t launches = 0;
    int last_cuda = 0;
    // guard regions: every device workspace that kernels index by a computed offset sits between two of them
    std::vector<unsigned char*> guard_bases;        // allocation bases; the user range starts kGuardBytes in
    std::vector<size_t> guard_sizes;                // user bytes, rounded up to kGuardBytes
};

namespace lrgd {

// Scratch that belongs to a captured graph: calls captured on one stream use it one after the other, whenever and wherever the graph is
// replayed, and nobody else does.  The graph and what is instantiated from it hold it through a user object, whose end marks it
// dead (no CUDA call may be made there); the memory is given back by a later call.
struct GraphScratch {
    const lr_ctx* owner;                            // the context it was made through, NULL once that is gone
    int device;
    unsigned long long capture;                     // id of the capture, and the stream in it
    cudaStream_t stream;
    unsigned char* base;                            // guard region, counters, scratch, guard region
    size_t body;
    std::atomic<bool> dead{false};
};
struct GraphScratches {
    std::mutex mu;
    std::vector<GraphScratch*> all;
    std::atomic<int> dead{0};
};
inline GraphScratches& graph_scratches() {
    static GraphScratches* const them = new GraphScratches();      // (never destroyed: graphs may end after the library's statics)
    return *them;
}
inline void end_of_graph(void* scratch) {
    static_cast<GraphScratch*>(scratch)->dead.store(true);
    graph_scratches().dead.fetch_add(1);
}
// Gives back what ended graphs held (cudaFree waits for what still runs).
inline void free_dead_scratch() {
    GraphScratches& g = graph_scratches();
    const std::lock_guard<std::mutex> hold(g.mu);
    for (size_t i = 0; i < g.all.size();) {
        GraphScratch* b = g.all[i];
        if (!b->dead.load()) { ++i; continue; }
        cudaFree(b->base);
        delete b;
        g.all[i] = g.all.back();
        g.all.pop_back();
        g.dead.fetch_sub(1);
    }
}

}  // namespace lrgd

namespace {

// Guard regions around the context's device workspaces (per-CTA partial rows, gradient buffer, velocity, optimiser scratch):
// kGuardBytes of a fixed pattern before and after each, written once at creation.  No kernel of the library has any
// business there, so a changed byte (lr_check_guards) means an index ran out of its array.
constexpr size_t kGuardBytes = 256;
constexpr int kGuardPattern = 0xA5;

// `bytes` of device memory (rounded up to *body) that start kGuardBytes into *base, between two guard regions
cudaError_t guarded_block(const lr_ctx* c, size_t bytes, unsigned char** base, size_t* body) {
    *body = (bytes + kGuardBytes - 1) / kGuardBytes * kGuardBytes;
    *base = nullptr;
    cudaError_t e = cudaMalloc(reinterpret_cast<void**>(base), *body + 2 * kGuardBytes);
    if (e != cudaSuccess) return e;
    e = cudaMemsetAsync(*base, kGuardPattern, kGuardBytes, c->hstream);
    if (e == cudaSuccess) e = cudaMemsetAsync(*base + kGuardBytes + *body, kGuardPattern, kGuardBytes, c->hstream);
    return e;
}

template <class T>
cudaError_t guarded_alloc(lr_ctx* c, T** user, size_t bytes) {
    unsigned char* base = nullptr;
    size_t body = 0;
    const cudaError_t e = guarded_block(c, bytes, &base, &body);
    if (!base) return e;
    c->guard_bases.push_back(base);
    c->guard_sizes.push_back(body);
    *user = reinterpret_cast<T*>(base + kGuardBytes);
    return e;
}

// While one of these lives, this host thread may allocate and free though a stream is being captured (here or in another thread).
struct RelaxedCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

// A named range around a whole library call, visible on a profiler's timeline (costs nothing when no tool is attached).
struct NvtxRange {
    explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
};

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(lr_ctx* c) {
        if (cudaGetDevice(&prev) != cudaSuccess) { prev = -1; }
        if (prev == c->device) { prev = -1; return; }        // nothing to switch, nothing to switch back
        cudaError_t e = cudaSetDevice(c->device);
        if (e != cudaSuccess) { c->last_cuda = int(e); ok = false; }
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

#define LR_CK(ctx, call)                                 \
    do {                                                 \
        cudaError_t e__ = (call);                        \
        if (e__ != cudaSuccess) {                        \
            (ctx)->last_cuda = int(e__);                 \
            return LR_ERR_CUDA;                          \
        }                                                \
    } while (0)

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// SMs the launch plans of this context may use (lr_set_sm_limit)
int plan_sms(const lr_ctx* ctx) { return ctx->sm_limit > 0 ? std::min(ctx->sm_limit, ctx->sm_count) : ctx->sm_count; }

// Launches `kern`; with `dependent` set, as a programmatic dependent launch: the kernel may start while the kernel
// before it in the stream is still draining, and synchronises with it on the device (grid_dependency_wait).
template <typename... KArgs, typename... Args>
cudaError_t launch_kernel(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool dependent,
                          Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = dependent ? attr : nullptr;
    cfg.numAttrs = dependent ? 1 : 0;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, args...);
    if (dependent && (e == cudaErrorNotSupported || e == cudaErrorInvalidValue)) {
        // a driver or stream that does not take the attribute: the ordinary launch computes the same thing
        cudaGetLastError();
        cfg.attrs = nullptr;
        cfg.numAttrs = 0;
        e = cudaLaunchKernelEx(&cfg, kern, args...);
    }
    return e;
}

// Raises a kernel's dynamic shared-memory limit to `smem` on the current device, once: the limit is remembered per
// kernel instantiation (Tag) and device, so that the thousands of launches of a fit do not repeat the runtime call.
template <class Tag>
cudaError_t ensure_dynamic_smem(const void* kern, int smem) {
    constexpr int kDevices = 64;
    static int have[kDevices] = {};
    static std::mutex mu;                          // contexts on different host threads may share an instantiation
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    if (dev >= 0 && dev < kDevices && have[dev] >= smem) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && dev >= 0 && dev < kDevices) have[dev] = smem;
    return e;
}
// The tensor-map encoder is a driver entry point, resolved at run time so that the library links against the runtime only.
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t tensor_map_encoder(EncodeTiledFn* out) {
    // resolved once per process; the initialisation of a function-local static is thread-safe
    struct Resolved { EncodeTiledFn fn = nullptr; cudaError_t err = cudaSuccess; };
    static const Resolved resolved = [] {
        Resolved r;
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        r.err = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
        if (r.err == cudaSuccess && (q != cudaDriverEntryPointSuccess || !fn)) r.err = cudaErrorNotSupported;
        if (r.err == cudaSuccess) r.fn = reinterpret_cast<EncodeTiledFn>(fn);
        return r;
    }();
    *out = resolved.fn;
    if (resolved.err != cudaSuccess) return resolved.err;
    // The encoder needs a current context, which a host thread has only after a runtime call that needs one too: setting the
    // device that is current anyway (0 by default) is such a call.
    int device = 0;
    const cudaError_t e = cudaGetDevice(&device);
    return e == cudaSuccess ? cudaSetDevice(device) : e;
}

int grow(lr_ctx* ctx, void** buf, size_t* have, size_t need) {
    if (*have >= need) return LR_OK;
    if (*buf) { LR_CK(ctx, cudaFree(*buf)); *buf = nullptr; *have = 0; }
    cudaError_t e = cudaMalloc(buf, need);
    if (e != cudaSuccess) { ctx->last_cuda = int(e); *buf = nullptr; return e == cudaErrorMemoryAllocation ? LR_ERR_NOMEM : LR_ERR_CUDA; }
    *have = need;
    return LR_OK;
}

}  // namespace
