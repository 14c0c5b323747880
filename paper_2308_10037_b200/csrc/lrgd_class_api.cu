// C-ABI layer of the losses over a vocabulary's classes: log-probabilities and their gradient, the clipped policy loss, the preference
// loss and distillation from a teacher's top logits.  The declarations and their contracts are in include/lrgd.h.
#include "../../include/lrgd.h"

#include <cmath>
#include <limits>
#include <type_traits>

#include "lrgd_class.cuh"
#include "lrgd_scratch.cuh"

using namespace lrgd;

namespace {

template <class E, int MODE, bool GRAD>
struct ClassRowsTag {};
template <class E, int MODE, bool GRAD, int J>
struct ClassShortTag {};

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;
constexpr int64_t kMaxClasses = int64_t(1) << 24;
constexpr int64_t kMaxPitch = int64_t(1) << 40;
constexpr int64_t kMaxPairs = int64_t(1) << 24;

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

double class_c64(float scale) { return double(scale) * 1.4426950408889634074; }            // scale * log2(e)
float class_c(float scale) { return float(class_c64(scale)); }
ClassScale class_scale(float scale) {
    const double c64 = class_c64(scale);
    ClassScale s{};
    s.c = s.down = float(c64);
    if (double(s.down) > c64) s.down = std::nextafter(s.down, 0.0f);
    s.rest = std::max(float(c64 - double(s.down)), std::numeric_limits<float>::denorm_min());
    return s;
}

int check_rows(int64_t T, int32_t V, int64_t ld, int32_t id_bytes, float scale) {
    if (T < 0 || T > kMaxRows || V < 1 || V > kMaxClasses || ld < V || ld > kMaxPitch) return LR_ERR_SHAPE;
    if (id_bytes != 4 && id_bytes != 8) return LR_ERR_VALUE;
    if (!(scale > 0.0f) || !std::isfinite(class_c(scale))) return LR_ERR_VALUE;
    return LR_OK;
}
bool norm_ok(float norm, float factor) { return std::isfinite(norm) && norm >= 0.0f && std::isfinite(factor); }

// Gradient rows either are the logits' own (the same address and ld) or share no element with them.
template <class E>
bool apart(const E* x, int64_t ld, const E* dx, int64_t ld_d, int64_t T, int64_t V) {
    if (T == 0) return true;
    if (x == dx) return ld == ld_d || T == 1;
    using Wide = __int128;                          // (a leading dimension may be anything up to 2^40)
    const Wide a = Wide(reinterpret_cast<uintptr_t>(x)), b = Wide(reinterpret_cast<uintptr_t>(dx)), es = sizeof(E);
    const Wide a_end = a + (Wide(T - 1) * ld + V) * es, b_end = b + (Wide(T - 1) * ld_d + V) * es;
    if (a_end <= b || b_end <= a) return true;
    if (ld != ld_d) return false;
    const Wide pitch = Wide(ld) * es, off = ((b - a) % pitch + pitch) % pitch;             // columns of one wider matrix
    return off >= V * es && off + V * es <= pitch;
}

constexpr int kShortGroups = 16;                    // 16-byte groups per lane of the short rows, at most
// Short rows: up to this many, every CTA adds up the weights for itself, beyond, a kernel before this one does (policy loss, 1000 x 200: 8.3 and
// 8.9 us; 4000 x 200: 11.1 and 10.2)
constexpr int kNormInline = 1024;

// How rows are worked on: a warp each (groups per lane: 1, 2, 4, 8 or 16), or by CTAs with rings, `cluster` to a row.
struct RowPlan {
    int lane_groups;             // 0: rings
    int cluster;
};
template <int MODE>
RowPlan plan_rows(const lr_ctx* ctx, int64_t T, int64_t V, int64_t es, bool grad, int depth) {
    const int64_t groups = V * es / 16, sms = plan_sms(ctx);
    RowPlan r{0, 1};
    if (groups <= 32 * kShortGroups) {
        for (r.lane_groups = 1; 32 * r.lane_groups < groups;) r.lane_groups *= 2;
        return r;
    }
    // Two thirds of a row have to fit into a team's ring (the rest is copied twice, and found in L2 the second time), or as many CTAs take a row
    // as there are SMs for, if rows are few.  Distillation, 2000 x 160000 bfloat16, 64 classes: 246 to 258 us, 303 with three quarters, which
    // takes eight CTAs instead of four; 4096 x 128000, 256 classes: 415, 607; 2048 x 100000 fp32, 128 classes: 290, 314 with a half.
    const int64_t stages = (groups + Ring<MODE>::kStageGroups - 1) / Ring<MODE>::kStageGroups;
    auto per_cta = [&] { return (stages + r.cluster - 1) / r.cluster; };
    while (r.cluster < kMaxCluster && ((grad && 2 * per_cta() > 3 * depth) || (r.cluster * 2 * T <= sms && r.cluster < stages))) r.cluster *= 2;
    return r;
}

// Scratch of the row kernels: sums of the CTAs, the order of the rows or parts of the sum of weights
struct RowScratch {
    size_t sums, prep, order;
    size_t bytes() const { return sums + prep + order; }
};
RowScratch row_scratch(const lr_ctx* ctx, int64_t T) {
    return {up256(size_t(ctx->sm_count) * 8 * 3 * sizeof(double)), up256(sizeof(ClassPrep)), up256(size_t(T) * sizeof(int) + 8)};
}

// Clusters of such a launch that are resident together (all CTAs have to be: rows are dealt out beforehand)
template <class Tag>
cudaError_t resident_clusters(const void* kern, const cudaLaunchConfig_t& cfg, int cluster, int* out) {
    struct Known {
        int device, cluster;
        size_t smem;
        int clusters;
    };
    static std::vector<Known> known;
    static std::mutex mu;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const std::lock_guard<std::mutex> hold(mu);
    for (const Known& k : known)
        if (k.device == device && k.cluster == cluster && k.smem == cfg.dynamicSmemBytes) {
            *out = k.clusters;
            return cudaSuccess;
        }
    e = cudaOccupancyMaxActiveClusters(out, kern, &cfg);
    if (e != cudaSuccess) return e;
    if (*out < 1) return cudaErrorNotSupported;
    try {
        known.push_back(Known{device, cluster, cfg.dynamicSmemBytes, *out});
    } catch (const std::bad_alloc&) {               // asked again the next time
    }
    return cudaSuccess;
}

template <class E, int MODE, bool GRAD>
int launch_ring(lr_ctx* ctx, ClassParams& p, const RowScratch& at, const Scratch& scratch, cudaStream_t st) {
    using Tag = ClassRowsTag<E, MODE, GRAD>;
    using R = Ring<MODE>;
    const auto kern = k_class_ring<E, MODE, GRAD>;
    const size_t smem = size_t(R::kTeams) * p.depth * R::kStageBytes + (MODE == kClassDistill ? R::kNumberWarps * class_top_bytes(p.K) : 0);
    LR_CK(ctx, ensure_dynamic_smem<Tag>(reinterpret_cast<const void*>(kern), int(smem)));
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(R::kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(p.cluster);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
    int clusters = 0;
    cfg.gridDim = dim3(unsigned(ctx->sm_count / p.cluster * p.cluster));
    LR_CK(ctx, resident_clusters<Tag>(reinterpret_cast<const void*>(kern), cfg, p.cluster, &clusters));
    clusters = int(std::min<int64_t>(p.T, std::max<int64_t>(1, int64_t(clusters) * plan_sms(ctx) / ctx->sm_count)));
    cfg.gridDim = dim3(unsigned(clusters * p.cluster));
    // With a row for every cluster, or where all rows count, the rows are looked at on the way; a few thousand are looked over by every CTA
    // (policy loss, 1000 x 32000 bfloat16: 37 us, 40 with a launch for it), more by a kernel before this one.
    const bool pick = p.T > clusters && (MODE != kClassDistill || p.weights);
    p.listed = pick && p.T <= kListedRows && p.T <= int64_t(clusters) * kListedMine;
    if (pick && !p.listed) {
        ClassPrep* out = reinterpret_cast<ClassPrep*>(scratch.data + at.sums);
        int* order = reinterpret_cast<int*>(scratch.data + at.sums + at.prep);
        const int r = launched(ctx, [&] { k_class_prep<MODE><<<1, kPrepThreads, 0, st>>>(p, order, out); });
        if (r != LR_OK) return r;
        p.prep = out;
        p.order = order;
        if (ctx->overlap) {
            attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[1].val.programmaticStreamSerializationAllowed = 1;
            cfg.numAttrs = 2;
        }
    }
    LR_CK(ctx, cudaLaunchKernelEx(&cfg, kern, p));
    ctx->launches += 1;
    return LR_OK;
}

template <class E, int MODE, bool GRAD>
int launch_short(lr_ctx* ctx, ClassParams& p, int lane_groups, const RowScratch& at, const Scratch& scratch, cudaStream_t st) {
    bool dependent = false;
    if (MODE != kClassLogp && p.norm == 0.0 && p.T > kNormInline) {
        double* part = reinterpret_cast<double*>(scratch.data + at.sums + at.prep);
        p.norm_part = part;
        p.norm_rows = std::max<int64_t>(1024, (p.T + 1023) / 1024);
        p.norm_parts = int((p.T + p.norm_rows - 1) / p.norm_rows);
        const int r = launched(ctx, [&] { k_class_norm<MODE><<<p.norm_parts, kNormThreads, 0, st>>>(p, part); });
        if (r != LR_OK) return r;
        dependent = ctx->overlap;
    }
    const size_t smem = MODE == kClassDistill ? kShortWarps * class_top_bytes(p.K) : 0;
    auto go = [&](auto groups) -> int {
        constexpr int J = decltype(groups)::value;
        if constexpr (MODE != kClassDistill && J * ClassGroup<E>::N <= 32) {
            if (p.T > int64_t(plan_sms(ctx)) * kShortWarps) {       // (both ways: see k_class_bundle)
                const dim3 grid(grid_for(ctx, p.T, kShortWarps * bundle_rows<E>(J), bundle_ctas(GRAD)));
                LR_CK(ctx, launch_kernel(k_class_bundle<E, MODE, GRAD, J>, grid, dim3(kShortWarps * 32), 0, st, dependent, p));
                ctx->launches += 1;
                return LR_OK;
            }
        }
        const dim3 grid(grid_for(ctx, p.T, kShortWarps, short_ctas(MODE, J)));
        using Tag = ClassShortTag<E, MODE, GRAD, J>;
        const auto kern = k_class_short<E, MODE, GRAD, J>;
        LR_CK(ctx, ensure_dynamic_smem<Tag>(reinterpret_cast<const void*>(kern), int(smem)));
        LR_CK(ctx, launch_kernel(kern, grid, dim3(kShortWarps * 32), smem, st, dependent, p));
        ctx->launches += 1;
        return LR_OK;
    };
    switch (lane_groups) {
        case 1: return go(std::integral_constant<int, 1>{});
        case 2: return go(std::integral_constant<int, 2>{});
        case 4: return go(std::integral_constant<int, 4>{});
        case 8: return go(std::integral_constant<int, 8>{});
        default: return go(std::integral_constant<int, kShortGroups>{});
    }
}

template <class E, int MODE, bool GRAD>
int launch_rows(lr_ctx* ctx, ClassParams& p, const RowScratch& at, const Scratch& scratch, cudaStream_t st) {
    p.cta_sum = reinterpret_cast<double*>(scratch.data);
    p.words = scratch.words;
    p.timeout = ctx->d_status;
    constexpr size_t kSmem = 224 << 10;             // of an SM, for ring and teacher's classes
    using R = Ring<MODE>;
    p.depth = R::kDepth;
    if (MODE == kClassDistill)
        while (p.depth > 1 && size_t(R::kTeams) * p.depth * R::kStageBytes + R::kNumberWarps * class_top_bytes(p.K) > kSmem) --p.depth;
    const RowPlan plan = plan_rows<MODE>(ctx, p.T, p.V, sizeof(E), GRAD, p.depth);
    p.cluster = plan.cluster;
    if (plan.lane_groups > 0) return launch_short<E, MODE, GRAD>(ctx, p, plan.lane_groups, at, scratch, st);
    return launch_ring<E, MODE, GRAD>(ctx, p, at, scratch, st);
}

template <class E>
ClassParams row_params(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_ids, int32_t id_bytes, int64_t ignore,
                       float scale) {
    ClassParams p{};
    p.x = d_logits;
    p.ld = ld;
    p.T = T;
    p.V = V;
    p.ids = d_ids;
    p.wide_ids = id_bytes == 8;
    p.ignore = ignore;
    p.scale = scale;
    p.c = class_c(scale);
    p.c64 = class_c64(scale);
    p.cs = class_scale(scale);
    p.status = ctx->d_status + 1;
    return p;
}

template <class E>
int launch_grad(lr_ctx* ctx, ClassGradParams& p, bool dependent, cudaStream_t st) {
    const int64_t groups = int64_t(p.V) * int64_t(sizeof(E)) / 16 + 1;
    const int threads = int(std::max<int64_t>(32, std::min<int64_t>(kClassGradThreads, (groups + 32 * kClassGradGroups - 1) / (32 * kClassGradGroups) * 32)));
    p.slices = int((groups + threads * kClassGradGroups - 1) / (threads * kClassGradGroups));
    LR_CK(ctx, launch_kernel(k_class_grad<E>, dim3(grid_for(ctx, p.T * p.slices, 1, 2048 / threads)), dim3(threads), 0, st, dependent && ctx->overlap, p));
    ctx->launches += 1;
    return LR_OK;
}

template <class E>
int logp_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes, int64_t ignore_id,
              float scale, float* d_logp, float* d_lse, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_rows(T, V, ld, id_bytes, scale);
    if (rc != LR_OK) return rc;
    if (T == 0) return LR_OK;
    if (!d_logits || !d_targets || !d_logp) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_targets, id_bytes) || !aligned(d_logp, 4) || !aligned(d_lse, 4)) return LR_ERR_ALIGNMENT;
    NvtxRange range("lr_logp");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    ClassParams p = row_params(ctx, d_logits, ld, T, V, d_targets, id_bytes, ignore_id, scale);
    p.logp = d_logp;
    p.lse = d_lse;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RowScratch at = row_scratch(ctx, T);
    Scratch scratch{};
    const int rs = gate_scratch(ctx, at.bytes(), st, &scratch);
    if (rs != LR_OK) return rs;
    return launch_rows<E, kClassLogp, false>(ctx, p, at, scratch, st);
}

template <class E>
int logp_grad_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes, int64_t ignore_id,
                   float scale, const float* d_lse, const float* d_dlogp, E* d_dlogits, int64_t ld_d, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_rows(T, V, ld, id_bytes, scale);
    if (rc != LR_OK) return rc;
    if (ld_d < V || ld_d > kMaxPitch) return LR_ERR_SHAPE;
    if (T == 0) return LR_OK;
    if (!d_logits || !d_targets || !d_lse || !d_dlogp || !d_dlogits) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_targets, id_bytes) || !aligned(d_lse, 4) || !aligned(d_dlogp, 4) || !aligned(d_dlogits, sizeof(E)))
        return LR_ERR_ALIGNMENT;
    if (!apart(d_logits, ld, d_dlogits, ld_d, T, V)) return LR_ERR_VALUE;
    NvtxRange range("lr_logp_grad");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    ClassGradParams p{};
    p.x = d_logits;
    p.ld = ld;
    p.T = T;
    p.V = V;
    p.ids = d_targets;
    p.wide_ids = id_bytes == 8;
    p.ignore = ignore_id;
    p.scale = scale;
    p.c = class_c(scale);
    p.c64 = class_c64(scale);
    p.lse = d_lse;
    p.g = d_dlogp;
    p.dx = d_dlogits;
    p.ld_d = ld_d;
    p.status = ctx->d_status + 1;
    return launch_grad<E>(ctx, p, false, static_cast<cudaStream_t>(stream));
}

template <class E>
int policy_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                const lr_policy_opt* opt, const float* d_advantages, const float* d_old_logp, const float* d_ref_logp, const float* d_weights,
                float* d_stats, float* d_logp, E* d_dlogits, int64_t ld_d, void* stream) {
    if (!ctx || !opt) return LR_ERR_NULL;
    const int rc = check_rows(T, V, ld, id_bytes, opt->scale);
    if (rc != LR_OK) return rc;
    if (d_dlogits && (ld_d < V || ld_d > kMaxPitch)) return LR_ERR_SHAPE;
    if (!(opt->clip_low >= 0.0f) || !(opt->clip_high >= 0.0f) || !std::isfinite(opt->kl_coef) || !norm_ok(opt->norm, opt->factor)) return LR_ERR_VALUE;
    if (!d_stats || (T > 0 && (!d_logits || !d_targets || !d_advantages))) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_targets, id_bytes) || !aligned(d_advantages, 4) || !aligned(d_old_logp, 4) ||
        !aligned(d_ref_logp, 4) || !aligned(d_weights, 4) || !aligned(d_stats, 4) || !aligned(d_logp, 4) || !aligned(d_dlogits, sizeof(E)))
        return LR_ERR_ALIGNMENT;
    if (d_dlogits && !apart(d_logits, ld, d_dlogits, ld_d, T, V)) return LR_ERR_VALUE;
    NvtxRange range("lr_policy_loss");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        LR_CK(ctx, cudaMemsetAsync(d_stats, 0, 4 * sizeof(float), st));
        return LR_OK;
    }
    ClassParams p = row_params(ctx, d_logits, ld, T, V, d_targets, id_bytes, opt->ignore_id, opt->scale);
    p.weights = d_weights;
    p.dx = d_dlogits;
    p.ld_d = ld_d;
    p.logp = d_logp;
    p.adv = d_advantages;
    p.old_logp = d_old_logp;
    p.ref_logp = d_ref_logp;
    p.ratio_low = float(1.0 - double(opt->clip_low));
    p.ratio_high = float(1.0 + double(opt->clip_high));
    p.log_low = opt->clip_low < 1.0f ? std::log1p(-double(opt->clip_low)) : -INFINITY;
    p.log_high = std::log1p(double(opt->clip_high));
    p.kl_coef = opt->kl_coef;
    p.norm = opt->norm;
    p.factor = opt->factor;
    p.out = d_stats;
    const RowScratch at = row_scratch(ctx, T);
    Scratch scratch{};
    const int rs = gate_scratch(ctx, at.bytes(), st, &scratch);
    if (rs != LR_OK) return rs;
    return d_dlogits ? launch_rows<E, kClassPolicy, true>(ctx, p, at, scratch, st) : launch_rows<E, kClassPolicy, false>(ctx, p, at, scratch, st);
}

template <class E>
int distill_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_ids, int32_t id_bytes, int32_t K,
                 const void* d_teacher, int32_t teacher_bytes, const lr_distill_opt* opt, const float* d_teacher_lse, const float* d_weights,
                 float* d_loss, float* d_row_kl, E* d_dlogits, int64_t ld_d, void* stream) {
    if (!ctx || !opt) return LR_ERR_NULL;
    const int rc = check_rows(T, V, ld, id_bytes, opt->scale);
    if (rc != LR_OK) return rc;
    if (K < 1 || K > kClassMaxTop || (d_dlogits && (ld_d < V || ld_d > kMaxPitch))) return LR_ERR_SHAPE;
    if ((teacher_bytes != 2 && teacher_bytes != 4) || !norm_ok(opt->norm, opt->factor)) return LR_ERR_VALUE;
    if (!d_loss || (T > 0 && (!d_logits || !d_ids || !d_teacher))) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_ids, id_bytes) || !aligned(d_teacher, teacher_bytes) || !aligned(d_teacher_lse, 4) ||
        !aligned(d_weights, 4) || !aligned(d_loss, 4) || !aligned(d_row_kl, 4) || !aligned(d_dlogits, sizeof(E)))
        return LR_ERR_ALIGNMENT;
    if (d_dlogits && !apart(d_logits, ld, d_dlogits, ld_d, T, V)) return LR_ERR_VALUE;
    NvtxRange range("lr_distill_loss");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        LR_CK(ctx, cudaMemsetAsync(d_loss, 0, sizeof(float), st));
        return LR_OK;
    }
    ClassParams p = row_params(ctx, d_logits, ld, T, V, d_ids, id_bytes, opt->ignore_id, opt->scale);
    p.weights = d_weights;
    p.dx = d_dlogits;
    p.ld_d = ld_d;
    p.teacher = d_teacher;
    p.teacher_half = teacher_bytes == 2;
    p.K = K;
    p.teacher_lse = d_teacher_lse;
    p.row_kl = d_row_kl;
    p.norm = opt->norm;
    p.factor = opt->factor;
    p.out = d_loss;
    if (p.norm == 0.0 && !d_weights) p.norm = double(T);
    const RowScratch at = row_scratch(ctx, T);
    Scratch scratch{};
    const int rs = gate_scratch(ctx, at.bytes(), st, &scratch);
    if (rs != LR_OK) return rs;
    return d_dlogits ? launch_rows<E, kClassDistill, true>(ctx, p, at, scratch, st) : launch_rows<E, kClassDistill, false>(ctx, p, at, scratch, st);
}

template <class E>
int pref_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes, const void* d_offsets,
              int32_t offset_bytes, int64_t pairs, const lr_pref_opt* opt, const float* d_ref_logp, const float* d_weights, float* d_loss,
              float* d_margins, float* d_seq_logp, E* d_dlogits, int64_t ld_d, void* stream) {
    if (!ctx || !opt) return LR_ERR_NULL;
    const int rc = check_rows(T, V, ld, id_bytes, opt->scale);
    if (rc != LR_OK) return rc;
    if (pairs < 0 || pairs > kMaxPairs || (d_dlogits && (ld_d < V || ld_d > kMaxPitch))) return LR_ERR_SHAPE;
    if ((offset_bytes != 4 && offset_bytes != 8) || !std::isfinite(opt->beta) || !std::isfinite(opt->margin) ||
        !(opt->smoothing >= 0.0f && opt->smoothing <= 1.0f) || !norm_ok(opt->norm, opt->factor))
        return LR_ERR_VALUE;
    if (!d_loss || (T > 0 && (!d_logits || !d_targets)) || (pairs > 0 && (!d_offsets || !d_margins))) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_targets, id_bytes) || !aligned(d_offsets, offset_bytes) || !aligned(d_ref_logp, 4) ||
        !aligned(d_weights, 4) || !aligned(d_loss, 4) || !aligned(d_margins, 4) || !aligned(d_seq_logp, 4) || !aligned(d_dlogits, sizeof(E)))
        return LR_ERR_ALIGNMENT;
    if (d_dlogits && !apart(d_logits, ld, d_dlogits, ld_d, T, V)) return LR_ERR_VALUE;
    NvtxRange range("lr_pref_loss");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (pairs == 0) {                               // no pair: nothing counts
        LR_CK(ctx, cudaMemsetAsync(d_loss, 0, sizeof(float), st));
        if (d_dlogits && T > 0) LR_CK(ctx, cudaMemset2DAsync(d_dlogits, size_t(ld_d) * sizeof(E), 0, size_t(V) * sizeof(E), size_t(T), st));
        return LR_OK;
    }
    const RowScratch at = row_scratch(ctx, T);
    const size_t rows = at.bytes(), stat = rows + up256(size_t(T) * sizeof(float2)), lp = up256(size_t(T) * 8), coef = up256(size_t(T) * 4),
                 loss = up256(size_t(pairs) * 8);
    Scratch scratch{};
    const int rs = gate_scratch(ctx, stat + lp + coef + loss, st, &scratch);
    if (rs != LR_OK) return rs;
    ClassPairParams q{};
    if (T > 0) {
        ClassParams p = row_params(ctx, d_logits, ld, T, V, d_targets, id_bytes, opt->ignore_id, opt->scale);
        p.stat = reinterpret_cast<float2*>(scratch.data + rows);
        p.logp64 = reinterpret_cast<double*>(scratch.data + stat);
        p.coef = reinterpret_cast<float*>(scratch.data + stat + lp);
        p.offsets = d_offsets;
        p.wide_offsets = offset_bytes == 8;
        p.sequences = 2 * pairs;
        const int r = launch_rows<E, kClassLogp, false>(ctx, p, at, scratch, st);
        if (r != LR_OK) return r;
    }
    q.ids = d_targets;
    q.wide_ids = id_bytes == 8;
    q.ignore = opt->ignore_id;
    q.V = V;
    q.T = T;
    q.offsets = d_offsets;
    q.wide_offsets = offset_bytes == 8;
    q.P = pairs;
    q.ref = d_ref_logp;
    q.weights = d_weights;
    q.beta = opt->beta;
    q.margin = opt->margin;
    q.smoothing = opt->smoothing;
    q.norm = opt->norm;
    q.factor = opt->factor;
    q.average = opt->average != 0;
    q.logp64 = reinterpret_cast<const double*>(scratch.data + stat);
    q.coef = reinterpret_cast<float*>(scratch.data + stat + lp);
    q.loss = d_loss;
    q.h = d_margins;
    q.seq_logp = d_seq_logp;
    q.pair_loss = reinterpret_cast<double*>(scratch.data + stat + lp + coef);
    q.words = scratch.words;
    q.status = ctx->d_status + 1;
    LR_CK(ctx, launch_kernel(k_class_pair, dim3(grid_for(ctx, pairs, 1, 8)), dim3(kPairThreads), 0, st, ctx->overlap && T > 0, q));
    ctx->launches += 1;
    if (!d_dlogits || T == 0) return LR_OK;
    ClassGradParams d{};
    d.x = d_logits;
    d.ld = ld;
    d.T = T;
    d.V = V;
    d.ids = d_targets;
    d.wide_ids = id_bytes == 8;
    d.ignore = opt->ignore_id;
    d.scale = opt->scale;
    d.c = class_c(opt->scale);
    d.c64 = class_c64(opt->scale);
    d.stat = reinterpret_cast<const float2*>(scratch.data + rows);
    d.g = q.coef;
    d.dx = d_dlogits;
    d.ld_d = ld_d;
    d.backwards = 1;
    return launch_grad<E>(ctx, d, true, st);
}

// bfloat16 is the unsigned 16-bit pattern of the interface
using u16 = unsigned short;
const u16* bf(const uint16_t* p) { return reinterpret_cast<const u16*>(p); }
u16* bf(uint16_t* p) { return reinterpret_cast<u16*>(p); }

}  // namespace

extern "C" {

int lr_logp(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes, int64_t ignore_id,
            float scale, float* d_logp, float* d_lse, void* stream) {
    return logp_impl<float>(ctx, d_logits, ld, T, V, d_targets, id_bytes, ignore_id, scale, d_logp, d_lse, stream);
}
int lr_logp_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                 int64_t ignore_id, float scale, float* d_logp, float* d_lse, void* stream) {
    return logp_impl<u16>(ctx, bf(d_logits), ld, T, V, d_targets, id_bytes, ignore_id, scale, d_logp, d_lse, stream);
}
int lr_logp_grad(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                 int64_t ignore_id, float scale, const float* d_lse, const float* d_dlogp, float* d_dlogits, int64_t ld_d, void* stream) {
    return logp_grad_impl<float>(ctx, d_logits, ld, T, V, d_targets, id_bytes, ignore_id, scale, d_lse, d_dlogp, d_dlogits, ld_d, stream);
}
int lr_logp_grad_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                      int64_t ignore_id, float scale, const float* d_lse, const float* d_dlogp, uint16_t* d_dlogits, int64_t ld_d, void* stream) {
    return logp_grad_impl<u16>(ctx, bf(d_logits), ld, T, V, d_targets, id_bytes, ignore_id, scale, d_lse, d_dlogp, bf(d_dlogits), ld_d, stream);
}
int lr_policy_loss(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                   const lr_policy_opt* opt, const float* d_advantages, const float* d_old_logp, const float* d_ref_logp,
                   const float* d_weights, float* d_stats, float* d_logp, float* d_dlogits, int64_t ld_d, void* stream) {
    return policy_impl<float>(ctx, d_logits, ld, T, V, d_targets, id_bytes, opt, d_advantages, d_old_logp, d_ref_logp, d_weights, d_stats, d_logp,
                              d_dlogits, ld_d, stream);
}
int lr_policy_loss_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                        const lr_policy_opt* opt, const float* d_advantages, const float* d_old_logp, const float* d_ref_logp,
                        const float* d_weights, float* d_stats, float* d_logp, uint16_t* d_dlogits, int64_t ld_d, void* stream) {
    return policy_impl<u16>(ctx, bf(d_logits), ld, T, V, d_targets, id_bytes, opt, d_advantages, d_old_logp, d_ref_logp, d_weights, d_stats, d_logp,
                            bf(d_dlogits), ld_d, stream);
}
int lr_pref_loss(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                 const void* d_offsets, int32_t offset_bytes, int64_t pairs, const lr_pref_opt* opt, const float* d_ref_logp,
                 const float* d_weights, float* d_loss, float* d_margins, float* d_seq_logp, float* d_dlogits, int64_t ld_d, void* stream) {
    return pref_impl<float>(ctx, d_logits, ld, T, V, d_targets, id_bytes, d_offsets, offset_bytes, pairs, opt, d_ref_logp, d_weights, d_loss,
                            d_margins, d_seq_logp, d_dlogits, ld_d, stream);
}
int lr_pref_loss_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_targets, int32_t id_bytes,
                      const void* d_offsets, int32_t offset_bytes, int64_t pairs, const lr_pref_opt* opt, const float* d_ref_logp,
                      const float* d_weights, float* d_loss, float* d_margins, float* d_seq_logp, uint16_t* d_dlogits, int64_t ld_d, void* stream) {
    return pref_impl<u16>(ctx, bf(d_logits), ld, T, V, d_targets, id_bytes, d_offsets, offset_bytes, pairs, opt, d_ref_logp, d_weights, d_loss,
                          d_margins, d_seq_logp, bf(d_dlogits), ld_d, stream);
}
int lr_distill_loss(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_ids, int32_t id_bytes, int32_t K,
                    const void* d_teacher, int32_t teacher_bytes, const lr_distill_opt* opt, const float* d_teacher_lse, const float* d_weights,
                    float* d_loss, float* d_row_kl, float* d_dlogits, int64_t ld_d, void* stream) {
    return distill_impl<float>(ctx, d_logits, ld, T, V, d_ids, id_bytes, K, d_teacher, teacher_bytes, opt, d_teacher_lse, d_weights, d_loss,
                               d_row_kl, d_dlogits, ld_d, stream);
}
int lr_distill_loss_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t V, const void* d_ids, int32_t id_bytes, int32_t K,
                         const void* d_teacher, int32_t teacher_bytes, const lr_distill_opt* opt, const float* d_teacher_lse,
                         const float* d_weights, float* d_loss, float* d_row_kl, uint16_t* d_dlogits, int64_t ld_d, void* stream) {
    return distill_impl<u16>(ctx, bf(d_logits), ld, T, V, d_ids, id_bytes, K, d_teacher, teacher_bytes, opt, d_teacher_lse, d_weights, d_loss,
                             d_row_kl, bf(d_dlogits), ld_d, stream);
}

}  // extern "C"
