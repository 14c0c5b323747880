// C-ABI layer of the token-gate operators: routing, token rows, rows kept in 8 bits, and their gradients.
// The declarations and their contracts are in include/lrgd.h.
#include "../../include/lrgd.h"

#include <cmath>
#include <new>
#include <type_traits>

#include "lrgd_ckpt8.cuh"
#include "lrgd_ckpt8_grad.cuh"
#include "lrgd_ctx.cuh"
#include "lrgd_embed.cuh"
#include "lrgd_route.cuh"
#include "lrgd_scratch.cuh"

using namespace lrgd;

namespace {

constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1;   // positions are sorted as 32-bit numbers
constexpr int64_t kMaxLd = int64_t(1) << 40;

int check_route(int64_t T, int32_t E, int64_t ld, const lr_route_opt* o) {
    if (!o) return LR_ERR_NULL;
    if (T < 0 || T > kMaxTokens || E < 1 || E > kRouteMaxExperts || ld < E || ld > kMaxLd) return LR_ERR_SHAPE;
    if (o->k < 1 || o->k > kRouteMaxK) return LR_ERR_SHAPE;
    if (o->score != LR_SCORE_SIGMOID && o->score != LR_SCORE_SOFTMAX) return LR_ERR_VALUE;
    if (!std::isfinite(o->factor)) return LR_ERR_VALUE;
    if (o->groups < 1 || o->groups > kRouteMaxGroups || E % o->groups || o->top_groups < 1 || o->top_groups > o->groups) return LR_ERR_SHAPE;
    if (int64_t(o->k) > int64_t(E / o->groups) * o->top_groups) return LR_ERR_SHAPE;
    return LR_OK;
}

// f(std::integral_constant<int, VPL>) for the number of experts a lane holds
template <class F>
void for_vpl(int E, F&& f) {
    if (E <= 64) f(std::integral_constant<int, 2>{});
    else if (E <= 128) f(std::integral_constant<int, 4>{});
    else if (E <= 256) f(std::integral_constant<int, 8>{});
    else if (E <= 512) f(std::integral_constant<int, 16>{});
    else f(std::integral_constant<int, 32>{});
}

template <class E>
int route_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt, const float* d_bias,
               int32_t* d_ids, float* d_weights, int32_t* d_counts, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_route(T, experts, ld, opt);
    if (rc != LR_OK) return rc;
    if (T > 0 && (!d_logits || !d_ids || !d_weights)) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_bias, 4) || !aligned(d_ids, 4) || !aligned(d_weights, 4) || !aligned(d_counts, 4))
        return LR_ERR_ALIGNMENT;
    NvtxRange range("lr_route");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        if (d_counts) LR_CK(ctx, cudaMemsetAsync(d_counts, 0, size_t(experts) * 4, st));
        return LR_OK;
    }
    const int grid = even_grid(ctx, T, kRouteWarps, 8);
    Scratch scratch{};
    if (d_counts && grid > 1) {                    // the CTAs add their counts up in words of the scratch
        const int rs = gate_scratch(ctx, 0, st, &scratch);
        if (rs != LR_OK) return rs;
    }
    const RouteParams p{d_logits, ld, T, experts, opt->k, opt->groups, opt->top_groups, opt->renorm != 0, opt->factor,
                        d_bias, d_ids, d_weights, d_counts, scratch.words};
    return launched(ctx, [&] {
        for_vpl(experts, [&](auto vpl) {
            constexpr int VPL = decltype(vpl)::value;
            const bool grouped = opt->top_groups < opt->groups;    // all groups kept: no need to look at them
            if (opt->score == LR_SCORE_SOFTMAX) {
                if (grouped) k_route<E, VPL, true, true><<<grid, kRouteThreads, 0, st>>>(p);
                else k_route<E, VPL, true, false><<<grid, kRouteThreads, 0, st>>>(p);
            } else {
                if (grouped) k_route<E, VPL, false, true><<<grid, kRouteThreads, 0, st>>>(p);
                else k_route<E, VPL, false, false><<<grid, kRouteThreads, 0, st>>>(p);
            }
        });
    });
}

template <class E>
int route_grad_impl(lr_ctx* ctx, const E* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt,
                    const int32_t* d_ids, const float* d_dweights, E* d_dlogits, int64_t ld_d, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_route(T, experts, ld, opt);
    if (rc != LR_OK) return rc;
    if (ld_d < experts || ld_d > kMaxLd) return LR_ERR_SHAPE;
    if (T == 0) return LR_OK;
    if (!d_logits || !d_ids || !d_dweights || !d_dlogits) return LR_ERR_NULL;
    if (!aligned(d_logits, sizeof(E)) || !aligned(d_ids, 4) || !aligned(d_dweights, 4) || !aligned(d_dlogits, sizeof(E))) return LR_ERR_ALIGNMENT;
    NvtxRange range("lr_route_grad");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const RouteGradParams p{d_logits, ld, T, experts, opt->k, opt->renorm != 0, opt->factor, d_ids, d_dweights, d_dlogits, ld_d};
    if (opt->score == LR_SCORE_SOFTMAX && !opt->renorm) {
        const int grid = even_grid(ctx, T, kRouteWarps, 8);
        return launched(ctx, [&] {
            for_vpl(experts, [&](auto vpl) { k_route_grad_all<E, decltype(vpl)::value><<<grid, kRouteThreads, 0, st>>>(p); });
        });
    }
    int lanes = 1;
    while (lanes < opt->k) lanes *= 2;
    constexpr int kVec = 16 / int(sizeof(E));
    const int vec = experts % kVec == 0 && ld_d % kVec == 0 && aligned(d_dlogits, 16);
    const int grid = even_grid(ctx, T, kRouteWarps * (32 / lanes), 8);
    return launched(ctx, [&] {
        if (opt->score == LR_SCORE_SOFTMAX) k_route_grad_chosen<E, true><<<grid, kRouteThreads, 0, st>>>(p, lanes, vec);
        else k_route_grad_chosen<E, false><<<grid, kRouteThreads, 0, st>>>(p, lanes, vec);
    });
}

int check_tokens(int64_t T, int64_t V, int32_t n, int32_t id_bytes) {
    if (T < 0 || T > kMaxTokens || V < 1 || V >= kMaxTokens || n < 1) return LR_ERR_SHAPE;
    if (id_bytes != 4 && id_bytes != 8) return LR_ERR_VALUE;
    return LR_OK;
}

template <class E>
int embed_impl(lr_ctx* ctx, const E* d_table, int64_t ld_table, const void* d_ids, int32_t id_bytes, int64_t T, int64_t V, int32_t n,
               float scale, E* d_out, int64_t ld_out, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_tokens(T, V, n, id_bytes);
    if (rc != LR_OK) return rc;
    if (ld_table < n || ld_table > kMaxLd || ld_out < n || ld_out > kMaxLd) return LR_ERR_SHAPE;
    if (!std::isfinite(scale)) return LR_ERR_VALUE;
    if (T == 0) return LR_OK;
    if (!d_table || !d_ids || !d_out) return LR_ERR_NULL;
    if (!aligned(d_table, sizeof(E)) || !aligned(d_out, sizeof(E)) || !aligned(d_ids, id_bytes)) return LR_ERR_ALIGNMENT;
    auto fits = [&](int64_t vec) {     // vectors of `vec` elements: every row of both matrices starts on one and holds whole ones
        const size_t b = size_t(vec) * sizeof(E);
        return n % vec == 0 && ld_table % vec == 0 && ld_out % vec == 0 && aligned(d_table, b) && aligned(d_out, b);
    };
    constexpr int kVec = 16 / int(sizeof(E));
    const int width = fits(kVec) ? kVec : sizeof(E) == 2 && fits(2) ? 2 : 1;
    const int64_t pieces = (int64_t(n) + 128 * width - 1) / (128 * width);
    if (pieces > 65535) return LR_ERR_SHAPE;
    NvtxRange range("lr_embed");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const EmbedParams p{d_table, ld_table, d_ids, T, V, n, scale, d_out, ld_out, ctx->d_status + 1};
    const dim3 grid(unsigned(grid_for(ctx, T, kEmbedThreads / 32, std::max<int>(1, int(32 / pieces)))), unsigned(pieces));
    auto go = [&](auto vec) {
        constexpr int VEC = decltype(vec)::value;
        return launched(ctx, [&] {
            if (id_bytes == 8) k_embed<E, VEC, long long><<<grid, kEmbedThreads, 0, st>>>(p);
            else k_embed<E, VEC, int><<<grid, kEmbedThreads, 0, st>>>(p);
        });
    };
    if (width == kVec) return go(std::integral_constant<int, kVec>{});
    if constexpr (sizeof(E) == 2) {
        if (width == 2) return go(std::integral_constant<int, 2>{});
    }
    return go(std::integral_constant<int, 1>{});
}

template <class E>
int embed_grad_impl(lr_ctx* ctx, const void* d_ids, int32_t id_bytes, const E* d_dout, int64_t ld_dout, int64_t T, int64_t V, int32_t n,
                    float scale, int64_t padding_id, int32_t accumulate, float* d_grad, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_tokens(T, V, n, id_bytes);
    if (rc != LR_OK) return rc;
    if (ld_dout < n || ld_dout > kMaxLd) return LR_ERR_SHAPE;
    if (!std::isfinite(scale)) return LR_ERR_VALUE;
    if (!d_grad || (T > 0 && (!d_ids || !d_dout))) return LR_ERR_NULL;
    if (!aligned(d_grad, 4) || !aligned(d_dout, sizeof(E)) || !aligned(d_ids, id_bytes)) return LR_ERR_ALIGNMENT;
    const int R = T >= 4096 ? 32 : 16;             // fewer rows per chunk where there are few chunks
    const int64_t chunks = (T + R - 1) / R;
    SortParams sp{};
    for (sp.passes = 1; V >> (kSortBits * sp.passes); ++sp.passes) {}               // keys 0..V
    // Rows cleared while the sort runs, whether a token points there or not; the others are cleared after it, where none does.
    // A pass over few positions takes about 5 us, in which the memory takes kClearPerPass bytes; kClearPerToken is what it takes in the
    // time of each further position (32768 positions, two passes: 25 us).  The join takes about 8 us: kClearLate.
    constexpr int64_t kClearPerPass = 28 << 20, kClearPerToken = 1100, kClearLate = 40 << 20;
    const int64_t row_bytes = int64_t(n) * 4;
    const int64_t early = accumulate ? 0 : std::min<int64_t>(V, (sp.passes * (kClearPerPass + T * kClearPerToken)) / row_bytes);
    constexpr int kVec = 16 / int(sizeof(E));
    const bool vec = n % kVec == 0 && ld_dout % kVec == 0 && aligned(d_dout, 16) && aligned(d_grad, 16);
    const int64_t width = vec ? RunCols<E, kVec>::kSlice : RunCols<E, 1>::kSlice, slices = (int64_t(n) + width - 1) / width;
    RunParams rp{};
    // long runs have more than one chunk to themselves
    rp.joiners = chunks < 3 ? 0 : int(std::min<int64_t>(chunks / 2, std::max<int64_t>(1, plan_sms(ctx) / slices)));
    rp.clear[0] = rp.clear[1] = V;
    rp.clear_rows = int(std::max<int64_t>(1, (64 << 10) / row_bytes));                  // about 64 KB per clearing CTA
    if (!accumulate) {
        rp.clear[0] = early;
        if (rp.joiners > 0) rp.clear[1] = std::max(early, V - kClearLate / row_bytes);
    }
    const int64_t mid = (rp.clear[1] - rp.clear[0] + rp.clear_rows - 1) / rp.clear_rows, late = (V - rp.clear[1] + rp.clear_rows - 1) / rp.clear_rows;
    if (slices > 65535 || chunks * slices + mid > INT32_MAX || late > INT32_MAX / 2) return LR_ERR_SHAPE;
    NvtxRange range("lr_embed_grad");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        if (!accumulate) LR_CK(ctx, cudaMemsetAsync(d_grad, 0, size_t(V) * n * 4, st));
        return LR_OK;
    }
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    const size_t list = up(size_t(T) * 8), runs = up(size_t(chunks / 2 + 2) * 4), bits = up((size_t(V) + 31) / 32 * 4),
                 piece = size_t(2) * chunks * n * 4;
    Scratch scratch{};
    const int rs = gate_scratch(ctx, 2 * list + runs + bits + piece, st, &scratch);
    if (rs != LR_OK) return rs;
    unsigned char* w = scratch.data;
    sp.ids = d_ids;
    sp.T = unsigned(T);
    sp.V = V;
    sp.padding = padding_id;
    for (int i = 0; i < 2; ++i) sp.place[i] = reinterpret_cast<uint2*>(w + i * list);
    sp.status = ctx->d_status + 1;
    sp.long_runs = reinterpret_cast<unsigned int*>(w + 2 * list);
    sp.present = accumulate ? nullptr : reinterpret_cast<unsigned int*>(w + 2 * list + runs);
    if (early == V) sp.present = nullptr;          // all rows are cleared beside the sort: nobody asks which tokens occur
    sp.zero = d_grad;
    sp.zero_count = early * n;
    int clusters = 1;
    if (early > 0) {
        const int64_t want = (sp.zero_count / 4 + kSortThreads * kSortCtas * 4 - 1) / (kSortThreads * kSortCtas * 4);
        clusters += int(std::max<int64_t>(1, std::min<int64_t>(want, plan_sms(ctx) * 2 / kSortCtas)));
    }
    int r = launched(ctx, [&] {
        if (id_bytes == 8) k_token_sort<long long><<<clusters * kSortCtas, kSortThreads, 0, st>>>(sp);
        else k_token_sort<int><<<clusters * kSortCtas, kSortThreads, 0, st>>>(sp);
    });
    if (r != LR_OK) return r;
    rp.place = sp.place[(sp.passes - 1) & 1];
    rp.T = unsigned(T);
    rp.V = unsigned(V);
    rp.R = R;
    rp.chunks = int(chunks);
    rp.slices = int(slices);
    rp.dout = d_dout;
    rp.ld = ld_dout;
    rp.n = n;
    rp.scale = scale;
    rp.grad = d_grad;
    rp.piece = reinterpret_cast<float*>(w + 2 * list + runs + bits);
    rp.long_runs = sp.long_runs;
    rp.present = sp.present;
    auto go = [&](auto vector, auto add) -> int {
        constexpr int VEC = decltype(vector)::value;
        constexpr bool ADD = decltype(add)::value;
        LR_CK(ctx, launch_kernel(k_run_sum<E, VEC, ADD>, dim3(unsigned(chunks * slices + mid)), dim3(kRunThreads), 0, st, ctx->overlap, rp));
        ctx->launches += 1;
        if (rp.joiners == 0) return LR_OK;
        LR_CK(ctx, launch_kernel(k_run_join<E, VEC, ADD>, dim3(unsigned(rp.joiners * slices + late)), dim3(kRunThreads * kJoinGroups), 0, st,
                                 ctx->overlap, rp));
        ctx->launches += 1;
        return LR_OK;
    };
    using Vector = std::integral_constant<int, kVec>;
    using Single = std::integral_constant<int, 1>;
    if (accumulate) return vec ? go(Vector{}, std::true_type{}) : go(Single{}, std::true_type{});
    return vec ? go(Vector{}, std::false_type{}) : go(Single{}, std::false_type{});
}

int check_ckpt(int64_t T, int32_t n, int64_t ld_q) {
    if (T < 0 || T > kMaxTokens || n < 1 || n > (1 << 24) || ld_q < n || ld_q > kMaxLd) return LR_ERR_SHAPE;
    return LR_OK;
}

template <class E>
int ckpt8_move(lr_ctx* ctx, bool save, const E* x, E* back, int64_t ld, int64_t T, int32_t n, int8_t* q, int64_t ld_q, float* s, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_ckpt(T, n, ld_q);
    if (rc != LR_OK) return rc;
    if (ld < n || ld > kMaxLd) return LR_ERR_SHAPE;
    if (T == 0) return LR_OK;
    const E* rows = save ? x : back;
    if (!rows || !q || !s) return LR_ERR_NULL;
    if (!aligned(rows, sizeof(E)) || !aligned(s, 4)) return LR_ERR_ALIGNMENT;
    NvtxRange range(save ? "lr_ckpt8_save" : "lr_ckpt8_load");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int groups = (n + kCkptGroup - 1) / kCkptGroup;
    const CkptParams p{x, back, ld, q, ld_q, s, T, n, groups};
    const bool vec = n % 8 == 0 && ld % (16 / int(sizeof(E))) == 0 && ld_q % 8 == 0 && aligned(rows, 16) && aligned(q, 8);
    const int blocks = (n + kCkptCols - 1) / kCkptCols;      // of columns, at most 2^24 / 1024
    const dim3 grid(unsigned(grid_for(ctx, T, kCkptThreads / 32, std::max(1, 32 / blocks))), unsigned(blocks));
    return launched(ctx, [&] {
        if (save) {
            if (vec) k_ckpt8_save<E, true><<<grid, kCkptThreads, 0, st>>>(p);
            else k_ckpt8_save<E, false><<<grid, kCkptThreads, 0, st>>>(p);
        } else {
            if (vec) k_ckpt8_load<E, true><<<grid, kCkptThreads, 0, st>>>(p);
            else k_ckpt8_load<E, false><<<grid, kCkptThreads, 0, st>>>(p);
        }
    });
}

template <class E, bool TMA>
struct CkptGradTag {};

template <class E>
int ckpt8_grad_impl(lr_ctx* ctx, const int8_t* d_q, int64_t ld_q, const float* d_s, int64_t T, int32_t n, const E* d_dz, int64_t ld_dz,
                    int32_t C, int32_t accumulate, float* d_grad_w, float* d_grad_b, void* stream) {
    if (!ctx) return LR_ERR_NULL;
    const int rc = check_ckpt(T, n, ld_q);
    if (rc != LR_OK) return rc;
    if (C < 1 || C > 65536 || ld_dz < C || ld_dz > (int64_t(1) << 28)) return LR_ERR_SHAPE;
    if (!d_grad_w || (T > 0 && (!d_q || !d_s || !d_dz))) return LR_ERR_NULL;
    if (!aligned(d_s, 4) || !aligned(d_dz, sizeof(E)) || !aligned(d_grad_w, 4) || !aligned(d_grad_b, 4)) return LR_ERR_ALIGNMENT;
    NvtxRange range("lr_ckpt8_grad");
    const std::lock_guard<std::mutex> one_call(ctx->gate_mu);
    DeviceGuard g(ctx);
    if (!g.ok) return LR_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (T == 0) {
        if (!accumulate) {
            LR_CK(ctx, cudaMemsetAsync(d_grad_w, 0, size_t(C) * n * 4, st));
            if (d_grad_b) LR_CK(ctx, cudaMemsetAsync(d_grad_b, 0, size_t(C) * 4, st));
        }
        return LR_OK;
    }
    // CTAs take two groups of columns, a block of classes and a range of rows; as many ranges as fill the SMs once
    const int groups = (n + kCkptGroup - 1) / kCkptGroup, pairs = (groups + 1) / 2;
    const bool one = C == 1;
    const int cblocks = (C + kTcMaxClasses - 1) / kTcMaxClasses, cp = ((C + cblocks - 1) / cblocks + 15) / 16 * 16;
    const int64_t unit = one ? kUnitRows : kTcRows, units = (T + unit - 1) / unit;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(units, plan_sms(ctx) * (one ? kUnitCtas : 1) / (int64_t(pairs) * cblocks)));
    const int64_t rows = (units + want - 1) / want * unit, chunks = (T + rows - 1) / rows;
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    float *part_w = nullptr, *part_b = nullptr;
    if (chunks > 1) {
        const size_t wb = up(size_t(chunks) * C * n * 4);
        Scratch scratch{};
        const int rs = gate_scratch(ctx, wb + size_t(chunks) * C * 4, st, &scratch);
        if (rs != LR_OK) return rs;
        part_w = reinterpret_cast<float*>(scratch.data);
        part_b = reinterpret_cast<float*>(scratch.data + wb);
    }
    TcGradParams p{};
    p.g = CkptGradParams{d_q, ld_q, d_s, T, n, groups, d_dz, ld_dz, C, int(chunks), rows, accumulate != 0, part_w, part_b, d_grad_w, d_grad_b};
    p.cp = cp;
    p.status = ctx->d_status;
    const dim3 grid{unsigned(pairs), unsigned(chunks), unsigned(cblocks)};
    int r = LR_OK;
    if (one) {
        r = launched(ctx, [&] {
            if (ld_q % 16 == 0 && n % 16 == 0 && aligned(d_q, 16)) k_ckpt8_grad_unit<E, true><<<grid, kUnitWarps * 32, 0, st>>>(p.g);
            else k_ckpt8_grad_unit<E, false><<<grid, kUnitWarps * 32, 0, st>>>(p.g);
        });
    } else {
        const bool tma = aligned(d_q, 16) && ld_q % 16 == 0;
        CUtensorMap map{};
        if (tma) {
            EncodeTiledFn encode = nullptr;
            LR_CK(ctx, tensor_map_encoder(&encode));
            const cuuint64_t dims[2] = {cuuint64_t(n), cuuint64_t(T)}, strides[1] = {cuuint64_t(ld_q)};
            const cuuint32_t box[2] = {kCkptGroup, kTcRows}, step[2] = {1, 1};
            if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(d_q), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
                ctx->last_cuda = int(cudaErrorInvalidValue);
                return LR_ERR_CUDA;
            }
        }
        const int smem = tc_smem_bytes(cp, tma);
        auto go = [&](auto kern, auto tag) -> int {
            LR_CK(ctx, ensure_dynamic_smem<decltype(tag)>(reinterpret_cast<const void*>(kern), smem));
            return launched(ctx, [&] { kern<<<grid, kTcThreads, smem, st>>>(map, p); });
        };
        r = tma ? go(k_ckpt8_grad_tc<E, true>, CkptGradTag<E, true>{}) : go(k_ckpt8_grad_tc<E, false>, CkptGradTag<E, false>{});
    }
    if (r != LR_OK || chunks == 1) return r;
    const int64_t values = int64_t(C) * n;
    const bool vec = values % 4 == 0 && aligned(d_grad_w, 16);
    // sixteen parts and fewer are added by one thread each; more leave too few loads in flight
    auto join = [&](auto kern, int64_t units, int per_cta) -> int {
        LR_CK(ctx, launch_kernel(kern, dim3(grid_for(ctx, units + C, per_cta, 16)), dim3(kJoinThreads), 0, st, ctx->overlap, p.g));
        ctx->launches += 1;
        return LR_OK;
    };
    if (chunks > 16) return join(k_ckpt8_join<1, 32>, values, kJoinThreads / 32);
    if (vec) return join(k_ckpt8_join<4, 1>, values / 4, kJoinThreads);
    return join(k_ckpt8_join<1, 1>, values, kJoinThreads);
}

// bfloat16 is the unsigned 16-bit pattern of the interface
using u16 = unsigned short;
const u16* bf(const uint16_t* p) { return reinterpret_cast<const u16*>(p); }
u16* bf(uint16_t* p) { return reinterpret_cast<u16*>(p); }

}  // namespace

extern "C" {

int lr_embed(lr_ctx* ctx, const float* d_table, int64_t ld_table, const void* d_ids, int32_t id_bytes, int64_t T, int64_t V, int32_t n,
             float scale, float* d_out, int64_t ld_out, void* stream) {
    return embed_impl<float>(ctx, d_table, ld_table, d_ids, id_bytes, T, V, n, scale, d_out, ld_out, stream);
}
int lr_embed_bf16(lr_ctx* ctx, const uint16_t* d_table, int64_t ld_table, const void* d_ids, int32_t id_bytes, int64_t T, int64_t V,
                  int32_t n, float scale, uint16_t* d_out, int64_t ld_out, void* stream) {
    return embed_impl<u16>(ctx, bf(d_table), ld_table, d_ids, id_bytes, T, V, n, scale, bf(d_out), ld_out, stream);
}
int lr_embed_grad(lr_ctx* ctx, const void* d_ids, int32_t id_bytes, const float* d_dout, int64_t ld_dout, int64_t T, int64_t V, int32_t n,
                  float scale, int64_t padding_id, int32_t accumulate, float* d_grad, void* stream) {
    return embed_grad_impl<float>(ctx, d_ids, id_bytes, d_dout, ld_dout, T, V, n, scale, padding_id, accumulate, d_grad, stream);
}
int lr_embed_grad_bf16(lr_ctx* ctx, const void* d_ids, int32_t id_bytes, const uint16_t* d_dout, int64_t ld_dout, int64_t T, int64_t V,
                       int32_t n, float scale, int64_t padding_id, int32_t accumulate, float* d_grad, void* stream) {
    return embed_grad_impl<u16>(ctx, d_ids, id_bytes, bf(d_dout), ld_dout, T, V, n, scale, padding_id, accumulate, d_grad, stream);
}

int lr_route(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt, const float* d_bias,
             int32_t* d_ids, float* d_weights, int32_t* d_counts, void* stream) {
    return route_impl<float>(ctx, d_logits, ld, T, experts, opt, d_bias, d_ids, d_weights, d_counts, stream);
}
int lr_route_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt,
                  const float* d_bias, int32_t* d_ids, float* d_weights, int32_t* d_counts, void* stream) {
    return route_impl<u16>(ctx, bf(d_logits), ld, T, experts, opt, d_bias, d_ids, d_weights, d_counts, stream);
}
int lr_route_grad(lr_ctx* ctx, const float* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt,
                  const int32_t* d_ids, const float* d_dweights, float* d_dlogits, int64_t ld_d, void* stream) {
    return route_grad_impl<float>(ctx, d_logits, ld, T, experts, opt, d_ids, d_dweights, d_dlogits, ld_d, stream);
}
int lr_route_grad_bf16(lr_ctx* ctx, const uint16_t* d_logits, int64_t ld, int64_t T, int32_t experts, const lr_route_opt* opt,
                       const int32_t* d_ids, const float* d_dweights, uint16_t* d_dlogits, int64_t ld_d, void* stream) {
    return route_grad_impl<u16>(ctx, bf(d_logits), ld, T, experts, opt, d_ids, d_dweights, bf(d_dlogits), ld_d, stream);
}

int lr_ckpt8_save(lr_ctx* ctx, const float* d_X, int64_t ld, int64_t T, int32_t n, int8_t* d_q, int64_t ld_q, float* d_s, void* stream) {
    return ckpt8_move<float>(ctx, true, d_X, nullptr, ld, T, n, d_q, ld_q, d_s, stream);
}
int lr_ckpt8_save_bf16(lr_ctx* ctx, const uint16_t* d_X, int64_t ld, int64_t T, int32_t n, int8_t* d_q, int64_t ld_q, float* d_s,
                       void* stream) {
    return ckpt8_move<u16>(ctx, true, bf(d_X), nullptr, ld, T, n, d_q, ld_q, d_s, stream);
}
int lr_ckpt8_load(lr_ctx* ctx, const int8_t* d_q, int64_t ld_q, const float* d_s, int64_t T, int32_t n, float* d_X, int64_t ld, void* stream) {
    return ckpt8_move<float>(ctx, false, nullptr, d_X, ld, T, n, const_cast<int8_t*>(d_q), ld_q, const_cast<float*>(d_s), stream);
}
int lr_ckpt8_load_bf16(lr_ctx* ctx, const int8_t* d_q, int64_t ld_q, const float* d_s, int64_t T, int32_t n, uint16_t* d_X, int64_t ld,
                       void* stream) {
    return ckpt8_move<u16>(ctx, false, nullptr, bf(d_X), ld, T, n, const_cast<int8_t*>(d_q), ld_q, const_cast<float*>(d_s), stream);
}
int lr_ckpt8_grad(lr_ctx* ctx, const int8_t* d_q, int64_t ld_q, const float* d_s, int64_t T, int32_t n, const float* d_dz, int64_t ld_dz,
                  int32_t C, int32_t accumulate, float* d_grad_w, float* d_grad_b, void* stream) {
    return ckpt8_grad_impl<float>(ctx, d_q, ld_q, d_s, T, n, d_dz, ld_dz, C, accumulate, d_grad_w, d_grad_b, stream);
}
int lr_ckpt8_grad_bf16(lr_ctx* ctx, const int8_t* d_q, int64_t ld_q, const float* d_s, int64_t T, int32_t n, const uint16_t* d_dz,
                       int64_t ld_dz, int32_t C, int32_t accumulate, float* d_grad_w, float* d_grad_b, void* stream) {
    return ckpt8_grad_impl<u16>(ctx, d_q, ld_q, d_s, T, n, bf(d_dz), ld_dz, C, accumulate, d_grad_w, d_grad_b, stream);
}

}  // extern "C"
