// Routing of tokens to experts: the k best of a gate's E logits per token, with weights, and the gradient of the weights.
//
//   sigmoid:  p_e = 1/(1+exp(-l_e)),                 chosen by  c_e = p_e + bias_e
//   softmax:  p_e = exp(l_e)/sum_j exp(l_j),         chosen by  c_e = l_e + bias_e   (the order of p, without its rounding)
//   groups:   the experts stand in `groups` equal groups; a group is worth the sum of its two largest c (sigmoid) or its largest
//             c (softmax); the `top_groups` best groups keep their experts
//   the k largest c among the kept ones, ties to the lower index; w_i = factor * p_i / sum of the chosen p  (or factor * p_i)
//
// An expert whose logit or choice value is -inf is never chosen; where fewer than k remain, the slots hold id -1 and weight 0.
// A row with a NaN (softmax: or +inf) has ids -1 and NaN weights.
//
// The comparisons are on integers (a float's bits mapped so that their unsigned order is the float order), so the
// choice is exact given the c values.  One warp per token, expert e in lane e % 32: a row is read once, coalesced, at any alignment.
// The choice: k rounds of a warp-wide maximum over the lanes' largest values give a bound that at least k experts reach; those that
// reach it (k and a few more) move to one lane each, where every lane counts how many of the others are better than its own.  That
// leaves no round in which a lane has to search its values again.  Issue-bound: 16384 tokens, 256 experts
// in 8 groups 23.5 us (1,070 warp instructions a token; 40 us with k searches of every lane's values); the 17.8 MB alone take 2.7.
#pragma once
#include "lrgd_convert.cuh"

namespace lrgd {

constexpr int kRouteThreads = 256;
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxK = 32;
constexpr int kRouteMaxGroups = 32;

struct RouteParams {
    const void* logits;
    long long ld;
    long long T;
    int E;
    int k;
    int groups;
    int top_groups;
    int renorm;
    float factor;
    const float* bias;         // nullable
    int* ids;
    float* weights;
    int* counts;               // nullable
    unsigned int* words;       // [kRouteMaxExperts + 1] zero on entry and on exit: running counts, then the ticket
};

struct RouteGradParams {
    const void* logits;
    long long ld;
    long long T;
    int E;
    int k;
    int renorm;
    float factor;
    const int* ids;
    const float* dweights;
    void* dlogits;
    long long ld_d;
};

__device__ __forceinline__ float load_as_float(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_as_float(const unsigned short* p) { return __uint_as_float(static_cast<uint32_t>(__ldg(p)) << 16); }
__device__ __forceinline__ void store_from_float(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_from_float(unsigned short* p, float v) { *p = bf16_bits_rne(v); }

__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t u = __float_as_uint(v);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}
// The sigmoid as it is written, 1 / (1 + exp(-x)): the choice compares these values, so their rounding is part of the definition.
__device__ __forceinline__ float plain_sigmoid(float x) { return __frcp_rn(1.0f + expf(-x)); }

// Sigmoids that are only needed relative to one another: sigmoid(x) * exp(-m) = 1 / (exp(m) + exp(m - x)) with m the largest
// chosen logit, at most 0.  With m = 0 it is the sigmoid itself; where all chosen ones would underflow, their ratio is kept.
// x = -inf (no expert) gives 0.
__device__ __forceinline__ float sigmoid_shift(float x) { return fminf(warp_max(x), 0.0f); }
__device__ __forceinline__ float relative_sigmoid(float x, float m) {
    return x > -INFINITY ? 1.0f / (expf(m) + expf(m - x)) : 0.0f;
}

constexpr uint32_t kKeyLowest = 0x00800000u;        // order_key of the lowest number; -inf and what is not to be chosen are below

// VPL: experts per lane (E <= 32 * VPL).
template <class E, int VPL, bool SOFTMAX, bool GROUPED>
__global__ void __launch_bounds__(kRouteThreads) k_route(const __grid_constant__ RouteParams p) {
    __shared__ int hist[VPL * 32];
    __shared__ float row_choice[GROUPED ? kRouteWarps : 1][GROUPED ? VPL * 32 : 1];
    __shared__ unsigned long long candidate[kRouteWarps][32];       // key, then ~expert: the larger is the better one
    __shared__ unsigned int last_cta;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr uint32_t kAll = 0xffffffffu;
    if (p.counts) {
        for (int e = threadIdx.x; e < p.E; e += kRouteThreads) hist[e] = 0;
        __syncthreads();
    }
    const int group_size = p.E / p.groups;
    const uint32_t group_inverse = ((1u << 20) + group_size - 1) / group_size;   // e / group_size = e * this >> 20 for e < 1024
    float bias[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) bias[j] = p.bias && j * 32 + lane < p.E ? __ldg(p.bias + j * 32 + lane) : 0.0f;
    for (long long t = static_cast<long long>(blockIdx.x) * kRouteWarps + warp; t < p.T; t += static_cast<long long>(gridDim.x) * kRouteWarps) {
        const E* row = static_cast<const E*>(p.logits) + t * p.ld;
        uint32_t key[VPL];
        float x[VPL];
        float row_max = -INFINITY;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[j] = j * 32 + lane < p.E ? load_as_float(row + j * 32 + lane) : -INFINITY;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            bad |= SOFTMAX ? !(x[j] < INFINITY) : x[j] != x[j];
            if constexpr (SOFTMAX) row_max = fmaxf(row_max, x[j]);
            float c = fmaxf((SOFTMAX ? x[j] : plain_sigmoid(x[j])) + bias[j], -INFINITY);      // (a NaN of the bias: -inf)
            if (!SOFTMAX && x[j] == -INFINITY) c = -INFINITY;
            key[j] = order_key(c + 0.0f);                           // (-0 as +0: they are equal)
            if constexpr (GROUPED) row_choice[warp][j * 32 + lane] = c;
        }
        bad = __any_sync(kAll, bad);
        if constexpr (GROUPED) {
            __syncwarp();
            // 32 / groups lanes per group find its two largest values, then the first of them collects the others' pairs
            const int per = 32 / p.groups, g = lane / per, sub = lane - g * per;
            float v1 = -INFINITY, v2 = -INFINITY;
            if (g < p.groups) {
                const float* mine = row_choice[warp] + g * group_size;
#pragma unroll 4
                for (int i = sub; i < group_size; i += per) {
                    const float c = mine[i];
                    v2 = fmaxf(v2, fminf(v1, c));
                    v1 = fmaxf(v1, c);
                }
            }
            float a1 = v1, a2 = v2;
            for (int i = 1; i < per; ++i) {
                const float o1 = __shfl_sync(kAll, v1, (lane + i) & 31), o2 = __shfl_sync(kAll, v2, (lane + i) & 31);
                a2 = fmaxf(fmaxf(fminf(a1, o1), a2), o2);
                a1 = fmaxf(a1, o1);
            }
            // what lane h < groups holds now: the worth of group h, below kKeyLowest if it has no expert to choose
            a1 = __shfl_sync(kAll, a1, (lane * per) & 31);
            a2 = __shfl_sync(kAll, a2, (lane * per) & 31);
            const float worth = SOFTMAX || !(a2 > -INFINITY) ? a1 : a1 + a2;
            const uint32_t wkey = lane < p.groups ? order_key(worth + 0.0f) : 0u;
            int better = 0;
            for (int h = 0; h < p.groups; ++h) {
                const uint32_t o = __shfl_sync(kAll, wkey, h);
                better += o > wkey || (o == wkey && h < lane);
            }
            const uint32_t kept = __ballot_sync(kAll, lane < p.groups && better < p.top_groups);
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if (!(__funnelshift_rc(kept, 0u, (j * 32 + lane) * group_inverse >> 20) & 1u)) key[j] = 0;    // (past E: 0, -inf before)
        }
        // a bound that at least k experts reach, if there are k: the k-th largest of the lanes' maxima (equal ones count as one)
        uint32_t best = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j) best = max(best, key[j]);
        uint32_t bound = 0, left = best;
        for (int r = 0; r < p.k; ++r) {
            bound = __reduce_max_sync(kAll, left);
            if (left == bound) left = 0;
        }
        bound = max(bound, kKeyLowest);
        int found = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const bool in = key[j] >= bound;
            const uint32_t who = __ballot_sync(kAll, in);
            if (who) {
                const int at = found + __popc(who & ((1u << lane) - 1u));
                if (in && at < 32) candidate[warp][at] = static_cast<unsigned long long>(key[j]) << 32 | ~unsigned(j * 32 + lane);
                found += __popc(who);
            }
        }
        __syncwarp();
        int my_id = -1, place = lane;               // this lane's expert and where it comes in the order
        if (found <= 32) {
            const unsigned long long own = lane < found ? candidate[warp][lane] : 0ull;
            int better = 0;
            for (int i = 0; i < found; ++i) better += candidate[warp][i] > own;
            if (lane < found && better < p.k) {
                my_id = static_cast<int>(~static_cast<unsigned int>(own));
                place = better;
            }
            found = min(found, p.k);
        } else {                                    // many equal values: one expert after the other, the lowest index first
            found = p.k;
            for (int r = 0; r < p.k; ++r) {
                int slot = 0;
                best = 0;
#pragma unroll
                for (int j = 0; j < VPL; ++j)
                    if (key[j] > best) { best = key[j]; slot = j; }
                const uint32_t top = __reduce_max_sync(kAll, best);
                const unsigned int e = __reduce_min_sync(kAll, best == top ? unsigned(slot * 32 + lane) : 0xffffffffu);
                if (lane == r) my_id = int(e);
#pragma unroll
                for (int j = 0; j < VPL; ++j)
                    if (j * 32 + lane == int(e)) key[j] = 0;
            }
        }
        __syncwarp();                               // the next token's values go to the same places
        // the chosen experts stand in lanes of their own: their probabilities again from the logits
        if (bad) { my_id = -1; found = 0; }
        float w = 0.0f;
        if constexpr (SOFTMAX) {
            float total = 1.0f, shift = 0.0f;
            if (p.renorm) {                         // the sum over the row cancels: exp relative to the largest chosen logit
                const float x = my_id >= 0 ? load_as_float(row + my_id) : -INFINITY;
                shift = warp_max(x);
                w = my_id >= 0 ? expf(x - shift) : 0.0f;
                total = warp_sum(w);
            } else {
                shift = warp_max(row_max);
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < VPL; ++j) s += x[j] > -INFINITY ? expf(x[j] - shift) : 0.0f;
                total = warp_sum(s);
                w = my_id >= 0 ? expf(load_as_float(row + my_id) - shift) : 0.0f;
            }
            w = my_id >= 0 ? w / total : 0.0f;
        } else {
            const float x = my_id >= 0 ? load_as_float(row + my_id) : -INFINITY;
            w = p.renorm ? relative_sigmoid(x, sigmoid_shift(x)) : plain_sigmoid(x);
            if (p.renorm) {
                const float total = warp_sum(w);
                w = total > 0.0f ? w / total : 0.0f;   // no expert chosen: 0
            }
        }
        int* out_ids = p.ids + t * p.k;
        float* out_weights = p.weights + t * p.k;
        if (my_id >= 0) {
            out_ids[place] = my_id;
            out_weights[place] = w * p.factor;
            if (p.counts) atomicAdd(hist + my_id, 1);
        }
        if (lane >= found && lane < p.k) {          // places that no expert fills
            out_ids[lane] = -1;
            out_weights[lane] = bad ? __int_as_float(0x7fc00000) : 0.0f;
        }
    }
    if (!p.counts) return;
    __syncthreads();
    if (gridDim.x == 1) {
        for (int e = threadIdx.x; e < p.E; e += kRouteThreads) p.counts[e] = hist[e];
        return;
    }
    // integer sums: their order does not matter.  The CTA that finishes last hands the totals over and leaves the words at zero.
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads)
        if (hist[e]) atomicAdd(p.words + e, static_cast<unsigned int>(hist[e]));
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last_cta = atomicAdd(p.words + kRouteMaxExperts, 1u) == gridDim.x - 1;
    __syncthreads();
    if (last_cta) {
        __threadfence();
        for (int e = threadIdx.x; e < p.E; e += kRouteThreads) p.counts[e] = static_cast<int>(atomicExch(p.words + e, 0u));
        if (threadIdx.x == 0) p.words[kRouteMaxExperts] = 0u;
    }
}

// Gradient of the weights back to the logits.  With g_i the gradient of weight i and S the sum of the chosen p:
//   sigmoid:            dl_i = factor g_i p_i (1 - p_i);                                        0 for the others
//   sigmoid, renorm:    dl_i = factor (g_i - sum_j g_j w_j) w_i (1 - p_i),  w_i = p_i / S;      0 for the others
//   softmax, renorm:    dl_i = factor (g_i - sum_j g_j w_j) w_i;                                0 for the others
//   softmax:            dl_e = p_e (dp_e - sum_i dp_i p_i) for every expert,  dp_i = factor g_i for the chosen, else 0
// Ids outside [0, E) (a slot that found no expert) carry no gradient.
//
// Where only the chosen experts have a gradient, a warp takes 32 / L tokens, L lanes each (L: k rounded up to a power of two): the few
// steps per token would leave most lanes of a warp idle.  It clears the tokens' rows (16 bytes at a time where they allow it), then
// the lanes store their experts' values.  32768 tokens, 128 experts: 6.2 us (one token per warp: 10.4); the 20 MB alone take 3.1.
template <class E, bool SOFTMAX>
__global__ void __launch_bounds__(kRouteThreads) k_route_grad_chosen(const __grid_constant__ RouteGradParams p, int lanes, int vec) {
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1), tokens = 32 / lanes;
    const long long step = static_cast<long long>(gridDim.x) * kRouteWarps * tokens;
    auto group_sum = [&](float v) {
        for (int m = lanes >> 1; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
        return v;
    };
    auto group_max = [&](float v) {
        for (int m = lanes >> 1; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
        return v;
    };
    for (long long t0 = (static_cast<long long>(blockIdx.x) * kRouteWarps + (threadIdx.x >> 5)) * tokens; t0 < p.T; t0 += step) {
        const long long t = t0 + lane / lanes;
        const bool mine = t < p.T && sub < p.k;
        int id = mine ? __ldg(p.ids + t * p.k + sub) : -1;
        if (id >= p.E) id = -1;
        const float g = id >= 0 ? __ldg(p.dweights + t * p.k + sub) : 0.0f;
        const float x = id >= 0 ? load_as_float(static_cast<const E*>(p.logits) + t * p.ld + id) : -INFINITY;
        // the rows of this warp's tokens
        const int rows = static_cast<int>(min(static_cast<long long>(tokens), p.T - t0));
        E* out = static_cast<E*>(p.dlogits) + t0 * p.ld_d;
        if (vec) {
            const int per_row = p.E * static_cast<int>(sizeof(E)) / 16;
            for (int r = 0; r < rows; ++r) {
                uint4* q = reinterpret_cast<uint4*>(out + r * p.ld_d);
                for (int i = lane; i < per_row; i += 32) q[i] = make_uint4(0u, 0u, 0u, 0u);
            }
        } else {
            for (int r = 0; r < rows; ++r)
                for (int i = lane; i < p.E; i += 32) store_from_float(out + r * p.ld_d + i, 0.0f);
        }
        float d;
        if (SOFTMAX) {
            const float top = group_max(x);
            const float w0 = id >= 0 ? expf(x - top) : 0.0f;
            const float w = w0 / fmaxf(group_sum(w0), 1.0f);     // the largest term is 1; no chosen expert at all: 0
            d = w * (g - group_sum(g * w));
        } else {
            // 1 - p is the sigmoid of -x: taken from a p that is rounded near 1 it would lose its bits (all of them from x = 17 on)
            const float rest = plain_sigmoid(-x);
            if (p.renorm) {
                const float r = relative_sigmoid(x, fminf(group_max(x), 0.0f)), S = group_sum(r);
                const float w = S > 0.0f ? r / S : 0.0f;
                d = (g - group_sum(g * w)) * w * rest;
            } else {
                d = g * plain_sigmoid(x) * rest;
            }
        }
        __syncwarp();                               // the chosen ones replace the zeros
        if (id >= 0) store_from_float(static_cast<E*>(p.dlogits) + t * p.ld_d + id, d * p.factor);
    }
}

// Softmax without renormalisation: every expert has a gradient.  One warp per token; lane r < k holds chosen expert r.
template <class E, int VPL>
__global__ void __launch_bounds__(kRouteThreads) k_route_grad_all(const __grid_constant__ RouteGradParams p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (long long t = static_cast<long long>(blockIdx.x) * kRouteWarps + warp; t < p.T; t += static_cast<long long>(gridDim.x) * kRouteWarps) {
        const E* row = static_cast<const E*>(p.logits) + t * p.ld;
        E* out = static_cast<E*>(p.dlogits) + t * p.ld_d;
        int id = lane < p.k ? __ldg(p.ids + t * p.k + lane) : -1;
        if (id >= p.E) id = -1;
        const float g = id >= 0 ? p.factor * __ldg(p.dweights + t * p.k + lane) : 0.0f;
        const float x = id >= 0 ? load_as_float(row + id) : -INFINITY;
        float v[VPL], m = -INFINITY, s = 0.0f;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = j * 32 + lane;
            v[j] = e < p.E ? load_as_float(row + e) : -INFINITY;
            m = fmaxf(m, v[j]);
        }
        const float shift = warp_max(m);
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            v[j] = shift > -INFINITY ? expf(v[j] - shift) : 0.0f;
            s += v[j];
        }
        const float total = warp_sum(s);
        const float q = id >= 0 ? expf(x - shift) / total : 0.0f;
        const float common = warp_sum(g * q);
        const float scale = common != 0.0f ? -common / total : 0.0f;       // (an empty row: total is 0)
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = j * 32 + lane;
            if (e < p.E) store_from_float(out + e, v[j] * scale);
        }
        __syncwarp();                               // the chosen ones replace what was just written
        if (id >= 0) store_from_float(out + id, q * (g - common));
    }
}

}  // namespace lrgd
