// Losses over a vocabulary's classes: rows x of V logits, l = scale * x, lse = log sum_v exp(l_v), p_v = exp(l_v - lse).
//
//   log-probability   lp = l_y - lse for the row's target y;   d lp / d x_v = scale * ([v = y] - p_v)
//   policy loss       r = exp(lp - old);  -min(r A, clip(r) A) + kl_coef * (exp(ref - lp) - (ref - lp) - 1)
//   preference loss   S = sum of lp over a sequence (or its mean), h = beta ((S_c - R_c) - (S_r - R_r)) - margin for a pair of
//                     sequences;  -(1 - smoothing) log sigmoid(h) - smoothing log sigmoid(-h)
//   distillation      q_k over K of the classes from a teacher's logits;  sum_k q_k (log q_k - lp_k)
//
// Everything needs a row's largest logit and the sum of its exponentials, and the gradients read the row again.  Exponentials are powers of
// two: with c = scale * log2(e) rounded to fp32 once, every term is 2^(fma(x, c, -m)), m = fl(c * largest x); lse = ln 2 * (m + log2 s)
// with the same m, so that the rounding of m cancels.  The gradient forms the same terms again and multiplies them by -g / s: the
// probabilities of a row add up to one.  Row sums are fp32 in trees of a thread's own terms, the few numbers of a row fp64.
#pragma once
#include <cmath>

#include "lrgd_embed.cuh"

namespace lrgd {

constexpr int kClassThreads = 512;
constexpr int kClassMaxTop = 1024;                  // classes of a teacher per row, at most
constexpr int kClassChunks = 8192;                  // pieces of work with a sum of their own, at most
constexpr double kLn2 = 0.693147180559945309417232121458;

enum ClassMode { kClassLogp = 0, kClassPolicy = 1, kClassDistill = 2 };

struct ClassParams {
    const void* x;
    long long ld;
    long long T;
    int V;
    const void* ids;             // targets [T]; distillation: the teacher's classes [T][K]
    int wide_ids;
    long long ignore;
    float c;                     // scale * log2(e)
    float scale;
    const float* weights;        // nullable [T]
    void* dx;
    long long ld_d;
    int* status;
    // log-probabilities
    float* logp;
    float* lse;
    // what the preference loss keeps of a row: m and s, lp in fp64; rows outside [offsets[0], offsets[count]) do not count
    float2* stat;
    double* logp64;
    float* coef;
    const void* offsets;
    int wide_offsets;
    long long offset_count;
    // policy
    const float* adv;
    const float* old_logp;
    const float* ref_logp;
    double ratio_low, ratio_high, kl_coef;
    // distillation
    const void* teacher;
    int teacher_half;            // bfloat16
    int K;
    const float* teacher_lse;
    float* row_kl;
    // sums
    double norm;                 // 0: the sum of the weights of the rows that count, from norm_part
    double factor;
    const double* norm_part;
    int norm_parts;
    long long chunk_rows;
    int chunks;
    double* chunk_sum;           // [chunks][3]
    unsigned int* words;         // [0] CTAs that are done
    float* out;                  // [4] policy, [1] distillation
};

__device__ __forceinline__ long long load_any_id(const void* ids, int wide, long long i) {
    return wide ? load_id<long long>(ids, i) : static_cast<long long>(load_id<int>(ids, i));
}
__device__ __forceinline__ float exp2_fast(float v) {               // 2^v, relative error below 2^-22, subnormal results are 0
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// 16 bytes of a row
template <class E>
struct ClassGroup {
    static constexpr int N = 16 / int(sizeof(E));
    static __device__ __forceinline__ void widen(const uint4& w, float (&v)[N]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 4) {
                v[i] = __uint_as_float(u[i]);
            } else {
                v[2 * i] = __uint_as_float(u[i] << 16);
                v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float (&v)[N]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 4) u[i] = __float_as_uint(v[i]);
            else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};

// A row as `head` elements, `groups` groups of 16 bytes that start on 16 bytes, and a tail
template <class E>
struct ClassRow {
    const E* x;
    E* dx;
    int head, groups, edges;
    bool wide_store;             // the groups of dx start on 16 bytes too
    __device__ __forceinline__ ClassRow(const void* base, long long ld, void* dbase, long long ld_d, long long t, int V) {
        constexpr int N = ClassGroup<E>::N;
        x = static_cast<const E*>(base) + t * ld;
        dx = dbase ? static_cast<E*>(dbase) + t * ld_d : nullptr;
        const int off = int(reinterpret_cast<uintptr_t>(x) & 15) / int(sizeof(E));
        head = min((N - off) % N, V);
        groups = (V - head) / N;
        edges = V - groups * N;
        wide_store = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15) == 0;
    }
    // element e of those outside the groups
    __device__ __forceinline__ int edge(int e) const { return e < head ? e : e + groups * ClassGroup<E>::N; }
    __device__ __forceinline__ uint4 load(int g) const { return *reinterpret_cast<const uint4*>(x + head + g * ClassGroup<E>::N); }
    __device__ __forceinline__ void store(int g, const float (&v)[ClassGroup<E>::N]) const {
        constexpr int N = ClassGroup<E>::N;
        E* at = dx + head + g * N;
        if (wide_store) {
            *reinterpret_cast<uint4*>(at) = ClassGroup<E>::narrow(v);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) store_from_float(at + i, v[i]);
        }
    }
};

// The running maximum and sum of a part of a row: s = sum of 2^(fma(x, c, -m)), m = fl(c * largest), m = -inf before the first finite x
struct ClassSum {
    float top = -INFINITY, m = -INFINITY, s = 0.0f;
    template <int N>
    __device__ __forceinline__ void add(const float (&v)[N], float c) {
        float t = top;
#pragma unroll
        for (int i = 0; i < N; ++i) t = fmaxf(t, v[i]);
        if (t > top) {
            const float next = t * c;
            s *= exp2_fast(m - next);
            top = t;
            m = next;
        }
        if (t == -INFINITY) {                       // nothing finite yet; a NaN has to be seen all the same
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (v[i] != v[i]) s = v[i];
            return;
        }
        float part = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) part += exp2_fast(fmaf(v[i], c, -m));
        s += part;
    }
    __device__ __forceinline__ void add(float v, float c) {
        const float one[1] = {v};
        add(one, c);
    }
    __device__ __forceinline__ void join(float top2, float m2, float s2) {
        if (top2 > top) {
            s = (s == 0.0f ? 0.0f : s * exp2_fast(m - m2)) + s2;
            top = top2;
            m = m2;
        } else if (s2 != 0.0f) {
            s += top2 == top ? s2 : s2 * exp2_fast(m2 - m);
        }
    }
};

// The sum over a warp, then over the CTA: every thread gets the same bits.  One barrier; `slot` is not used again before the next one.
__device__ __forceinline__ void class_sum_cta(ClassSum& a, float (*slot)[3]) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        const float t = __shfl_down_sync(0xffffffffu, a.top, d), m = __shfl_down_sync(0xffffffffu, a.m, d),
                    s = __shfl_down_sync(0xffffffffu, a.s, d);
        a.join(t, m, s);
    }
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
        slot[warp][0] = a.top;
        slot[warp][1] = a.m;
        slot[warp][2] = a.s;
    }
    __syncthreads();
    a = ClassSum{};
    for (int w = 0; w < warps; ++w) a.join(slot[w][0], slot[w][1], slot[w][2]);
    if (a.top == -INFINITY) a.m = 0.0f;             // no finite logit: s is 0 (or NaN)
}

// Whether a row counts, with its target and weight
__device__ __forceinline__ bool class_counts(const ClassParams& p, long long t, int mode, long long* target, float* weight) {
    *weight = p.weights ? __ldg(p.weights + t) : 1.0f;
    bool live = *weight != 0.0f;                    // (a NaN counts)
    *target = 0;
    if (mode != kClassDistill) {
        *target = load_any_id(p.ids, p.wide_ids, t);
        live = live && *target != p.ignore;
        if (live && (*target < 0 || *target >= p.V)) {
            live = false;
            atomicExch(p.status, -4);               // LR_ERR_VALUE: a target outside the classes
        }
    }
    return live;
}

constexpr int kNormThreads = 256;
constexpr int kNormRows = 4096;                     // rows of a part

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// norm_part[b] = sum of the weights of rows that count among rows b * kNormRows ...
template <int MODE>
__global__ void __launch_bounds__(kNormThreads) k_class_norm(const __grid_constant__ ClassParams p, double* part) {
    __shared__ double warp_part[kNormThreads / 32];
    grid_dependency_release();
    const long long first = static_cast<long long>(blockIdx.x) * kNormRows, last = min(first + kNormRows, p.T);
    double sum = 0.0;
    for (long long t = first + threadIdx.x; t < last; t += kNormThreads) {
        long long target;
        float w;
        if (class_counts(p, t, MODE, &target, &w)) sum += w;
    }
    sum = warp_sum64(sum);
    if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < kNormThreads / 32; ++w) sum += warp_part[w];
        part[blockIdx.x] = sum;
    }
}

// 1 / norm, 0 where nothing counts
__device__ __forceinline__ double class_inv_norm(const ClassParams& p) {
    double n = p.norm;
    if (n == 0.0)
        for (int i = 0; i < p.norm_parts; ++i) n += __ldcg(p.norm_part + i);
    return n == 0.0 ? 0.0 : 1.0 / n;
}

// A row's numbers, from its statistics: lp and, for the gradient, k (what the terms 2^(..) are multiplied by) and at (the value at the target)
struct ClassNumbers {
    float k, at;
    double sums[3];
};
__device__ __forceinline__ double class_lse2(float m, float s) { return static_cast<double>(m) + log2(static_cast<double>(s)); }

// lp of the target whose logit is xy; above 0 it is rounding
__device__ __forceinline__ double class_logp(const ClassParams& p, float xy, float m, float s) {
    const double lp = kLn2 * (static_cast<double>(xy) * p.c - class_lse2(m, s));
    return lp > 0.0 ? 0.0 : lp;
}

__device__ __forceinline__ ClassNumbers class_policy_row(const ClassParams& p, long long t, float w, float xy, float m, float s, double inv) {
    ClassNumbers r;
    const double lp = class_logp(p, xy, m, s);
    if (p.logp) p.logp[t] = static_cast<float>(lp);
    const double a = __ldg(p.adv + t), ratio = p.old_logp ? exp(lp - __ldg(p.old_logp + t)) : 1.0;
    const double held = fmin(fmax(ratio, p.ratio_low), p.ratio_high);
    const bool clipped = ratio * a > held * a;
    double g = clipped ? 0.0 : -ratio * a, kl = 0.0;
    if (p.ref_logp) {
        const double d = __ldg(p.ref_logp + t) - lp, e = expm1(d);
        kl = e - d;
        g -= p.kl_coef * e;
    }
    r.sums[0] = -w * (clipped ? held : ratio) * a;
    r.sums[1] = w * kl;
    r.sums[2] = clipped ? w : 0.0;
    g *= w * inv * p.factor * p.scale;
    r.k = static_cast<float>(-g / s);
    r.at = static_cast<float>(-g * expm1(lp));
    return r;
}

// The teacher's side of a row, by one warp: top.q (weights of its classes, those of equal classes not yet added up), top.x (the student's
// logits there), top.id (-1: absent).  Returns Q = sum of q and, per lane, the part of sum q * log2(q) - q * c * x that is its own.
struct ClassTop {
    float q[kClassMaxTop];
    float x[kClassMaxTop];
    int id[kClassMaxTop];
};
template <class E>
__device__ __forceinline__ void class_top_load(const ClassParams& p, long long t, const E* row, ClassTop& top, float& largest) {
    const int lane = threadIdx.x & 31;
    largest = -INFINITY;
    for (int k = lane; k < p.K; k += 32) {
        const long long at = t * p.K + k;
        long long id = load_any_id(p.ids, p.wide_ids, at);
        const float v = p.teacher_half ? load_local(static_cast<const unsigned short*>(p.teacher) + at) : static_cast<const float*>(p.teacher)[at];
        if (id < 0 || id >= p.V) {
            if (id != p.ignore) atomicExch(p.status, -4);
            id = -1;
        }
        if (v == -INFINITY) id = -1;
        top.id[k] = static_cast<int>(id);
        top.q[k] = v;
        top.x[k] = id >= 0 ? load_local(row + id) : 0.0f;
        if (id >= 0) largest = fmaxf(largest, v);
    }
    largest = warp_max(largest);
}
// After it: top.q holds q
__device__ __forceinline__ double class_top_weights(const ClassParams& p, long long t, ClassTop& top, float largest, double& cross) {
    const int lane = threadIdx.x & 31;
    const double base = p.teacher_lse ? static_cast<double>(__ldg(p.teacher_lse + t)) * (static_cast<double>(p.c) / p.scale)
                                      : (largest == -INFINITY ? 0.0 : static_cast<double>(largest) * p.c);
    double sum = 0.0;
    cross = 0.0;                                    // sum of 2^a (a - c x), a = c v - base
    for (int k = lane; k < p.K; k += 32) {
        const bool here = top.id[k] >= 0;
        const double a = static_cast<double>(top.q[k]) * p.c - base;
        const double e = here ? exp2(a) : 0.0;
        sum += e;
        if (e != 0.0) cross += e * (a - static_cast<double>(top.x[k]) * p.c);
        top.q[k] = static_cast<float>(e);
    }
    sum = warp_sum64(sum);
    cross = warp_sum64(cross);
    return sum;
}

// ---- one CTA per row -----------------------------------------------------------------------------------
// Bound by HBM: a row is read once for its statistics and, while it is still in L2, once more for the gradient.
template <class E, int MODE, bool GRAD>
__global__ void __launch_bounds__(kClassThreads) k_class_rows(const __grid_constant__ ClassParams p) {
    constexpr int N = ClassGroup<E>::N;
    __shared__ float slot[2][kClassThreads / 32][3];
    __shared__ float now[2];
    __shared__ float top_sum, top_scale;
    __shared__ bool last_cta;
    __shared__ double warp_part[kClassThreads / 32][3];
    extern __shared__ __align__(16) unsigned char class_smem[];
    ClassTop& top = *reinterpret_cast<ClassTop*>(class_smem);
    const int tid = threadIdx.x, threads = blockDim.x;
    grid_dependency_wait();
    long long from = 0, to = p.T;
    if (MODE == kClassLogp && p.offsets) {
        from = load_any_id(p.offsets, p.wide_offsets, 0);
        to = load_any_id(p.offsets, p.wide_offsets, p.offset_count);
    }
    double inv = 0.0;
    if (MODE != kClassLogp && tid == 0) inv = class_inv_norm(p);
    int turn = 0;
    for (int chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        double sums[3] = {0.0, 0.0, 0.0};
        const long long first = chunk * p.chunk_rows, end = min(first + p.chunk_rows, p.T);
        for (long long t = first; t < end; ++t) {
            const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
            long long target;
            float w;
            bool live = class_counts(p, t, MODE, &target, &w);
            if (MODE == kClassLogp) live = live && t >= from && t < to;
            if (!live) {
                if (GRAD) {
                    const float zero[N] = {};
                    for (int g = tid; g < row.groups; g += threads) row.store(g, zero);
                    if (tid < row.edges) store_from_float(row.dx + row.edge(tid), 0.0f);
                }
                if (tid == 0) {
                    if (MODE == kClassDistill) {
                        if (p.row_kl) p.row_kl[t] = 0.0f;
                    } else if (p.logp) {
                        p.logp[t] = 0.0f;
                    }
                    if (MODE == kClassLogp && p.lse) p.lse[t] = 0.0f;
                    if (MODE == kClassLogp && p.stat) {
                        p.stat[t] = make_float2(0.0f, 1.0f);
                        p.logp64[t] = 0.0;
                        p.coef[t] = 0.0f;
                    }
                }
                continue;
            }
            float largest = 0.0f, xy = 0.0f;
            if (MODE == kClassDistill) {
                if (tid < 32) class_top_load(p, t, row.x, top, largest);
            } else if (tid == 0) {
                xy = load_local(row.x + target);
            }
            ClassSum sum;
            int g = tid;
            for (; g + 3 * threads < row.groups; g += 4 * threads) {
                uint4 raw[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) raw[j] = row.load(g + j * threads);
                float v[4 * N];
#pragma unroll
                for (int j = 0; j < 4; ++j) ClassGroup<E>::widen(raw[j], reinterpret_cast<float(&)[N]>(v[j * N]));
                sum.add(v, p.c);
            }
            for (; g < row.groups; g += threads) {
                float v[N];
                ClassGroup<E>::widen(row.load(g), v);
                sum.add(v, p.c);
            }
            float edge = 0.0f;
            if (tid < row.edges) {
                edge = load_local(row.x + row.edge(tid));
                sum.add(edge, p.c);
            }
            class_sum_cta(sum, slot[turn]);
            turn ^= 1;
            if (MODE == kClassLogp) {
                if (tid == 0) {
                    const double lse2 = class_lse2(sum.m, sum.s), lp = class_logp(p, xy, sum.m, sum.s);
                    if (p.logp) p.logp[t] = static_cast<float>(lp);
                    if (p.lse) p.lse[t] = static_cast<float>(kLn2 * lse2);
                    if (p.stat) {
                        p.stat[t] = make_float2(sum.m, sum.s);
                        p.logp64[t] = lp;
                        p.coef[t] = 0.0f;
                    }
                }
                continue;
            }
            if (MODE == kClassPolicy && tid == 0) {
                const ClassNumbers r = class_policy_row(p, t, w, xy, sum.m, sum.s, inv);
                now[0] = r.k;
                now[1] = r.at;
#pragma unroll
                for (int i = 0; i < 3; ++i) sums[i] += r.sums[i];
            }
            if (MODE == kClassDistill && tid < 32) {
                double cross;
                const double part = class_top_weights(p, t, top, largest, cross);
                const double one = p.teacher_lse || part == 0.0 ? 1.0 : 1.0 / part, q = part * one;      // q: the sum of the weights
                if (tid == 0) {
                    // sum q (log2 q - c x + lse2): with the teacher's own normalisation log2 q is smaller by log2(part)
                    double kl = 0.0;
                    if (part != 0.0) kl = kLn2 * (cross * one + q * (class_lse2(sum.m, sum.s) + log2(one)));
                    if (p.row_kl) p.row_kl[t] = static_cast<float>(kl);
                    sums[0] += w * kl;
                    const double gain = w * inv * p.factor * p.scale;
                    now[0] = static_cast<float>(q == 0.0 ? 0.0 : gain * q / sum.s);
                    now[1] = static_cast<float>(gain);
                    top_sum = static_cast<float>(q);
                    top_scale = static_cast<float>(one);
                }
            }
            if (!GRAD) continue;
            __syncthreads();
            const float k = now[0], m = -sum.m;
            const int where = MODE == kClassPolicy ? static_cast<int>(target) - row.head : -1;
            for (g = tid; g < row.groups; g += threads) {
                float v[N];
                ClassGroup<E>::widen(row.load(g), v);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = exp2_fast(fmaf(v[i], p.c, m)) * k;
                if (MODE == kClassPolicy && where >= g * N && where < g * N + N) {
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (where == g * N + i) v[i] = now[1];
                }
                row.store(g, v);
            }
            if (tid < row.edges) {
                const bool hit = MODE == kClassPolicy && row.edge(tid) == static_cast<int>(target);
                store_from_float(row.dx + row.edge(tid), hit ? now[1] : exp2_fast(fmaf(edge, p.c, m)) * k);
            }
            if (MODE == kClassDistill) {
                __syncthreads();                    // the classes' values replace what was just written
                const float gain = now[1], one = top_scale;
                for (int j = tid; j < p.K; j += threads) {
                    const int id = top.id[j];
                    if (id < 0) continue;
                    float q = 0.0f;                 // a class that the teacher names twice has both weights
                    for (int i = 0; i < p.K; ++i)
                        if (top.id[i] == id) q += top.q[i];
                    store_from_float(row.dx + id, fmaf(exp2_fast(fmaf(top.x[j], p.c, m)), k, -gain * (q * one)));
                }
                __syncthreads();
            }
        }
        if (MODE != kClassLogp && tid == 0)
            for (int i = 0; i < 3; ++i) p.chunk_sum[3 * static_cast<long long>(chunk) + i] = sums[i];
    }
    if (MODE == kClassLogp) return;
    // the CTA that is done last adds the chunks up, in a fixed order
    if (tid == 0) {
        __threadfence();
        last_cta = atomicAdd(p.words, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last_cta) return;
    __threadfence();
    double sums[3] = {0.0, 0.0, 0.0};
    for (int chunk = tid; chunk < p.chunks; chunk += threads)
        for (int i = 0; i < 3; ++i) sums[i] += __ldcg(p.chunk_sum + 3 * static_cast<long long>(chunk) + i);
    for (int i = 0; i < 3; ++i) {
        sums[i] = warp_sum64(sums[i]);
        if ((tid & 31) == 0) warp_part[tid >> 5][i] = sums[i];
    }
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < 3; ++i) {
            sums[i] = 0.0;
            for (int w = 0; w < threads / 32; ++w) sums[i] += warp_part[w][i];
            sums[i] *= inv;
        }
        if (MODE == kClassPolicy) {
            p.out[0] = static_cast<float>(p.factor * (sums[0] + p.kl_coef * sums[1]));
            for (int i = 0; i < 3; ++i) p.out[1 + i] = static_cast<float>(sums[i]);
        } else {
            p.out[0] = static_cast<float>(p.factor * sums[0]);
        }
        p.words[0] = 0;
    }
}

// ---- gradient of log-probabilities ---------------------------------------------------------------------
// Rows whose statistics are known: from the caller (lse, fp32) or from k_class_rows (m and s).  One read, one write.
struct ClassGradParams {
    const void* x;
    long long ld;
    long long T;
    int V;
    const void* ids;
    int wide_ids;
    long long ignore;
    float c;
    float scale;
    const float* lse;
    const float2* stat;
    const float* g;
    void* dx;
    long long ld_d;
    int* status;                 // NULL: targets outside the classes have been reported
    int slices;                  // of a row
    int slice_groups;
    int backwards;               // from the last row on: what was read last may still be in L2
};

constexpr int kClassGradThreads = 256;

template <class E>
__global__ void __launch_bounds__(kClassGradThreads) k_class_grad(const __grid_constant__ ClassGradParams p) {
    constexpr int N = ClassGroup<E>::N;
    const int tid = threadIdx.x, threads = blockDim.x;
    grid_dependency_wait();
    const long long items = p.T * p.slices;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const long long i = p.backwards ? items - 1 - item : item, t = i / p.slices;
        const int slice = static_cast<int>(i - t * p.slices);
        const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
        const long long target = load_any_id(p.ids, p.wide_ids, t);
        const float gt = p.g[t] * p.scale;
        bool live = target != p.ignore && gt != 0.0f;
        if (target != p.ignore && (target < 0 || target >= p.V)) {
            live = false;
            if (p.status && tid == 0) atomicExch(p.status, -4);
        }
        const int end = min((slice + 1) * p.slice_groups, row.groups);
        int g = slice * p.slice_groups + tid;
        const bool edges = slice == 0 && tid < row.edges;
        if (!live) {
            const float zero[N] = {};
            for (; g < end; g += threads) row.store(g, zero);
            if (edges) store_from_float(row.dx + row.edge(tid), 0.0f);
            continue;
        }
        float m, k;
        if (p.stat) {
            const float2 st = p.stat[t];
            m = -st.x;
            k = -gt / st.y;
        } else {                                    // lse in the units of c, the part below fp32 put into the factor
            const double l2 = static_cast<double>(p.lse[t]) * (static_cast<double>(p.c) / p.scale);
            m = -static_cast<float>(l2);
            k = -gt * exp2_fast(static_cast<float>(-static_cast<double>(m) - l2));
        }
        const int where = static_cast<int>(target) - row.head;
        for (; g < end; g += threads) {
            float v[N];
            ClassGroup<E>::widen(row.load(g), v);
            const bool hit = where >= g * N && where < g * N + N;
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = exp2_fast(fmaf(v[j], p.c, m)) * k;
            if (hit) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (where == g * N + j) v[j] += gt;
            }
            row.store(g, v);
        }
        if (edges) {
            const int at = row.edge(tid);
            const float v = exp2_fast(fmaf(load_local(row.x + at), p.c, m)) * k;
            store_from_float(row.dx + at, at == target ? v + gt : v);
        }
    }
}

// ---- pairs ---------------------------------------------------------------------------------------------
struct ClassPairParams {
    const void* ids;
    int wide_ids;
    long long ignore;
    int V;
    long long T;
    const void* offsets;         // [2 P + 1]
    int wide_offsets;
    long long P;
    const float* ref;            // nullable [2 P]
    const float* weights;        // nullable [P]
    double beta, margin, smoothing, norm, factor;
    int average;
    const double* logp64;
    float* coef;                 // per row, 0 where no sequence is
    float* loss;                 // [1]
    float* h;                    // [P]
    float* seq_logp;             // nullable [2 P]
    double* pair_loss;           // [P]
    unsigned int* words;
    int* status;
};

constexpr int kPairThreads = 256;

// One CTA per pair, the two sequences by half of it each; the last CTA adds the pairs up.
__global__ void __launch_bounds__(kPairThreads) k_class_pair(const __grid_constant__ ClassPairParams p) {
    __shared__ double warp_part[kPairThreads / 32][2];
    __shared__ double total[3];
    __shared__ bool last_cta;
    const int tid = threadIdx.x, warp = tid >> 5, side = tid >= kPairThreads / 2, lane = tid & (kPairThreads / 2 - 1);
    grid_dependency_wait();
    double sum = 0.0;                               // of the weights, the same in every CTA
    if (p.norm == 0.0 && p.weights)
        for (long long i = tid; i < p.P; i += kPairThreads) sum += __ldg(p.weights + i);
    sum = warp_sum64(sum);
    if ((tid & 31) == 0) warp_part[warp][0] = sum;
    __syncthreads();
    double norm = p.norm;
    if (norm == 0.0) {
        norm = p.weights ? 0.0 : static_cast<double>(p.P);
        if (p.weights)
            for (int i = 0; i < kPairThreads / 32; ++i) norm += warp_part[i][0];
    }
    const double inv = norm == 0.0 ? 0.0 : 1.0 / norm;
    for (long long pair = blockIdx.x; pair < p.P; pair += gridDim.x) {
        __syncthreads();
        const long long seq = pair + (side ? p.P : 0);
        long long a = load_any_id(p.offsets, p.wide_offsets, seq), z = load_any_id(p.offsets, p.wide_offsets, seq + 1);
        if (a < 0 || z < a || z > p.T) {            // no sequence: nothing is read
            if (lane == 0) atomicExch(p.status, -4);
            a = z = 0;
        }
        double lp = 0.0, count = 0.0;
        for (long long t = a + lane; t < z; t += kPairThreads / 2) {
            const long long id = load_any_id(p.ids, p.wide_ids, t);
            if (id == p.ignore || id < 0 || id >= p.V) continue;
            lp += p.logp64[t];
            count += 1.0;
        }
        lp = warp_sum64(lp);
        count = warp_sum64(count);
        if ((tid & 31) == 0) {
            warp_part[warp][0] = lp;
            warp_part[warp][1] = count;
        }
        __syncthreads();
        double s[2], size[2];
        for (int j = 0; j < 2; ++j) {
            s[j] = 0.0;
            size[j] = 0.0;
            for (int i = 0; i < kPairThreads / 64; ++i) {
                s[j] += warp_part[j * (kPairThreads / 64) + i][0];
                size[j] += warp_part[j * (kPairThreads / 64) + i][1];
            }
            if (!p.average || size[j] == 0.0) size[j] = 1.0;
            s[j] /= size[j];
        }
        if (tid == 0) {
            const double d = (s[0] - (p.ref ? static_cast<double>(__ldg(p.ref + pair)) : 0.0)) -
                             (s[1] - (p.ref ? static_cast<double>(__ldg(p.ref + p.P + pair)) : 0.0));
            const double h = p.beta * d - p.margin, w = p.weights ? static_cast<double>(__ldg(p.weights + pair)) : 1.0;
            // log sigmoid(h) = -softplus(-h), log sigmoid(-h) = -softplus(h)
            const double soft = log1p(exp(-fabs(h))), plus = fmax(h, 0.0) + soft, minus = fmax(-h, 0.0) + soft;
            const double right = 1.0 / (1.0 + exp(-h)), wrong = 1.0 / (1.0 + exp(h));
            const double loss = (1.0 - p.smoothing) * minus + p.smoothing * plus;
            p.pair_loss[pair] = w == 0.0 ? 0.0 : w * loss;
            p.h[pair] = static_cast<float>(h);
            if (p.seq_logp) {
                p.seq_logp[pair] = static_cast<float>(s[0]);
                p.seq_logp[p.P + pair] = static_cast<float>(s[1]);
            }
            total[0] = w == 0.0 ? 0.0 : w * inv * p.factor * p.beta * (p.smoothing * right - (1.0 - p.smoothing) * wrong);
        }
        __syncthreads();
        const float g = static_cast<float>((side ? -total[0] : total[0]) / size[side]);
        for (long long t = a + lane; t < z; t += kPairThreads / 2) p.coef[t] = g;
    }
    if (tid == 0) {
        __threadfence();
        last_cta = atomicAdd(p.words, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last_cta) return;
    __threadfence();
    sum = 0.0;
    for (long long i = tid; i < p.P; i += kPairThreads) sum += __ldcg(p.pair_loss + i);
    sum = warp_sum64(sum);
    __syncthreads();
    if ((tid & 31) == 0) warp_part[warp][0] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = 0.0;
        for (int i = 0; i < kPairThreads / 32; ++i) sum += warp_part[i][0];
        p.loss[0] = static_cast<float>(p.factor * sum * inv);
        p.words[0] = 0;
    }
}

}  // namespace lrgd
