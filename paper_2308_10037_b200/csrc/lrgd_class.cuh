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

constexpr int kClassMaxTop = 1024;                  // classes of a teacher per row, at most
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
    float* coef;                 // set to 0
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
    double norm;                 // 0: the sum of the weights of the rows that count
    double factor;
    // rows and their CTAs
    const int* order;            // the rows that count, then the others (k_class_prep); NULL: all rows, looked at one by one
    const struct ClassPrep* prep;
    int cluster;                 // CTAs per row
    int depth;                   // stages in a warp's ring
    double* cta_sum;             // [CTAs][3]
    int* timeout;                // status word of waits
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

// Two fp32 values in one 64-bit register (see f32x2_fma)
__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t f32x2_mul(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// 2^(x * c - m) of both halves
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x, uint64_t c, uint64_t minus_m) {
    float lo, hi;
    f32x2_unpack(f32x2_fma(x, c, minus_m), lo, hi);
    return f32x2_pack(exp2_fast(lo), exp2_fast(hi));
}

// 16 bytes of a row
template <class E>
struct ClassGroup {
    static constexpr int N = 16 / int(sizeof(E));
    static constexpr int P = N / 2;
    static __device__ __forceinline__ uint32_t word(const uint4& w, int i) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    // elements 2 i and 2 i + 1
    static __device__ __forceinline__ uint64_t pair(const uint4& w, int i) {
        if constexpr (sizeof(E) == 4) return f32x2_pack(__uint_as_float(word(w, 2 * i)), __uint_as_float(word(w, 2 * i + 1)));
        else return f32x2_pack(__uint_as_float(word(w, i) << 16), __uint_as_float(word(w, i) & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 narrow(const uint64_t (&v)[P]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float lo, hi;
            f32x2_unpack(v[i], lo, hi);
            if constexpr (sizeof(E) == 4) {
                u[2 * i] = __float_as_uint(lo);
                u[2 * i + 1] = __float_as_uint(hi);
            } else {
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(hi), "f"(lo));
            }
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
    // the largest of J groups, NaN left out
    template <int J>
    static __device__ __forceinline__ float largest(const uint4 (&raw)[J]) {
        if constexpr (sizeof(E) == 4) {
            float t = __uint_as_float(raw[0].x);
#pragma unroll
            for (int i = 1; i < 4 * J; ++i) t = fmaxf(t, __uint_as_float(word(raw[i / 4], i % 4)));
            return t;
        } else {
            uint32_t t = raw[0].x;
#pragma unroll
            for (int i = 1; i < 4 * J; ++i) asm("max.bf16x2 %0, %1, %2;" : "=r"(t) : "r"(t), "r"(word(raw[i / 4], i % 4)));
            return fmaxf(__uint_as_float(t << 16), __uint_as_float(t & 0xffff0000u));
        }
    }
};

__device__ __forceinline__ void store_streaming(void* at, const uint4& v) {
    asm volatile("st.global.cs.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

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
    __device__ __forceinline__ void store(int g, const uint64_t (&v)[ClassGroup<E>::P]) const {
        constexpr int N = ClassGroup<E>::N;
        E* at = dx + head + g * N;
        if (wide_store) {
            store_streaming(at, ClassGroup<E>::narrow(v));
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                float lo, hi;
                f32x2_unpack(v[i], lo, hi);
                store_from_float(at + 2 * i, lo);
                store_from_float(at + 2 * i + 1, hi);
            }
        }
    }
};

// The running maximum and sum of a part of a row: s = sum of 2^(fma(x, c, -m)), m = fl(c * largest), m = -inf before the first finite x
struct ClassSum {
    float top = -INFINITY, m = -INFINITY, s = 0.0f;
    // room for terms up to t; false where nothing finite has come yet
    __device__ __forceinline__ bool raise(float t, float c) {
        if (t > top) {
            const float next = t * c;
            s *= exp2_fast(m - next);
            top = t;
            m = next;
        }
        return top != -INFINITY;
    }
    __device__ __forceinline__ void add(float v, float c) {
        if (raise(v, c)) s += exp2_fast(fmaf(v, c, -m));
        else if (v != v) s = v;
    }
    template <class E, int J>
    __device__ __forceinline__ void add_groups(const uint4 (&raw)[J], float c) {
        using G = ClassGroup<E>;
        if (!raise(G::template largest<J>(raw), c)) {               // a NaN has to be seen all the same
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < G::P; ++i) {
                    float lo, hi;
                    f32x2_unpack(G::pair(raw[j], i), lo, hi);
                    if (lo != lo || hi != hi) s = NAN;
                }
            return;
        }
        const uint64_t c2 = f32x2_pack(c, c), m2 = f32x2_pack(-m, -m);
        uint64_t part = 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < G::P; ++i) part = f32x2_add(part, exp2_pair(G::pair(raw[j], i), c2, m2));
        float lo, hi;
        f32x2_unpack(part, lo, hi);
        s += lo + hi;
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

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A row's numbers, from its statistics: lp and, for the gradient, k (what the terms 2^(..) are multiplied by) and at (the value at the target)
struct ClassNumbers {
    float k, at;
    double sums[3];
};
// log2 of the sum.  exp2_fast drops the bits of its argument below 2^-23 or so: terms below 1/2 come out 4.9e-8 too small in the mean
// (measured over 4 M random arguments; 2.2e-8 between 1/2 and 1, the largest term is exact).  One row's lp does not show that, the sum over a
// long sequence does; in the gradient it cancels, whose numerator has the same terms.
__device__ __forceinline__ double class_lse2(float m, float s) {
    const double sum = s;
    return static_cast<double>(m) + log2(sum + 4.9e-8 * (sum - 1.0));
}

// lp of the target whose logit is xy; above 0 it is rounding
__device__ __forceinline__ double class_logp(const ClassParams& p, float xy, float m, float s) {
    const double lp = kLn2 * (static_cast<double>(xy) * p.c - class_lse2(m, s));
    return lp > 0.0 ? 0.0 : lp;
}

__device__ __forceinline__ ClassNumbers class_policy_row(const ClassParams& p, long long t, float w, float xy, float m, float s, double inv, bool write) {
    ClassNumbers r;
    const double lp = class_logp(p, xy, m, s);
    if (p.logp && write) p.logp[t] = static_cast<float>(lp);
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

// ---- which rows count ----------------------------------------------------------------------------------
// One CTA writes the numbers of the rows that count into `order`, in their order, those of the others behind them, and sums the weights.
// Rows that do not count get their zeros here (all but their gradient).  T = 8192: 3 us, beside the start of k_class_rows.
constexpr int kPrepThreads = 1024;
constexpr int kPrepItems = 8;

struct ClassPrep {
    double norm;
    int live;
};

template <int MODE>
__device__ __forceinline__ void class_dead_row(const ClassParams& p, long long t) {
    if (MODE == kClassDistill) {
        if (p.row_kl) p.row_kl[t] = 0.0f;
    } else {
        if (p.logp) p.logp[t] = 0.0f;
        if (MODE == kClassLogp && p.lse) p.lse[t] = 0.0f;
        if (MODE == kClassLogp && p.logp64) {
            p.logp64[t] = 0.0;
            p.coef[t] = 0.0f;
        }
    }
}

template <int MODE>
__global__ void __launch_bounds__(kPrepThreads) k_class_prep(const __grid_constant__ ClassParams p, int* order, ClassPrep* prep) {
    __shared__ double warp_norm[kPrepThreads / 32];
    __shared__ int warp_live[kPrepThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_release();
    long long from = 0, to = p.T;
    if (MODE == kClassLogp && p.offsets) {
        from = load_any_id(p.offsets, p.wide_offsets, 0);
        to = load_any_id(p.offsets, p.wide_offsets, p.offset_count);
    }
    double norm = 0.0;
    int before = 0;                                 // rows that count so far
    for (long long base = 0; base < p.T; base += kPrepThreads * kPrepItems) {
        const long long first = base + warp * (32 * kPrepItems) + lane;
        unsigned int mask[kPrepItems];
        int mine = 0;
#pragma unroll
        for (int j = 0; j < kPrepItems; ++j) {
            const long long t = first + 32 * j;
            bool live = false;
            if (t < p.T) {
                long long target;
                float w;
                live = class_counts(p, t, MODE, &target, &w);
                if (MODE == kClassLogp) live = live && t >= from && t < to;
                if (live) norm += w;
                else class_dead_row<MODE>(p, t);
            }
            mask[j] = __ballot_sync(0xffffffffu, live);
            mine += __popc(mask[j]);
        }
        __syncthreads();                            // the last turn's counts have been read
        if (lane == 0) warp_live[warp] = mine;
        __syncthreads();
        int at = before, all = 0;
        for (int w = 0; w < kPrepThreads / 32; ++w) {
            const int n = warp_live[w];
            if (w < warp) at += n;
            all += n;
        }
        before += all;
#pragma unroll
        for (int j = 0; j < kPrepItems; ++j) {
            const long long t = first + 32 * j;
            const int ahead = at + __popc(mask[j] & ((1u << lane) - 1));
            // of the rows up to t, t - ahead do not count: they fill `order` from its end
            if (t < p.T) order[(mask[j] >> lane & 1) ? ahead : p.T - 1 - (t - ahead)] = static_cast<int>(t);
            at += __popc(mask[j]);
        }
    }
    norm = warp_sum64(norm);
    if (lane == 0) warp_norm[warp] = norm;
    __syncthreads();
    if (threadIdx.x == 0) {
        norm = 0.0;
        for (int w = 0; w < kPrepThreads / 32; ++w) norm += warp_norm[w];
        prep->norm = norm;
        prep->live = before;
    }
}

// ---- a teacher's classes -------------------------------------------------------------------------------
// Entry j of a row belongs to thread j mod (threads of the CTA).  q is 2^(c * v - base of the entry's warp); `part` turns it into the weight.
struct ClassTop {
    int* id;                     // [K], -1: absent
    float* q;                    // [K]
    float* x;                    // [K] the student's logits
    int* table;                  // [size] the classes seen so far, -1: free
    int size;                    // a power of two, at least 2 K
    double (*warp)[3];           // [warps] base, sum of q, sum of q * (c * v - base - c * x)
    float* part;                 // [warps]
    int* twice;                  // [2] some class is named twice
};
__host__ __device__ inline int class_table_size(int K) {
    int n = 64;
    while (n < 2 * K) n *= 2;
    return n;
}
__host__ __device__ inline size_t class_top_bytes(int K, int warps) {
    return size_t(K) * 12 + size_t(class_table_size(K)) * 4 + size_t(warps) * 32 + 64;
}
__device__ __forceinline__ ClassTop class_top_at(unsigned char* at, int K, int warps) {
    ClassTop top;
    top.warp = reinterpret_cast<double(*)[3]>(at);
    at += warps * 24;
    top.part = reinterpret_cast<float*>(at);
    at += warps * 4;
    top.twice = reinterpret_cast<int*>(at);
    at += 8;
    top.size = class_table_size(K);
    top.table = reinterpret_cast<int*>(at);
    at += top.size * 4;
    top.id = reinterpret_cast<int*>(at);
    top.q = reinterpret_cast<float*>(at + 4 * K);
    top.x = reinterpret_cast<float*>(at + 8 * K);
    return top;
}
struct ClassEntry {
    long long id;
    float v;
};
__device__ __forceinline__ ClassEntry class_entry(const ClassParams& p, long long t, int j) {
    ClassEntry e{0, -INFINITY};
    if (j < p.K) {
        const long long at = t * p.K + j;
        e.id = load_any_id(p.ids, p.wide_ids, at);
        e.v = p.teacher_half ? __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const unsigned short*>(p.teacher) + at)) << 16)
                             : __ldg(static_cast<const float*>(p.teacher) + at);
    }
    return e;
}
// id in [0, V), or -1 where the entry is absent
__device__ __forceinline__ int class_entry_id(const ClassParams& p, const ClassEntry& e) {
    if (e.id < 0 || e.id >= p.V) {
        if (e.id != p.ignore) atomicExch(p.status, -4);
        return -1;
    }
    return e.v == -INFINITY ? -1 : static_cast<int>(e.id);
}
// Writes an entry down; true where its class has been seen in this row
__device__ __forceinline__ bool class_entry_put(const ClassTop& top, int j, int id, float v, float x) {
    top.id[j] = id;
    top.q[j] = v;
    top.x[j] = x;
    if (id < 0) return false;
    unsigned int at = static_cast<unsigned int>(id) * 2654435761u;
    for (at = (at >> 12) & (top.size - 1);; at = (at + 1) & (top.size - 1)) {       // ends: at most K of 2 K places are taken
        const int was = atomicCAS(top.table + at, -1, id);
        if (was == -1) return false;
        if (was == id) return true;
    }
}
// A warp's share of the row: its entries' q, their sums
__device__ __forceinline__ void class_top_warp(const ClassParams& p, long long t, const ClassTop& top, float largest) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    largest = warp_max(largest);
    const double base = p.teacher_lse ? static_cast<double>(__ldg(p.teacher_lse + t)) * (static_cast<double>(p.c) / p.scale)
                                      : (largest == -INFINITY ? 0.0 : static_cast<double>(largest) * p.c);
    double sum = 0.0, cross = 0.0;
    for (int j = threadIdx.x; j < p.K; j += blockDim.x) {
        const double a = static_cast<double>(top.q[j]) * p.c - base;
        const double e = top.id[j] >= 0 ? exp2(a) : 0.0;
        sum += e;
        if (e != 0.0) cross += e * (a - static_cast<double>(top.x[j]) * p.c);
        top.q[j] = static_cast<float>(e);
    }
    sum = warp_sum64(sum);
    cross = warp_sum64(cross);
    if (lane == 0) {
        top.warp[warp][0] = sum == 0.0 && !p.teacher_lse ? -INFINITY : base;
        top.warp[warp][1] = sum;
        top.warp[warp][2] = cross;
    }
}

// ---- rows ----------------------------------------------------------------------------------------------
// One CTA per row, or a cluster of C where there are fewer rows than SMs.  A row's 16-byte groups are dealt out to the warps in stages of
// 2 KB; every warp brings its own stages into its own ring of shared memory with bulk copies, as far ahead as the ring allows, over the ends of
// rows too.  First pass: running maximum and sum; one barrier joins the warps (one more the CTAs).  Second pass: the gradient, from the
// stages that are still in the ring, then from those that were overwritten, which come from L2 again.  A stage is given back when it has been
// read for the last time, always in the order of the copies, so the ring needs no bookkeeping beyond two counters.
constexpr int kRingThreads = 512;
constexpr int kStageGroups = 128;
constexpr int kStageBytes = kStageGroups * 16;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_store_f32(const float* local, uint32_t rank, float v) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// A warp's stages of a row
template <class E>
struct WarpRow {
    const E* x;                  // first group
    int groups;
    int stages;
    __device__ __forceinline__ void set(const ClassParams& p, long long t, int gw, int tw) {
        const ClassRow<E> row(p.x, p.ld, nullptr, 0, t, p.V);
        x = row.x + row.head;
        groups = row.groups;
        const int all = (groups + kStageGroups - 1) / kStageGroups;
        stages = all > gw ? (all - gw + tw - 1) / tw : 0;
    }
};

template <class E, int MODE, bool GRAD>
__global__ void __launch_bounds__(kRingThreads, 2) k_class_rows(const __grid_constant__ ClassParams p) {
    using G = ClassGroup<E>;
    constexpr int N = G::N;
    constexpr int J = kStageGroups / 32;            // groups of a stage per lane
    __shared__ float slot[2][kRingThreads / 32][3];
    __shared__ float cta_slot[2][kMaxCluster][4];
    __shared__ float now[2];
    __shared__ int abort_word;
    __shared__ bool last_cta;
    extern __shared__ __align__(128) unsigned char class_smem[];
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5, depth = p.depth;
    const int C = p.cluster, rank = C > 1 ? int(cluster_rank()) : 0, q = blockIdx.x / C, Q = gridDim.x / C;
    const int gw = rank * warps + warp, tw = C * warps;
    unsigned char* ring = class_smem + size_t(warp) * depth * kStageBytes;
    uint64_t* bars = reinterpret_cast<uint64_t*>(class_smem + size_t(warps) * depth * kStageBytes) + warp * depth;
    ClassTop top{};
    if (MODE == kClassDistill) {
        top = class_top_at(class_smem + size_t(warps) * depth * (kStageBytes + 8), p.K, warps);
        for (int i = tid; i < top.size; i += threads) top.table[i] = -1;
        if (tid < 2) top.twice[tid] = 0;
    }
    volatile int* abort_flag = &abort_word;
    if (tid == 0) abort_word = 0;
    if (lane == 0) {
        for (int i = 0; i < depth; ++i) mbar_init(bars + i, 1);
        fence_mbar_init();
    }
    if (C > 1) cluster_barrier();                   // (a CTA that writes into another's shared memory has to find it started)
    else __syncthreads();
    grid_dependency_wait();
    const uint64_t first_use = l2_policy_evict_first();
    const int live = p.order ? p.prep->live : int(p.T);
    const int mine = live > q ? (live - q + Q - 1) / Q : 0;
    // rows of this CTA, 64 of them known ahead: lane i holds the numbers of rows 32 * block + i and 32 * (block + 1) + i
    int block = 0, order0 = 0, order1 = 0;
    auto fetch = [&](int b) { const int k = 32 * b + lane; return p.order && k < mine ? __ldg(p.order + q + static_cast<long long>(k) * Q) : 0; };
    order0 = fetch(0);
    order1 = fetch(1);
    auto row_of = [&](int k) -> int {
        if (!p.order) return q + k * Q;
        return __shfl_sync(0xffffffffu, (k >> 5) == block ? order0 : order1, k & 31);
    };
    // copies: row and stage that come next, the ring's place and how many places are taken
    WarpRow<E> next{};
    int next_row = 0, next_stage = 0, next_uses = 0, in_slot = 0, taken = 0;
    if (mine > 0) {
        next.set(p, row_of(0), gw, tw);
        next_uses = next.stages + (GRAD ? max(0, next.stages - depth) : 0);
    }
    auto copy_ahead = [&](int row_now) {
        while (taken < depth && next_row < mine) {
            if (next_stage == next_uses) {
                if (next_row - row_now >= 30) return;
                ++next_row;
                next_stage = 0;
                if (next_row < mine) {
                    next.set(p, row_of(next_row), gw, tw);
                    next_uses = next.stages + (GRAD ? max(0, next.stages - depth) : 0);
                }
                continue;
            }
            const int stage = next_stage < next.stages ? next_stage : next_stage - next.stages;
            const int first = (stage * tw + gw) * kStageGroups, bytes = min(kStageGroups, next.groups - first) * 16;
            if (lane == 0) {
                fence_proxy_async_smem();
                mbar_arrive_expect_tx(bars + in_slot, bytes);
                bulk_copy_g2s(ring + in_slot * kStageBytes, next.x + static_cast<long long>(first) * N, bytes, bars + in_slot, first_use);
            }
            ++next_stage;
            ++taken;
            if (++in_slot == depth) in_slot = 0;
        }
    };
    int out_slot = 0, out_parity = 0, wait_slot = 0, wait_parity = 0;   // the place that is given back next; the copy that is waited for next
    bool gone = false;                              // a wait ran out: nothing is copied any more
    auto give_back = [&](int row_now) {             // what is in registers now may be overwritten
        __syncwarp();
        if (gone) return;
        --taken;
        if (++out_slot == depth) {
            out_slot = 0;
            out_parity ^= 1;
        }
        copy_ahead(row_now);
    };
    auto wait_copy = [&]() -> const unsigned char* {
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(bars + wait_slot, wait_parity, abort_flag))) gone = true;
        const unsigned char* at = ring + wait_slot * kStageBytes;
        if (++wait_slot == depth) {
            wait_slot = 0;
            wait_parity ^= 1;
        }
        return at;
    };
    copy_ahead(0);

    double inv = 0.0;                               // warp 0: 1 / norm, 0 where nothing counts
    if (MODE != kClassLogp && warp == 0) {
        double n = p.norm;
        if (n == 0.0 && p.order) n = p.prep->norm;
        if (n == 0.0 && !p.order) {                 // few rows: every CTA adds their weights up
            for (long long t = lane; t < p.T; t += 32) {
                long long target;
                float w;
                if (class_counts(p, t, MODE, &target, &w)) n += w;
            }
            n = warp_sum64(n);
        }
        inv = n == 0.0 ? 0.0 : 1.0 / n;
    }
    long long from = 0, to = p.T;
    if (MODE == kClassLogp && !p.order && p.offsets) {
        from = load_any_id(p.offsets, p.wide_offsets, 0);
        to = load_any_id(p.offsets, p.wide_offsets, p.offset_count);
    }
    double sums[3] = {0.0, 0.0, 0.0};
    int turn = 0;
    for (int k = 0; k < mine; ++k) {
        if ((k >> 5) != block) {
            ++block;
            order0 = order1;
            order1 = fetch(block + 1);
        }
        copy_ahead(k);                              // (a warp without a stage of the rows before gives nothing back)
        const long long t = row_of(k);
        const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
        WarpRow<E> own;
        own.set(p, t, gw, tw);
        long long target = 0;
        float w = 1.0f;
        bool counts = true;
        if (p.order) {
            if (p.weights) w = __ldg(p.weights + t);
            if (MODE != kClassDistill) target = load_any_id(p.ids, p.wide_ids, t);
        } else {
            counts = class_counts(p, t, MODE, &target, &w);
            if (MODE == kClassLogp) counts = counts && t >= from && t < to;
        }
        const bool edges = gw == 0 && lane < row.edges;
        float xy = 0.0f, edge = 0.0f;
        if (counts) {
            if (MODE != kClassDistill && tid == 0) xy = load_local(row.x + target);
            if (edges) edge = load_local(row.x + row.edge(lane));
        }
        float largest = -INFINITY;
        if (MODE == kClassDistill && counts) {
            bool twice = false;
            for (int j = tid; j < p.K; j += threads) {
                const ClassEntry e = class_entry(p, t, j);
                const int id = class_entry_id(p, e);
                if (id >= 0) largest = fmaxf(largest, e.v);
                twice |= class_entry_put(top, j, id, e.v, id >= 0 ? load_local(row.x + id) : 0.0f);
            }
            if (twice) top.twice[turn] = 1;
            class_top_warp(p, t, top, largest);
        }
        ClassSum sum;
        const int dropped = GRAD ? max(0, own.stages - depth) : own.stages;
        for (int i = 0; i < own.stages; ++i) {
            const int left = min(kStageGroups, own.groups - (i * tw + gw) * kStageGroups) - lane;
            const unsigned char* at = wait_copy();
            uint4 raw[J];
#pragma unroll
            for (int j = 0; j < J; ++j) raw[j] = *reinterpret_cast<const uint4*>(at + (lane + 32 * j) * 16);
            if (i < dropped) give_back(k);
            if (left > 32 * (J - 1)) {
                sum.add_groups<E, J>(raw, p.c);
            } else {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const uint4 one[1] = {raw[j]};
                    if (32 * j < left) sum.add_groups<E, 1>(one, p.c);
                }
            }
        }
        if (edges) sum.add(edge, p.c);
        class_sum_cta(sum, slot[turn]);
        bool stop = *abort_flag != 0;
        if (C > 1) {
            if (tid < C) {
                cluster_store_f32(&cta_slot[turn][rank][0], tid, sum.top);
                cluster_store_f32(&cta_slot[turn][rank][1], tid, sum.m);
                cluster_store_f32(&cta_slot[turn][rank][2], tid, sum.s);
                cluster_store_f32(&cta_slot[turn][rank][3], tid, stop ? 1.0f : 0.0f);
            }
            cluster_barrier();
            sum = ClassSum{};
            stop = false;
            for (int r = 0; r < C; ++r) {
                sum.join(cta_slot[turn][r][0], cta_slot[turn][r][1], cta_slot[turn][r][2]);
                stop = stop || cta_slot[turn][r][3] != 0.0f;
            }
        }
        if (stop) {
            gone = true;
            break;
        }
        if (sum.top == -INFINITY) sum.m = 0.0f;     // no finite logit: s is 0 (or NaN)
        if (MODE == kClassLogp) {
            if (gw == 0 && lane == 0) {
                if (counts) {
                    const double lse2 = class_lse2(sum.m, sum.s), lp = class_logp(p, xy, sum.m, sum.s);
                    if (p.logp) p.logp[t] = static_cast<float>(lp);
                    if (p.lse) p.lse[t] = static_cast<float>(kLn2 * lse2);
                    if (p.stat) {
                        p.stat[t] = make_float2(sum.m, sum.s);
                        p.logp64[t] = lp;
                        p.coef[t] = 0.0f;
                    }
                } else {
                    class_dead_row<MODE>(p, t);
                }
            }
            turn ^= 1;
            continue;
        }
        if (MODE == kClassPolicy && tid == 0) {
            if (counts) {
                const ClassNumbers r = class_policy_row(p, t, w, xy, sum.m, sum.s, inv, rank == 0);
                now[0] = r.k;
                now[1] = r.at;
#pragma unroll
                for (int i = 0; i < 3; ++i) sums[i] += r.sums[i];
            } else if (rank == 0) {
                class_dead_row<MODE>(p, t);
            }
        }
        bool twice = false;
        if (MODE == kClassDistill) {
            twice = top.twice[turn] != 0;
            if (counts && warp == 0) {
                const bool here = lane < warps;
                double base = here ? top.warp[lane][0] : -INFINITY, all = here ? top.warp[lane][1] : 0.0, cross = here ? top.warp[lane][2] : 0.0;
                double most = base;
#pragma unroll
                for (int d = 16; d >= 1; d >>= 1) most = fmax(most, __shfl_xor_sync(0xffffffffu, most, d));
                const double f = all == 0.0 ? 0.0 : exp2(base - most);
                cross = warp_sum64(all == 0.0 ? 0.0 : f * (cross + (base - most) * all));
                all = warp_sum64(f * all);
                // with the teacher's own normalisation log2 q is smaller by log2(all)
                const double one = p.teacher_lse || all == 0.0 ? 1.0 : 1.0 / all, mass = all * one;
                if (here) top.part[lane] = static_cast<float>(f * one);
                if (lane == 0) {
                    double kl = 0.0;
                    if (all != 0.0) kl = kLn2 * (cross * one + mass * (class_lse2(sum.m, sum.s) + log2(one)));
                    if (p.row_kl && rank == 0) p.row_kl[t] = static_cast<float>(kl);
                    sums[0] += w * kl;
                    const double gain = w * inv * p.factor * p.scale;
                    now[0] = static_cast<float>(mass == 0.0 ? 0.0 : gain * mass / sum.s);
                    now[1] = static_cast<float>(gain);
                }
            } else if (!counts && rank == 0 && tid == 0) {
                class_dead_row<MODE>(p, t);
            }
            // the table is empty again before the next row's classes come
            for (int i = tid; i < top.size; i += threads) top.table[i] = -1;
            if (tid == 0) top.twice[turn ^ 1] = 0;
        }
        turn ^= 1;
        if (MODE == kClassDistill || GRAD) __syncthreads();
        if (!GRAD) continue;
        const float factor = counts ? now[0] : 0.0f, m = -sum.m;
        const uint64_t c2 = f32x2_pack(p.c, p.c), m2 = f32x2_pack(m, m), factor2 = f32x2_pack(factor, factor);
        auto second = [&](int i, const unsigned char* at) {
            const int first = (i * tw + gw) * kStageGroups, left = min(kStageGroups, own.groups - first) - lane;
            uint4 raw[J];
#pragma unroll
            for (int j = 0; j < J; ++j) raw[j] = *reinterpret_cast<const uint4*>(at + (lane + 32 * j) * 16);
            give_back(k);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if (32 * j >= left) break;
                uint64_t v[G::P];
#pragma unroll
                for (int e = 0; e < G::P; ++e) v[e] = counts ? f32x2_mul(exp2_pair(G::pair(raw[j], e), c2, m2), factor2) : 0;
                row.store(first + lane + 32 * j, v);
            }
        };
        for (int i = dropped; i < own.stages; ++i) second(i, ring + out_slot * kStageBytes);
        for (int i = 0; i < dropped; ++i) second(i, wait_copy());
        if (edges) store_from_float(row.dx + row.edge(lane), counts ? exp2_fast(fmaf(edge, p.c, m)) * factor : 0.0f);
        if (!counts) continue;
        __syncwarp();                               // the targets' values replace what was just written, by the warp that wrote it
        auto owner = [&](int column) {
            const int g = column - row.head;
            return g < 0 || g >= row.groups * N ? 0 : (g / (N * kStageGroups)) % tw;
        };
        if (MODE == kClassPolicy) {
            if (lane == 0 && owner(int(target)) == gw) store_from_float(row.dx + target, now[1]);
        } else {
            const float gain = now[1];
            for (int j = lane; j < p.K; j += 32) {
                const int id = top.id[j];
                if (id < 0 || owner(id) != gw) continue;
                float weight = top.q[j] * top.part[(j % threads) >> 5];
                if (twice) {                        // a class that the teacher names twice has both weights
                    weight = 0.0f;
                    for (int i = 0; i < p.K; ++i)
                        if (top.id[i] == id) weight += top.q[i] * top.part[(i % threads) >> 5];
                }
                store_from_float(row.dx + id, fmaf(exp2_fast(fmaf(top.x[j], p.c, m)), factor, -gain * weight));
            }
            __syncthreads();                        // the next row's classes replace these
        }
    }
    if (gone) {
        // the copies in flight have to land before the shared memory is given up
        for (; taken > 0; --taken) {
            mbar_wait_drain(bars + out_slot, out_parity);
            if (++out_slot == depth) {
                out_slot = 0;
                out_parity ^= 1;
            }
        }
        if (tid == 0) atomicExch(p.timeout, kStatusTimeout);
    }
    // gradients of rows that do not count
    if (GRAD && p.order) {
        for (long long k = live + q; k < p.T; k += Q) {
            const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, __ldg(p.order + k), p.V);
            const uint64_t zero[G::P] = {};
            for (int g = rank * threads + tid; g < row.groups; g += C * threads) row.store(g, zero);
            if (gw == 0 && lane < row.edges) store_from_float(row.dx + row.edge(lane), 0.0f);
        }
    }
    if (MODE == kClassLogp || rank != 0) return;
    // the CTA that is done last adds the CTAs' sums up, in a fixed order
    if (tid == 0) {
        for (int i = 0; i < 3; ++i) p.cta_sum[3 * q + i] = sums[i];
        __threadfence();
        last_cta = atomicAdd(p.words, 1u) == unsigned(Q) - 1;
    }
    __syncthreads();
    if (!last_cta || warp != 0) return;
    __threadfence();
    for (int i = 0; i < 3; ++i) {
        sums[i] = 0.0;
        for (int r = lane; r < Q; r += 32) sums[i] += __ldcg(p.cta_sum + 3 * r + i);
        sums[i] = warp_sum64(sums[i]) * inv;
    }
    if (lane == 0) {
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
    using G = ClassGroup<E>;
    constexpr int N = G::N;
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
            const uint64_t zero[G::P] = {};
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
        const uint64_t c2 = f32x2_pack(p.c, p.c), m2 = f32x2_pack(m, m), k2 = f32x2_pack(k, k);
        for (; g < end; g += threads) {
            const uint4 raw = row.load(g);
            uint64_t v[G::P];
#pragma unroll
            for (int j = 0; j < G::P; ++j) v[j] = f32x2_mul(exp2_pair(G::pair(raw, j), c2, m2), k2);
            if (where >= g * N && where < g * N + N) {
#pragma unroll
                for (int j = 0; j < G::P; ++j) {
                    const int at = where - g * N - 2 * j;
                    v[j] = f32x2_add(v[j], f32x2_pack(at == 0 ? gt : 0.0f, at == 1 ? gt : 0.0f));
                }
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
