// Losses over a vocabulary's classes: rows x of V logits, l = scale * x, lse = log sum_v exp(l_v), p_v = exp(l_v - lse).
//
//   log-probability   lp = l_y - lse for the row's target y;   d lp / d x_v = scale * ([v = y] - p_v)
//   policy loss       r = exp(lp - old);  -min(r A, clip(r) A) + kl_coef * (exp(ref - lp) - (ref - lp) - 1)
//   preference loss   S = sum of lp over a sequence (or its mean), h = beta ((S_c - R_c) - (S_r - R_r)) - margin for a pair of
//                     sequences;  -(1 - smoothing) log sigmoid(h) - smoothing log sigmoid(-h)
//   distillation      q_k over K of the classes from a teacher's logits;  sum_k q_k (log q_k - lp_k)
//
// Everything needs a row's largest logit `top` and the sum s of its exponentials, and the gradients read the row again.  Exponentials are
// powers of two: with c = scale * log2(e) rounded to fp32 once, every term is 2^((x - top) * c), and lse = scale * top + log s.  (The difference
// comes first, so that rows far from zero keep their bits, and rows of the type's lowest value their sum: x * c would overflow there.)  The
// gradient forms the same terms again and multiplies them by -g / s: the probabilities of a row add up to one.  Row sums are fp32 in trees of a
// thread's own terms, the few numbers of a row fp64.
#pragma once
#include <cmath>

#include "lrgd_embed.cuh"

namespace lrgd {

constexpr int kClassMaxTop = 1024;                  // classes of a teacher per row, at most
constexpr double kLn2 = 0.693147180559945309417232121458;

enum ClassMode { kClassLogp = 0, kClassPolicy = 1, kClassDistill = 2 };

struct ClassScale {              // scale * log2(e)
    float c;                     // to the nearest
    float down, rest;            // in two parts; rest is above 0, so that -inf stays -inf in the product with each
};

struct ClassParams {
    const void* x;
    long long ld;
    long long T;
    int V;
    const void* ids;             // targets [T]; distillation: the teacher's classes [T][K]
    int wide_ids;
    long long ignore;
    ClassScale cs;               // scale * log2(e) ...
    float c;                     // ... to the nearest
    double c64;
    float scale;
    const float* weights;        // nullable [T]
    void* dx;
    long long ld_d;
    int* status;
    // log-probabilities
    float* logp;
    float* lse;
    // what the preference loss keeps of a row: its largest logit and its sum, lp in fp64; rows before and behind all sequences do not count
    float2* stat;
    double* logp64;
    float* coef;                 // set to 0
    const void* offsets;
    int wide_offsets;
    long long sequences;
    // policy
    const float* adv;
    const float* old_logp;
    const float* ref_logp;
    float ratio_low, ratio_high, kl_coef;
    double log_low, log_high;    // of 1 - clip_low (-inf where that is not above 0) and 1 + clip_high
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
    int listed;                  // long rows: every CTA lists its rows for itself (see class_list)
    const int* order;            // the rows that count, then the others (k_class_prep).  Neither: all rows, looked at one by one
    const struct ClassPrep* prep;
    int cluster;                 // long rows: CTAs per row (a power of two), stages in a ring
    int depth;
    const double* norm_part;     // short rows: the sum of the weights in parts (k_class_norm), or none
    int norm_parts;
    long long norm_rows;         // of a part
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

// A log-sum-exp in units of the logits, lse / scale, as high + low / c: high is the nearest finite fp32 (lse / scale may be past them where scale is
// tiny), low what that leaves of the exponent.
struct ClassBase {
    float high, low;
};
__device__ __forceinline__ ClassBase class_base(float lse, float scale, double c64) {
    const double own = static_cast<double>(lse) / scale;
    const float high = fminf(fmaxf(static_cast<float>(own), -3.4028234e38f), 3.4028234e38f);       // (a NaN is in low)
    return {high, static_cast<float>((own - static_cast<double>(high)) * c64)};
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
// 2^((x - top) * c), and of both halves.  The unit for powers drops the last bits of its argument: results below 1/2 come out 5e-8 too small in the mean
// (measured over 4 M random arguments, alike from 2^-1 to 2^-115), those above it 2e-8; 2^0 is exact.  One row's lp does not show that, the sum over a
// long sequence does.  So the argument is raised by as much, in the same instruction; the mean error is then below 4e-9, and 2^0 is 1 still: ties
// and rows of one value are exact.  A row's many terms are raised alike (those above 1/2 are few, and come out 3e-8 too large).
constexpr float kPowerLift = 7e-8f, kPowerLiftHigh = 3e-8f, kPowerLiftRaise = 4e-8f;
__device__ __forceinline__ float class_power(float x, float top, float c) { return exp2_fast(fmaf(x - top, c, kPowerLift)); }
__device__ __forceinline__ uint64_t class_powers(uint64_t x, uint64_t minus_top, uint64_t c) {
    float lo, hi;
    f32x2_unpack(f32x2_fma(f32x2_add(x, minus_top), c, f32x2_pack(kPowerLift, kPowerLift)), lo, hi);
    return f32x2_pack(exp2_fast(lo), exp2_fast(hi));
}
// The exponent of a difference d.  WHOLE: with what fp32 leaves of scale * log2(e), 1.3e-8 of it at a scale of 1, which is the same for all rows: 5e-8 in
// lp where the largest logit is 10 above most.  An instruction more per two logits, so only for log-probabilities that are added up: they wait
// for HBM anyway (the policy loss does not: 8192 x 128000 676 us instead of 661).
template <bool WHOLE>
__device__ __forceinline__ float class_exponent(float d, ClassScale c, float lift) {
    return WHOLE ? fmaf(d, c.down, fmaf(d, c.rest, lift)) : fmaf(d, c.c, lift);
}
template <bool WHOLE>
__device__ __forceinline__ uint64_t class_powers(uint64_t x, uint64_t minus_top, ClassScale c) {
    if constexpr (!WHOLE) {
        return class_powers(x, minus_top, f32x2_pack(c.c, c.c));
    } else {
        float lo, hi;
        const uint64_t d = f32x2_add(x, minus_top);
        f32x2_unpack(f32x2_fma(d, f32x2_pack(c.down, c.down), f32x2_fma(d, f32x2_pack(c.rest, c.rest), f32x2_pack(kPowerLift, kPowerLift))), lo, hi);
        return f32x2_pack(exp2_fast(lo), exp2_fast(hi));
    }
}
// What carries a sum of terms up to `top` to the larger maximum `most`: often above 1/2, and several of them one after the other, so both kinds are told
// apart (rows of 32003 logits with a spread of 0.3: the mean error of lp 2e-8 at most, 8e-8 with 7e-8 for all).  Within a thread the running maximum
// takes a number between the two (policy loss 8192 x 128000: 661 us; told apart there too: 679).
template <bool WHOLE>
__device__ __forceinline__ float class_carry(float top, float most, ClassScale c) {
    return exp2_fast(class_exponent<WHOLE>(top - most, c, (top - most) * c.c > -1.0f ? kPowerLiftHigh : kPowerLift));
}

// 16 bytes of a row
template <class E>
struct ClassGroup {
    static constexpr int N = 16 / int(sizeof(E));
    static constexpr int P = N / 2;
    static __device__ __forceinline__ uint32_t word(const uint4& w, int i) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    static __device__ __forceinline__ uint4 nothing() {         // all -inf
        constexpr uint32_t w = sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
        return make_uint4(w, w, w, w);
    }
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
            float t[J];
#pragma unroll
            for (int j = 0; j < J; ++j)
                t[j] = fmaxf(fmaxf(__uint_as_float(raw[j].x), __uint_as_float(raw[j].y)), fmaxf(__uint_as_float(raw[j].z), __uint_as_float(raw[j].w)));
#pragma unroll
            for (int j = 1; j < J; ++j) t[0] = fmaxf(t[0], t[j]);
            return t[0];
        } else {
            uint32_t t[J];
#pragma unroll
            for (int j = 0; j < J; ++j) t[j] = max2(max2(raw[j].x, raw[j].y), max2(raw[j].z, raw[j].w));
#pragma unroll
            for (int d = 1; d < J; d *= 2)
#pragma unroll
                for (int j = 0; j + d < J; j += 2 * d) t[j] = max2(t[j], t[j + d]);
            return fmaxf(__uint_as_float(t[0] << 16), __uint_as_float(t[0] & 0xffff0000u));
        }
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
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
        head = min((N - off) & (N - 1), V);
        groups = (V - head) / N;
        edges = V - groups * N;
        wide_store = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15) == 0;
    }
    // element e of those outside the groups
    __device__ __forceinline__ int edge(int e) const { return e < head ? e : e + groups * ClassGroup<E>::N; }
    __device__ __forceinline__ uint4 load(int g) const { return *reinterpret_cast<const uint4*>(x + head + g * ClassGroup<E>::N); }
    __device__ __forceinline__ void store(int g, const uint64_t (&v)[ClassGroup<E>::P]) const { store_at(dx + head + g * ClassGroup<E>::N, v); }
    __device__ __forceinline__ void store_at(E* at, const uint64_t (&v)[ClassGroup<E>::P]) const {
        constexpr int N = ClassGroup<E>::N;
        if (wide_store) {
            *reinterpret_cast<uint4*>(at) = ClassGroup<E>::narrow(v);
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

__device__ __forceinline__ float warp_largest(float v) {
    const uint32_t key = __reduce_max_sync(0xffffffffu, order_key(v));
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}
// The running maximum and sum of a part of a row: s = sum of 2^((x - top) * c), top = -inf before the first finite x
struct ClassSum {
    float top = -INFINITY, s = 0.0f;
    // room for terms up to t; false where nothing finite has come yet
    template <bool WHOLE>
    __device__ __forceinline__ bool raise(float t, ClassScale c) {
        if (t > top) {
            s *= exp2_fast(class_exponent<WHOLE>(top - t, c, kPowerLiftRaise));
            top = t;
        }
        return top != -INFINITY;
    }
    template <bool WHOLE>
    __device__ __forceinline__ void add(float v, ClassScale c) {
        if (raise<WHOLE>(v, c)) s += exp2_fast(class_exponent<WHOLE>(v - top, c, kPowerLift));
        else if (v != v) s = v;
    }
    template <class E, int J, bool WHOLE>
    __device__ __forceinline__ void add_groups(const uint4 (&raw)[J], ClassScale c) {
        using G = ClassGroup<E>;
        if (!raise<WHOLE>(G::template largest<J>(raw), c)) {               // a NaN has to be seen all the same
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
        const uint64_t top2 = f32x2_pack(-top, -top);
        uint64_t part[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < G::P; ++i) part[i & 1] = f32x2_add(part[i & 1], class_powers<WHOLE>(G::pair(raw[j], i), top2, c));
        float lo, hi;
        f32x2_unpack(f32x2_add(part[0], part[1]), lo, hi);
        s += lo + hi;
    }
    // the sum over the lanes of a warp, the same bits in all of them
    template <bool WHOLE>
    __device__ __forceinline__ void over_warp(ClassScale c) {
        const float most = warp_largest(top);
        s = s == 0.0f ? 0.0f : s * class_carry<WHOLE>(top, most, c);       // (a NaN stays one)
        top = most;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    }
    // where no logit is finite s is 0 (or NaN): lse is -inf, a probability NaN
    __device__ __forceinline__ void settle() {
        if (top == -INFINITY) top = 0.0f;
    }
};

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

// The rows that sequences hold: those from the first to the last that a sequence names whose own offsets neither fall nor leave the rows.  With more
// than kSpanSequences all rows are taken (the coefficient of a row that no sequence names is 0 all the same).
constexpr int kSpanSequences = 256;
struct ClassSpan {
    int from, to;
    __device__ __forceinline__ bool has(long long t) const { return unsigned(static_cast<int>(t) - from) < unsigned(to - from); }
    __device__ __forceinline__ void join(const ClassParams& p, int i) {         // sequence i
        const long long a = load_any_id(p.offsets, p.wide_offsets, i), z = load_any_id(p.offsets, p.wide_offsets, i + 1);
        if (a >= 0 && a < z && z <= p.T) {
            from = min(from, static_cast<int>(a));
            to = max(to, static_cast<int>(z));
        }
    }
    __device__ __forceinline__ void over_warp() {
        from = __reduce_min_sync(0xffffffffu, from);
        to = max(from, __reduce_max_sync(0xffffffffu, to));
    }
};
// (by one warp)
__device__ __forceinline__ ClassSpan class_warp_span(const ClassParams& p) {
    if (!p.offsets || p.sequences > kSpanSequences) return {0, static_cast<int>(p.T)};
    ClassSpan span{static_cast<int>(p.T), 0};
    for (int i = threadIdx.x & 31; i < p.sequences; i += 32) span.join(p, i);
    span.over_warp();
    return span;
}
// (by all threads of a CTA, a sequence each: 100 pairs in front of 6101 rows by a warp alone take 4 us more)
__device__ __forceinline__ ClassSpan class_span(const ClassParams& p) {
    if (!p.offsets || p.sequences > kSpanSequences) return {0, static_cast<int>(p.T)};
    constexpr int kWarps = kSpanSequences / 32;
    __shared__ ClassSpan part[kWarps];
    ClassSpan span{static_cast<int>(p.T), 0};
    if (threadIdx.x < p.sequences) span.join(p, threadIdx.x);
    span.over_warp();
    if (threadIdx.x < kSpanSequences && (threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = span;
    __syncthreads();
    span = part[threadIdx.x & (kWarps - 1)];
    span.over_warp();
    return span;
}

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// log of the sum.  It is 2^e f with 1 <= f < 2, so that the fp32 logarithm is one of a number below 1 and off by 6e-8 at most.
__device__ __forceinline__ double class_log(float s) {
    if (!(s > 0.0f && s < INFINITY)) return logf(s);
    const uint32_t bits = __float_as_uint(s);       // (at least 1 where it is positive: the largest term)
    const int e = static_cast<int>(bits >> 23) - 127;
    const float f = __uint_as_float((bits & 0x7fffffu) | 0x3f800000u);
    return kLn2 * (e + static_cast<double>(log2f(f)));
}

// ---- which rows count ----------------------------------------------------------------------------------
// One CTA writes the numbers of the rows that count into `order`, in their order, those of the others behind them, and sums the weights.
// Rows that do not count get their zeros here (all but their gradient).  Bound by latency, 8192 rows at a turn: about 4 us.
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
    static_assert(kPrepThreads == 32 * 32, "a lane for every warp");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_release();
    const ClassSpan span = MODE == kClassLogp ? class_span(p) : ClassSpan{};
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
                if (MODE == kClassLogp) live = live && span.has(t);
                if (live) norm += w;
                else class_dead_row<MODE>(p, t);
            }
            mask[j] = __ballot_sync(0xffffffffu, live);
            mine += __popc(mask[j]);
        }
        __syncthreads();                            // the last turn's counts have been read
        if (lane == 0) warp_live[warp] = mine;
        __syncthreads();
        const int of_lane = warp_live[lane];
        const int all = __reduce_add_sync(0xffffffffu, of_lane);
        int at = before + __reduce_add_sync(0xffffffffu, lane < warp ? of_lane : 0);
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
    if (warp == 0) {
        norm = warp_sum64(warp_norm[lane]);
        if (lane == 0) {
            prep->norm = norm;
            prep->live = before;
        }
    }
}

// ---- a teacher's classes -------------------------------------------------------------------------------
// One warp has them: entry j belongs to lane j mod 32.  q is 2^((v - base) * c), times a factor it is the weight.
struct ClassTop {
    int* id;                     // [K], -1: absent
    float* q;                    // [K]
    float* x;                    // [K] the student's logits
    uint32_t* marks;             // a bitmap of classes, 2^bits
    int bits;
};
__host__ __device__ inline int class_mark_bits(int K) {             // at least 32 places for a class: 64 of them find one or so taken
    int bits = 10;
    while (bits < 15 && (1 << bits) < 32 * K) ++bits;
    return bits;
}
__host__ __device__ inline size_t class_top_bytes(int K) { return ((size_t(1) << class_mark_bits(K)) / 8 + size_t(K) * 12 + 15) / 16 * 16; }
__device__ __forceinline__ ClassTop class_top_at(unsigned char* at, int K) {
    ClassTop top;
    top.marks = reinterpret_cast<uint32_t*>(at);
    top.bits = class_mark_bits(K);
    at += (1 << top.bits) / 8;
    top.id = reinterpret_cast<int*>(at);
    top.q = reinterpret_cast<float*>(at + 4 * K);
    top.x = reinterpret_cast<float*>(at + 8 * K);
    return top;
}
__device__ __forceinline__ void class_clear_marks(const ClassTop& top) {
    for (int i = threadIdx.x & 31; i < (1 << top.bits) / 128; i += 32) reinterpret_cast<uint4*>(top.marks)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
}
// Asks for a row's classes and the teacher's logits to be in L2 (4096 x 128000 bfloat16, 256 classes: 418 us without, 414 with; up to 128 classes the
// same)
__device__ __forceinline__ void class_top_ahead(const ClassParams& p, long long t) {
    const int id_bytes = p.K * (p.wide_ids ? 8 : 4), v_bytes = p.K * (p.teacher_half ? 2 : 4);
    const char* ids = static_cast<const char*>(p.ids) + t * id_bytes;
    const char* v = static_cast<const char*>(p.teacher) + t * v_bytes;
    for (int b = 128 * (threadIdx.x & 31); b < id_bytes; b += 128 * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(ids + b));
    for (int b = 128 * (threadIdx.x & 31); b < v_bytes; b += 128 * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(v + b));
}
// ... and the logits at them, by the CTAs of a cluster together, each of which will read them all (2048 x 100000 fp32, 256 classes: 331 us without, 302
// with; 128 classes 302 and 290; 4096 x 128000 bfloat16, 256 classes 424 and 414, 64 classes 372 and 374; a CTA alone would ask for what it reads
// next)
template <class E>
__device__ __forceinline__ void class_top_logits_ahead(const ClassParams& p, long long t, int rank) {
    const E* row = static_cast<const E*>(p.x) + t * p.ld;
#pragma unroll 2
    for (int j = 32 * rank + (threadIdx.x & 31); j < p.K; j += 32 * p.cluster) {
        const long long id = load_any_id(p.ids, p.wide_ids, t * p.K + j);
        if (id >= 0 && id < p.V) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + id));
    }
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
    if (e.id == p.ignore) return -1;                // (a class of the vocabulary or not)
    if (e.id < 0 || e.id >= p.V) {
        atomicExch(p.status, -4);                   // LR_ERR_VALUE
        return -1;
    }
    return e.v == -INFINITY ? -1 : static_cast<int>(e.id);
}
// Marks the class; true where this place of the bitmap is taken, by the same class or by another one
__device__ __forceinline__ bool class_mark(const ClassTop& top, int id) {
    uint32_t h = static_cast<uint32_t>(id) * 2654435761u;
    h ^= h >> 15;
    h = h * 2246822519u >> (32 - top.bits);
    const uint32_t bit = 1u << (h & 31);
    return (atomicOr(top.marks + (h >> 5), bit) & bit) != 0;
}

// What the entries add up to, in fp64: the divergence is a difference of sums of its size and larger.
struct ClassTopSum {
    double all, mixed;           // sum of q, of q * (scale * (v - base) - scale * (x - near))
    float near;                  // the largest of their x
    bool twice;                  // some class is named twice
};
// Reads a row's classes; the bitmap is empty before and after.  U entries of a lane are on their way together.
template <int U, class E>
__device__ __forceinline__ ClassTopSum class_top_read(const ClassParams& p, long long t, const E* row, const ClassTop& top) {
    const int lane = threadIdx.x & 31;
    ClassTopSum r{0.0, 0.0, -INFINITY, false};
    float largest = -INFINITY;
    const float own = p.teacher_lse ? __ldg(p.teacher_lse + t) : 0.0f;
    for (int j0 = 0; j0 < p.K; j0 += 32 * U) {
        ClassEntry e[U];
        int id[U];
        float x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) e[i] = class_entry(p, t, j0 + 32 * i + lane);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            id[i] = j0 + 32 * i + lane < p.K ? class_entry_id(p, e[i]) : -1;
            x[i] = id[i] >= 0 ? load_local(row + id[i]) : 0.0f;
        }
        uint32_t taken = 0;                         // bit i: the place of entry i in the bitmap was taken, by the same class or another one
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (id[i] >= 0 && class_mark(top, id[i])) taken |= 1u << i;
            const int j = j0 + 32 * i + lane;
            if (j < p.K) {
                top.id[j] = id[i];
                top.q[j] = e[i].v;
                top.x[j] = x[i];
            }
            if (id[i] >= 0) {
                largest = fmaxf(largest, e[i].v);
                r.near = fmaxf(r.near, x[i]);
            }
        }
        __syncwarp();
        for (uint32_t lanes = __ballot_sync(0xffffffffu, taken != 0); lanes && !r.twice; lanes = __ballot_sync(0xffffffffu, taken != 0)) {
            const int from = __ffs(lanes) - 1, i = __ffs(__shfl_sync(0xffffffffu, taken, from)) - 1, which = top.id[j0 + 32 * i + from];
            if (lane == from) taken &= taken - 1;
            int same = 0;
            for (int j = lane; j < min(p.K, j0 + 32 * U); j += 32) same += top.id[j] == which;
            r.twice = __reduce_add_sync(0xffffffffu, same) > 1;
        }
    }
    largest = warp_max(largest);
    r.near = warp_max(r.near);
    if (r.near == -INFINITY) r.near = 0.0f;
    // base is the largest v, or the teacher's own lse / scale.  The exponent is fp64, its power fp32 (exp2f is good to 2 units of the last place)
    // with what the fp32 exponent leaves.
    const double base = p.teacher_lse ? static_cast<double>(own) / p.scale : largest == -INFINITY ? 0.0 : static_cast<double>(largest);
    for (int j = lane; j < p.K; j += 32) {
        const double a = (static_cast<double>(top.q[j]) - base) * p.c64;
        const float near = static_cast<float>(a + kPowerLift), power = exp2f(near);         // (the lift as in class_power)
        float e = 0.0f;
        if (top.id[j] >= 0 && power != 0.0f) {
            e = fmaf(power, static_cast<float>(a + kPowerLift - near) * static_cast<float>(kLn2), power);
            r.all += e;
            r.mixed += e * (kLn2 * a - static_cast<double>(top.x[j] - r.near) * p.scale);
        }
        top.q[j] = e;
    }
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        const double all = __shfl_xor_sync(0xffffffffu, r.all, d), mixed = __shfl_xor_sync(0xffffffffu, r.mixed, d);
        r.all += all;
        r.mixed += mixed;
    }
    class_clear_marks(top);
    return r;
}

// ---- a row's last numbers ------------------------------------------------------------------------------
// What the statistics of a row that counts give, by one warp: outputs of the row (with `write`), its part of the sums, and for the gradient
// factor (what the terms 2^(..) are multiplied by) and at (policy: the value at the target; distillation: what q is multiplied by).
struct ClassNumbers {
    float factor, at;
};
// What a row has beside its logits, fetched before its statistics are known
struct ClassInputs {
    long long target;
    float w, xy, adv, old_logp, ref_logp;
    ClassTopSum top;
};
template <int MODE, int U = 8, class E>
__device__ __forceinline__ void class_inputs(const ClassParams& p, long long t, const E* row, const ClassTop& top, ClassInputs& in) {
    if (MODE == kClassDistill) {
        in.top = class_top_read<U>(p, t, row, top);
        return;
    }
    in.xy = load_local(row + in.target);
    if (MODE == kClassPolicy) {
        in.adv = __ldg(p.adv + t);
        in.old_logp = p.old_logp ? __ldg(p.old_logp + t) : 0.0f;
        in.ref_logp = p.ref_logp ? __ldg(p.ref_logp + t) : 0.0f;
    }
}
// exp(d) - 1 - d.  Near 0, where that is the difference of nearly equal numbers, by its series: d^2/2 (1 + d/3 (1 + d/4 (...))), cut off where a
// term of |d| = 1/4 is below 2e-8 of the sum.
__device__ __forceinline__ float class_kl(float d) {
    if (fabsf(d) < 0.25f) {
        float r = 1.0f;
#pragma unroll
        for (int i = 8; i >= 3; --i) r = fmaf(d * (1.0f / i), r, 1.0f);
        return 0.5f * d * d * r;
    }
    return d == INFINITY ? d : expm1f(d) - d;
}
// Half of fp32's range at most (a NaN stays one): a difference of two such numbers is finite, and a row's factor times a power that is 0 is 0 also
// where the formula is past fp32.
__device__ __forceinline__ float class_held(float v) {
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(1.69e38f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(-1.69e38f));
    return v;
}
// ... and what of it is written down afterwards
struct ClassTerms {
    double lp, lse;
    float first, kl, clipped;    // the row's loss: its parts (policy: the first and whether it is clipped; distillation: kl)
};
// (by W lanes, each with the same arguments)
template <int MODE, int W = 32>
__device__ __forceinline__ ClassNumbers class_numbers(const ClassParams& p, const ClassInputs& in, const ClassSum& sum, double inv, ClassTerms& terms) {
    const int lane = threadIdx.x & (W - 1);
    const double log_s = class_log(sum.s);
    ClassNumbers r{};
    terms = ClassTerms{0.0, static_cast<double>(sum.top) * p.scale + log_s, 0.0f, 0.0f, 0.0f};
    const float gain = static_cast<float>(in.w * inv * p.factor * p.scale);
    if (MODE == kClassDistill) {
        // with the teacher's own normalisation log q is smaller by log(all)
        const float all = static_cast<float>(in.top.all), one = p.teacher_lse || all == 0.0f ? 1.0f : 1.0f / all, mass = p.teacher_lse || all == 0.0f ? all : 1.0f;
        const double ahead = (static_cast<double>(sum.top) - in.top.near) * p.scale + log_s;
        if (all == 0.0f) {
            terms.kl = 0.0f;
        } else if (p.teacher_lse) {
            terms.kl = static_cast<float>(in.top.mixed + in.top.all * ahead);
        } else {                                    // (1 / all to fp64: a step of Newton's)
            const double whole = one * (2.0 - in.top.all * one);
            terms.kl = static_cast<float>(in.top.mixed * whole + ahead - logf(all));
        }
        r.factor = mass == 0.0f ? 0.0f : gain * mass / sum.s;
        r.at = gain * one;
        return r;
    }
    terms.lp = (static_cast<double>(in.xy) - sum.top) * p.scale - log_s;
    if (terms.lp > 0.0) terms.lp = 0.0;             // rounding
    if (MODE == kClassPolicy) {
        // exp(lp - old) - 1, exp(ref - lp) - 1 and exp(lp) - 1: one lane each.  The differences are fp64, their exponentials fp32 (one unit in
        // the last place), which is what outputs in fp32 show.
        const float d = static_cast<float>(lane == 0 ? terms.lp - in.old_logp : lane == 1 ? in.ref_logp - terms.lp : terms.lp);
        const float e = expm1f(d);
        float ratio = p.old_logp ? __shfl_sync(0xffffffffu, e, 0, W) + 1.0f : 1.0f;
        if (ratio > 3.4e38f) ratio = 3.4e38f;       // (no infinity: an advantage of 0 has no loss whatever the ratio)
        const float away = __shfl_sync(0xffffffffu, e, 1, W), rest = __shfl_sync(0xffffffffu, e, 2, W);
        // r A > r' A: the ratio is past the border on the side that A pulls to.  Decided on its fp64 logarithm, because a row gains or loses all of
        // its gradient there.
        const float a = in.adv, held = a > 0.0f ? p.ratio_high : p.ratio_low;
        const double log_ratio = p.old_logp ? terms.lp - in.old_logp : 0.0;
        const bool clipped = a > 0.0f ? log_ratio > p.log_high : a < 0.0f && log_ratio < p.log_low;
        float g = clipped ? 0.0f : class_held(-ratio * a);
        if (p.ref_logp && p.kl_coef != 0.0f) g -= class_held(p.kl_coef * away);
        terms.first = -(clipped ? held : ratio) * a;
        terms.clipped = clipped ? 1.0f : 0.0f;
        g = class_held(g * gain);
        r.factor = -g / sum.s;
        r.at = -g * rest;
    }
    return r;
}
// (`write` in one lane)
template <int MODE>
__device__ __forceinline__ void class_account(const ClassParams& p, long long t, const ClassInputs& in, const ClassSum& sum, const ClassTerms& terms,
                                              bool write, double (&sums)[3]) {
    if (MODE == kClassDistill) {
        if (p.row_kl && write) p.row_kl[t] = terms.kl;
        sums[0] += static_cast<double>(in.w) * terms.kl;
        return;
    }
    if (p.logp && write) p.logp[t] = static_cast<float>(terms.lp);
    if (MODE == kClassLogp) {
        if (p.lse && write) p.lse[t] = static_cast<float>(terms.lse);
        if (p.stat && write) {
            p.stat[t] = make_float2(sum.top, sum.s);
            p.logp64[t] = terms.lp;
            p.coef[t] = 0.0f;
        }
    } else {
        sums[0] += static_cast<double>(in.w) * terms.first;
        if (p.ref_logp) sums[1] += static_cast<double>(in.w) * class_kl(static_cast<float>(in.ref_logp - terms.lp));
        sums[2] += terms.clipped != 0.0f ? in.w : 0.0f;
    }
}
// What the gradient is at entry j of the teacher's classes
__device__ __forceinline__ float class_top_value(const ClassParams& p, const ClassTop& top, int j, bool twice, float largest, const ClassNumbers& r) {
    const int id = top.id[j];
    float q = top.q[j];
    if (twice) {                                    // a class that the teacher names twice has both weights
        q = 0.0f;
        for (int i = 0; i < p.K; ++i)
            if (top.id[i] == id) q += top.q[i];
    }
    return fmaf(class_power(top.x[j], largest, p.c), r.factor, -r.at * q);
}
// Thread `me` of `many`: its part of the sum of the weights of the rows first ... last - 1 that count, four rows' loads at a time
template <int MODE>
__device__ __forceinline__ double class_norm_part(const ClassParams& p, long long first, long long last, int me, int many) {
    constexpr int U = 4;
    double n = 0.0;
    for (long long t = first + me; t < last; t += U * many) {
        long long id[U];
        float w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long at = t + u * many;
            w[u] = at >= last ? 0.0f : p.weights ? __ldg(p.weights + at) : 1.0f;
            id[u] = at < last && MODE != kClassDistill ? load_any_id(p.ids, p.wide_ids, at) : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (w[u] != 0.0f && (MODE == kClassDistill || (id[u] != p.ignore && id[u] >= 0 && id[u] < p.V))) n += w[u];
    }
    return n;
}
// The warp that is done last adds the sums of all `ctas` warps that call this up, in a fixed order
template <int MODE>
__device__ __forceinline__ void class_finish(const ClassParams& p, int me, int ctas, double inv, double (&sums)[3]) {
    const int lane = threadIdx.x & 31;
    int last = 0;
    if (lane == 0) {
        for (int i = 0; i < 3; ++i) p.cta_sum[3 * me + i] = sums[i];
        __threadfence();
        last = atomicAdd(p.words, 1u) == unsigned(ctas) - 1;
    }
    if (!__shfl_sync(0xffffffffu, last, 0)) return;
    __threadfence();
    for (int i = 0; i < 3; ++i) {
        sums[i] = 0.0;
        for (int r = lane; r < ctas; r += 32) sums[i] += __ldcg(p.cta_sum + 3 * r + i);
        sums[i] = warp_sum64(sums[i]) * inv;
    }
    if (lane == 0) {
        if (MODE == kClassPolicy) {
            const double kl = p.kl_coef != 0.0f ? static_cast<double>(p.kl_coef) * sums[1] : 0.0;       // (0 * inf where it is only watched)
            p.out[0] = static_cast<float>(p.factor * (sums[0] + kl));
            for (int i = 0; i < 3; ++i) p.out[1 + i] = static_cast<float>(sums[i]);
        } else {
            p.out[0] = static_cast<float>(p.factor * sums[0]);
        }
        p.words[0] = 0;
    }
}

// ---- long rows -----------------------------------------------------------------------------------------
// A CTA per row, or a cluster of C.  Its warps have different work, and hand rows to each other through mbarriers:
//   two or four teams of warps take turns at the rows: first pass (running maximum and sum), then, when the row's numbers are known, second pass
//     (the gradient).  While one team waits, or reduces, the others work;
//   a warp per team copies its rows' 16-byte groups, in stages of 8, 18 or 32 KB, into the team's ring of shared memory, as far ahead as the ring
//     allows (a ring of its own, because who skips another team's stages cannot tell an mbarrier's phases apart);
//   kNumberWarps warps take turns at the rows: they fetch what a row has beside its logits, join the sums of the team's warps (and of the
//     cluster's CTAs, by 8-byte messages), work out the row's numbers in fp64, and put the values at the targets over the gradient.
//     Between them they write zeros into the gradients of rows that do not count, as many at every row (all at once they fill the queues
//     of the memory system that the others wait in).
// The logits stay in the ring between the passes, so they are read once: the host takes clusters so large that two thirds of a row fit.
// Stages that the ring could not hold are copied once more (`dropped`), from L2.  Stages are given back in the order of the copies.
// Bound by HBM for log-probabilities (6000 x 100000 fp32, 80 % counting, 290 us: 6.6 TB/s); with a gradient by HBM and by the waits between the passes:
// 52 % of the issue slots and 56 % of the unit for powers are busy, 132 of 148 SMs work where a row takes four CTAs.  8192 x 128000 bfloat16, three
// quarters counting, policy loss 664 us (5.5 TB/s; 714 under the power cap of a long run); 4096 x 128000, 64 classes of a teacher 375 us (5.6);
// 2048 x 100000 fp32, 256 classes 302 us (5.2: bound by the number warps).
// Who shares the work, by what is asked for.  Log-probabilities alone: large stages, the second pass does not exist.  The policy loss: four teams, which
// hide one another's waits better than two (in the kernel's first form 650 us instead of 690; three 715, five of three warps 839).
// Distillation: the teacher's classes take the room of a stage, and every row more of the number warps' time, so there are two teams, of
// nine warps (375 us; of eight 380).
constexpr int kMaxCluster = 8;

// Up to this many rows the CTAs look all of them over themselves, which takes as long as a launch of k_class_prep less (T = 300: 2 us).
constexpr int kListedRows = 4096;
constexpr int kListedMine = 256;                    // ... if no cluster has more of them
struct ClassList {
    double norm[32], total;
    int count[32], all;
    unsigned short live[kListedMine], dead[kListedMine];
};

template <int MODE>
struct Ring {
    static constexpr int kTeams = MODE == kClassPolicy ? 4 : 2;
    static constexpr int kTeamWarps = MODE == kClassPolicy ? 4 : MODE == kClassDistill ? 9 : 8;
    static constexpr int kPassWarps = kTeams * kTeamWarps;
    static constexpr int kNumberWarps = 4;          // (eight: policy 672 us instead of 664, distillation 403 instead of 375, of 256 classes 326 instead of 303)
    static constexpr int kThreads = 32 * (kPassWarps + kTeams + kNumberWarps);
    static constexpr int kLaneGroups = MODE == kClassLogp ? 8 : 4;              // of a stage
    static constexpr int kWarpGroups = 32 * kLaneGroups;
    static constexpr int kStageGroups = kTeamWarps * kWarpGroups;
    static constexpr int kStageBytes = kStageGroups * 16;
    static constexpr int kDepth = (224 << 10) / (kTeams * kStageBytes);         // stages of a team's ring, at most
    static constexpr int kRows = 4;                 // rows under way between the warps; a multiple of kNumberWarps and kTeams

    struct alignas(16) Shared {
        uint64_t full[kTeams][kDepth], free[kTeams][kDepth];
        // of row k, at k mod kRows: the team's sums are there; the row's numbers are there; its gradient is written
        uint64_t summed[kRows], ready[kRows], written[kRows];
        // the cluster's sums, twice as many rows: a CTA that is ahead sends row k + kRows before this one has looked at row k, but not row
        // k + 2 kRows, for which it needs this CTA's row k + kRows, which the warp that looks at row k sends later
        uint64_t joined[2 * kRows];
        float2 cta_sum[2 * kRows][kMaxCluster];
        float2 warp_sum[kRows][kTeamWarps];         // largest logit, sum
        float2 row[kRows];                          // factor, top
        ClassList list;
        int abort_word;
    };
};

// A CTA lists its rows (see kListedRows): its cluster's are every Q-th of those that count, and every Q-th of the others.
template <int MODE>
__device__ __forceinline__ void class_list(const ClassParams& p, ClassList& list, int q, int Q, bool write) {
    constexpr int kWarps = Ring<MODE>::kThreads / 32, kTurns = (kListedRows + 32 * kWarps - 1) / (32 * kWarps);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, turns = (int(p.T) + 32 * kWarps - 1) / (32 * kWarps);
    const ClassSpan span = MODE == kClassLogp ? class_span(p) : ClassSpan{};
    unsigned int mask[kTurns];
    double norm = 0.0;
    int count = 0;
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
        const int t = (warp * turns + j) * 32 + lane;
        bool live = false;
        if (j < turns && t < p.T) {
            long long target;
            float w;
            live = class_counts(p, t, MODE, &target, &w);
            if (MODE == kClassLogp) live = live && span.has(t);
            if (live) norm += w;
        }
        mask[j] = __ballot_sync(0xffffffffu, live);
        count += __popc(mask[j]);
    }
    norm = warp_sum64(norm);
    if (lane == 0) {
        list.count[warp] = count;
        list.norm[warp] = norm;
    }
    __syncthreads();
    const int of_lane = lane < kWarps ? list.count[lane] : 0;
    int at = __reduce_add_sync(0xffffffffu, lane < warp ? of_lane : 0);
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
        const int t = (warp * turns + j) * 32 + lane, ahead = at + __popc(mask[j] & ((1u << lane) - 1));
        at += __popc(mask[j]);
        if (j >= turns || t >= p.T) continue;
        const bool live = mask[j] >> lane & 1;
        const int i = live ? ahead : t - ahead;
        if (i % Q != q) continue;
        (live ? list.live : list.dead)[i / Q] = static_cast<unsigned short>(t);
        if (!live && write) class_dead_row<MODE>(p, t);
    }
    if (warp == 0) {
        const int all = __reduce_add_sync(0xffffffffu, of_lane);
        norm = warp_sum64(lane < kWarps ? list.norm[lane] : 0.0);
        if (lane == 0) {
            list.all = all;
            list.total = norm;
        }
    }
    __syncthreads();
}

__device__ __forceinline__ uint64_t l2_policy_evict_normal() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Two floats into the same place of another CTA's shared memory; 8 bytes are counted on its barrier
__device__ __forceinline__ void send_f32x2(const float2* local, const uint64_t* bar, uint32_t rank, float a, float b) {
    uint32_t to, to_bar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to_bar) : "r"(smem_u32(bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                 ::"r"(to), "f"(a), "f"(b), "r"(to_bar)
                 : "memory");
}

template <class E, int MODE, bool GRAD>
__global__ void __launch_bounds__(Ring<MODE>::kThreads, 1) k_class_ring(const __grid_constant__ ClassParams p) {
    using G = ClassGroup<E>;
    using R = Ring<MODE>;
    constexpr int N = G::N, J = R::kLaneGroups, kTeams = R::kTeams, kTeamWarps = R::kTeamWarps, kPassWarps = R::kPassWarps,
                  kNumberWarps = R::kNumberWarps, kRows = R::kRows, kWarpGroups = R::kWarpGroups, kStageGroups = R::kStageGroups,
                  kStageBytes = R::kStageBytes;
    constexpr bool kWhole = MODE == kClassLogp;
    __shared__ typename R::Shared sh;
    extern __shared__ __align__(128) unsigned char class_smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, depth = p.depth;
    const int C = p.cluster, shift = __ffs(C) - 1, rank = C > 1 ? int(cluster_rank()) : 0, q = blockIdx.x / C, Q = gridDim.x / C;
    volatile int* abort_flag = &sh.abort_word;
    if (tid == 0) {
        sh.abort_word = 0;
        for (int i = 0; i < kTeams * R::kDepth; ++i) {
            mbar_init(&sh.full[0][0] + i, 1);
            mbar_init(&sh.free[0][0] + i, kTeamWarps);
        }
        for (int i = 0; i < kRows; ++i) {
            mbar_init(sh.summed + i, kTeamWarps);
            mbar_init(sh.ready + i, 1);
            mbar_init(sh.written + i, kTeamWarps);
        }
        for (int i = 0; i < 2 * kRows; ++i) mbar_init(sh.joined + i, 1);
        fence_mbar_init();
    }
    __syncthreads();
    if (C > 1) cluster_barrier();                   // who writes into another CTA's shared memory has to find it started
    grid_dependency_wait();
    const bool known = p.order || p.listed;         // which rows count
    if (p.listed) class_list<MODE>(p, sh.list, q, Q, rank == 0);
    const int live = p.listed ? sh.list.all : p.order ? p.prep->live : int(p.T);
    const int mine = live > q ? (live - q + Q - 1) / Q : 0;
    auto row_of = [&](int k) -> int {
        const long long at = q + static_cast<long long>(k) * Q;
        if (k >= mine || !known) return static_cast<int>(at);
        if (p.listed) return sh.list.live[k];
        int t;                                      // (volatile: fetched here, well before it is needed)
        asm volatile("ld.global.b32 %0, [%1];" : "=r"(t) : "l"(p.order + at));
        return t;
    };
    auto stages_of = [&](int groups) {              // of this CTA: every C-th
        const int all = (groups + kStageGroups - 1) / kStageGroups;
        return all > rank ? (all - rank + C - 1) >> shift : 0;
    };
    if (warp >= kPassWarps && warp < kPassWarps + kTeams) {
        if (lane == 0) {
            const int team = warp - kPassWarps;
            uint64_t *full = sh.full[team], *free = sh.free[team];
            unsigned char* ring = class_smem + team * depth * kStageBytes;
            // what is read again, by a later pass or because the ring cannot hold it, may stay in L2
            const uint64_t again_policy = l2_policy_evict_normal(), once = MODE == kClassLogp && p.stat ? again_policy : l2_policy_evict_first();
            int slot = 0, parity = 0, copies = 0;
            bool ok = true;
            int t = row_of(team);
            for (int k = team; k < mine && ok; k += kTeams) {
                const ClassRow<E> row(p.x, p.ld, nullptr, 0, t, p.V);
                t = row_of(k + kTeams);
                const int stages = stages_of(row.groups), again = GRAD ? max(0, stages - depth) : 0;
                for (int i = 0; i < stages + again; ++i) {
                    const int first = ((i < stages ? i : i - stages) * C + rank) * kStageGroups;
                    const uint32_t bytes = min(kStageGroups, row.groups - first) * 16;
                    if (copies >= depth && !mbar_wait_bounded(free + slot, parity ^ 1, abort_flag)) {
                        ok = false;
                        break;
                    }
                    fence_proxy_async_smem();
                    mbar_arrive_expect_tx(full + slot, bytes);
                    bulk_copy_g2s(ring + slot * kStageBytes, row.x + row.head + static_cast<long long>(first) * N, bytes, full + slot, i < again ? again_policy : once);
                    if (copies < depth) ++copies;
                    if (++slot == depth) {
                        slot = 0;
                        parity ^= 1;
                    }
                }
            }
            // whatever happened, the copies have to land before the shared memory is given up
            for (; copies > 0; --copies) {
                if (slot == 0) {
                    slot = depth;
                    parity ^= 1;
                }
                mbar_wait_drain(full + --slot, parity);
            }
        }
    } else if (warp < kPassWarps) {
        const int team = warp / kTeamWarps, in_team = warp % kTeamWarps;
        uint64_t *full = sh.full[team], *free = sh.free[team];
        const unsigned char* ring = class_smem + team * depth * kStageBytes + (in_team * kWarpGroups + lane) * 16;
        int slot = 0, parity = 0;                   // of the copy that comes next
        bool ok = true;
        auto wait = [&](uint64_t* bar, int parity_now) {
            if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar, parity_now, abort_flag))) ok = false;
        };
        auto next_slot = [&]() {
            if (++slot == depth) {
                slot = 0;
                parity ^= 1;
            }
        };
        auto read_stage = [&](int at, uint4 (&raw)[J]) {
#pragma unroll
            for (int j = 0; j < J; ++j) raw[j] = *reinterpret_cast<const uint4*>(ring + at * kStageBytes + j * 512);
        };
        auto give_back = [&](int at) {              // what is in registers now may be overwritten
            __syncwarp();
            if (lane == 0 && ok) mbar_arrive(free + at);           // (where a wait ran out the copy may still be on its way)
        };
        int t_next = row_of(team);
        for (int k = team; k < mine && ok; k += kTeams) {
            const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t_next, p.V);
            t_next = row_of(k + kTeams);
            const int stages = stages_of(row.groups), dropped = GRAD ? max(0, stages - depth) : stages;
            const int at = k % kRows;
            ClassSum sum;
            int held = slot;                        // the first stage that is kept
            for (int i = 0; i < stages; ++i) {
                const int left = row.groups - (i * C + rank) * kStageGroups - in_team * kWarpGroups;
                wait(full + slot, parity);
                uint4 raw[J];
                read_stage(slot, raw);
                if (i < dropped) give_back(slot);
                next_slot();
                if (i + 1 == dropped) held = slot;
                if (left <= 0) continue;
                if (left < kWarpGroups) {
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        if (32 * j + lane >= left) raw[j] = G::nothing();
                }
                sum.add_groups<E, J, kWhole>(raw, p.cs);
            }
            sum.over_warp<kWhole>(p.cs);
            if (!GRAD && k >= kRows) wait(sh.ready + at, (k / kRows - 1) & 1);      // the sums of row k - kRows have been read
            if (lane == 0) {
                sh.warp_sum[at][in_team] = make_float2(sum.top, sum.s);
                mbar_arrive(sh.summed + at);
            }
            if (!GRAD) continue;
            wait(sh.ready + at, (k / kRows) & 1);
            if (!ok) break;
            const float2 numbers = sh.row[at];
            const bool zero_row = numbers.x == 0.0f;       // it does not count, or has no teacher: whatever its logits hold
            const uint64_t c2 = f32x2_pack(p.c, p.c), top2 = f32x2_pack(-numbers.y, -numbers.y), factor2 = f32x2_pack(numbers.x, numbers.x);
            auto second = [&](int i, int from) {
                const int first = (i * C + rank) * kStageGroups + in_team * kWarpGroups, left = row.groups - first;
                uint4 raw[J];
                read_stage(from, raw);
                give_back(from);
                E* out = row.dx + row.head + (first + lane) * N;
                auto group = [&](int j) {
                    uint64_t v[G::P];
#pragma unroll
                    for (int e = 0; e < G::P; ++e) v[e] = f32x2_mul(class_powers(G::pair(raw[j], e), top2, c2), factor2);
                    row.store_at(out + 32 * N * j, v);
                };
                if (zero_row) {
                    const uint64_t zero[G::P] = {};
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        if (32 * j + lane < left) row.store_at(out + 32 * N * j, zero);
                } else if (left >= kWarpGroups) {
#pragma unroll
                    for (int j = 0; j < J; ++j) group(j);
                } else {
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        if (32 * j + lane < left) group(j);
                }
            };
            for (int i = dropped; i < stages; ++i) {
                second(i, held);
                if (++held == depth) held = 0;
            }
            for (int i = 0; i < dropped; ++i) {
                wait(full + slot, parity);
                second(i, slot);
                next_slot();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sh.written + at);
        }
    } else {
        const int h = warp - kPassWarps - kTeams;
        ClassTop top{};
        if (MODE == kClassDistill) {
            top = class_top_at(class_smem + kTeams * depth * kStageBytes + h * class_top_bytes(p.K), p.K);
            class_clear_marks(top);
        }
        double sums[3] = {0.0, 0.0, 0.0}, inv = 0.0;
        if (MODE != kClassLogp) {
            double n = p.norm;
            if (n == 0.0) n = p.listed ? sh.list.total : p.order ? p.prep->norm : warp_sum64(class_norm_part<MODE>(p, 0, p.T, lane, 32));
            inv = n == 0.0 ? 0.0 : 1.0 / n;
        }
        const ClassSpan span = MODE == kClassLogp && !known ? class_warp_span(p) : ClassSpan{};
        bool ok = true;
        auto wait = [&](uint64_t* bar, int parity) {
            if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag))) ok = false;
            return ok;
        };
        // this cluster's rows that do not count, in pieces of kZeroGroups groups; row k's turn is piece pieces * k / mine and on
        constexpr int kZeroGroups = 512;
        const int dead = known ? max(0, (int(p.T) - live - q + Q - 1) / Q) : 0, per_row = (p.V / N + kZeroGroups * C) / (kZeroGroups * C);
        auto zero_pieces = [&](long long first, long long last) {
            const uint64_t zero[G::P] = {};
            for (; first < last; ++first) {
                const int i = static_cast<int>(first / per_row), piece = static_cast<int>(first - static_cast<long long>(i) * per_row);
                const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, p.listed ? sh.list.dead[i] : __ldg(p.order + live + q + static_cast<long long>(i) * Q), p.V);
                const int start = (piece * C + rank) * kZeroGroups, end = min(start + kZeroGroups, row.groups);
                for (int g = start + lane; g < end; g += 32) row.store(g, zero);
                if (piece == 0 && rank == 0 && lane < row.edges) store_from_float(row.dx + row.edge(lane), 0.0f);
            }
        };
        const long long pieces = static_cast<long long>(dead) * per_row;
        auto zeros = [&](int k) {
            if (dead > 0) zero_pieces(pieces * k / mine, pieces * (k + 1) / mine);
        };
        if (GRAD && mine == 0) zero_pieces(pieces * h / kNumberWarps, pieces * (h + 1) / kNumberWarps);
        for (int k = h; k < mine; k += kNumberWarps) {
            const long long t = row_of(k);
            const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
            ClassInputs in{};
            bool counts = class_counts(p, t, MODE, &in.target, &in.w);
            if (MODE == kClassLogp && !known) counts = counts && span.has(t);
            const bool edges = rank == 0 && lane < row.edges;
            const float edge = counts && edges ? load_local(row.x + row.edge(lane)) : 0.0f;
            if (MODE == kClassDistill && k + kNumberWarps < mine) class_top_ahead(p, row_of(k + kNumberWarps));
            if (counts) class_inputs<MODE>(p, t, row.x, top, in);
            const int at = k % kRows, parity = (k / kRows) & 1;
            if (!wait(sh.summed + at, parity)) break;
            ClassSum sum;
            if (lane < kTeamWarps) sum = ClassSum{sh.warp_sum[at][lane].x, sh.warp_sum[at][lane].y};
            if (edges) sum.add<kWhole>(edge, p.cs);
            sum.over_warp<kWhole>(p.cs);
            if (C > 1) {
                // The gradient may replace the logits, and a CTA that has all sums writes over the target's: what this one reads of the row has to be
                // here before its sum goes out.  Edges are in the sum and a teacher's classes in shared memory; the target's logit is
                // made part of what is sent (where it is no number, neither is the sum).
                if (MODE == kClassPolicy && in.xy != in.xy) sum.s = in.xy;
                const int at2 = k % (2 * kRows);
                if (lane == 0) mbar_arrive_expect_tx(sh.joined + at2, 8 * C);
                __syncwarp();
                if (lane < C) send_f32x2(&sh.cta_sum[at2][rank], sh.joined + at2, lane, sum.top, sum.s);
                if (!wait(sh.joined + at2, (k / (2 * kRows)) & 1)) break;
                sum = ClassSum{};
                if (lane < C) sum = ClassSum{sh.cta_sum[at2][lane].x, sh.cta_sum[at2][lane].y};
                sum.over_warp<kWhole>(p.cs);
            }
            sum.settle();
            ClassNumbers now{};
            ClassTerms terms;
            if (counts) now = class_numbers<MODE>(p, in, sum, inv, terms);
            if (lane == 0) {
                if (GRAD) sh.row[at] = make_float2(now.factor, sum.top);
                mbar_arrive(sh.ready + at);
            }
            if (counts) class_account<MODE>(p, t, in, sum, terms, rank == 0 && lane == 0, sums);
            else if (rank == 0 && lane == 0) class_dead_row<MODE>(p, t);
            if (MODE == kClassDistill && C > 1 && k + kNumberWarps < mine) class_top_logits_ahead<E>(p, row_of(k + kNumberWarps), rank);
            if (!GRAD) continue;
            zeros(k);
            if (edges) store_from_float(row.dx + row.edge(lane), now.factor != 0.0f ? class_power(edge, sum.top, p.c) * now.factor : 0.0f);
            // the values at the targets replace what the passes have written, in this CTA's stages
            if (!wait(sh.written + at, parity)) break;
            if (!counts) continue;
            auto here = [&](int column) {
                const int g = (column - row.head) / N;
                return column < row.head || g >= row.groups ? rank == 0 : (g / kStageGroups & (C - 1)) == rank;
            };
            if (MODE == kClassPolicy) {
                __syncwarp();
                if (lane == 0 && here(int(in.target))) store_from_float(row.dx + in.target, now.at);
            } else {
                __syncwarp();
                for (int j = lane; j < p.K; j += 32)
                    if (top.id[j] >= 0 && here(top.id[j])) store_from_float(row.dx + top.id[j], class_top_value(p, top, j, in.top.twice, sum.top, now));
                __syncwarp();
            }
        }
        if (MODE != kClassLogp && rank == 0) class_finish<MODE>(p, q * kNumberWarps + h, Q * kNumberWarps, inv, sums);
    }
    __syncwarp();
    if (C > 1) cluster_barrier();                   // what was sent has arrived before a CTA's shared memory is given up
    if (tid == 0 && *abort_flag) atomicExch(p.timeout, kStatusTimeout);
}

// ---- short rows ----------------------------------------------------------------------------------------
// A warp per row, the row in its registers between the passes: no barrier, no shared memory but for a teacher's classes.  Up to four groups a
// lane the next row's logits are on their way meanwhile, and always its target.  A row takes about 600 instructions beside 8 a logit and lane
// (its numbers, set up and stored by a whole warp), which k_class_bundle shares among rows of up to 1024 logits where there are many; they
// depend on one another, and 16 to 32 warps an SM do not hide that.  32768 rows of 1000 bfloat16: distillation of 16 classes 54 us (its bytes
// take 21); of 2000, log-probabilities 34 (20); of 4000, policy loss 121 (80).
constexpr int kShortWarps = 8;
__host__ __device__ constexpr int short_ctas(int mode, int J) { return J <= 2 && mode != kClassDistill ? 4 : J <= 8 ? 3 : 2; }       // per SM, in registers

// (by all threads of a CTA)
template <int MODE>
__device__ __forceinline__ double short_inverse_norm(const ClassParams& p) {
    if (MODE == kClassLogp) return 0.0;
    __shared__ double warp_part[kShortWarps];
    double n = p.norm;
    if (n == 0.0 && p.norm_parts > 0) {
        for (int i = threadIdx.x & 31; i < p.norm_parts; i += 32) n += __ldcg(p.norm_part + i);
        n = warp_sum64(n);
    } else if (n == 0.0) {
        n = warp_sum64(class_norm_part<MODE>(p, 0, p.T, threadIdx.x, kShortWarps * 32));
        if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = n;
        __syncthreads();
        n = 0.0;
        for (int w = 0; w < kShortWarps; ++w) n += warp_part[w];
    }
    return n == 0.0 ? 0.0 : 1.0 / n;
}
// Every warp's sums, the same in all of its lanes, to the outputs
template <int MODE>
__device__ __forceinline__ void short_finish(const ClassParams& p, double inv, double (&sums)[3]) {
    __shared__ double cta_part[kShortWarps][3];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (MODE == kClassLogp) return;
    if (lane == 0)
        for (int i = 0; i < 3; ++i) cta_part[warp][i] = sums[i];
    __syncthreads();
    if (warp != 0) return;
    for (int i = 0; i < 3; ++i) {
        sums[i] = 0.0;
        for (int w = 0; w < kShortWarps; ++w) sums[i] += cta_part[w][i];
    }
    class_finish<MODE>(p, blockIdx.x, gridDim.x, inv, sums);
}

template <class E, int MODE, bool GRAD, int J>
__global__ void __launch_bounds__(kShortWarps * 32, short_ctas(MODE, J)) k_class_short(const __grid_constant__ ClassParams p) {
    using G = ClassGroup<E>;
    constexpr bool kAhead = J <= 4 && MODE != kClassDistill;
    constexpr int B = J < 4 ? J : 4;                // groups that are worked on together
    extern __shared__ __align__(128) unsigned char class_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    ClassTop top{};
    if (MODE == kClassDistill) {
        top = class_top_at(class_smem + warp * class_top_bytes(p.K), p.K);
        class_clear_marks(top);
    }
    grid_dependency_wait();
    const ClassSpan span = MODE == kClassLogp ? class_warp_span(p) : ClassSpan{};
    struct Row {
        ClassInputs in;
        uint4 raw[J];
        float edge;
        bool counts;
    };
    auto look = [&](long long t, Row& r) {          // its target and weight
        r.counts = false;
        if (t >= p.T) return;
        r.counts = class_counts(p, t, MODE, &r.in.target, &r.in.w);
        if (MODE == kClassLogp) r.counts = r.counts && span.has(t);
    };
    auto load = [&](long long t, Row& r) {          // its logits and what goes with them
        if (!r.counts) return;
        const ClassRow<E> row(p.x, p.ld, nullptr, 0, t, p.V);
#pragma unroll
        for (int j = 0; j < J; ++j) r.raw[j] = 32 * j + lane < row.groups ? row.load(32 * j + lane) : G::nothing();
        r.edge = lane < row.edges ? load_local(row.x + row.edge(lane)) : 0.0f;
        if (MODE != kClassDistill) class_inputs<MODE>(p, t, row.x, top, r.in);
    };
    double sums[3] = {0.0, 0.0, 0.0};
    const long long step = static_cast<long long>(gridDim.x) * kShortWarps;
    long long t = static_cast<long long>(blockIdx.x) * kShortWarps + warp;
    Row now{}, next{};
    look(t, now);
    load(t, now);
    look(t + step, next);
    const double inv = short_inverse_norm<MODE>(p); // (beside the first row's loads)
    for (; t < p.T; t += step) {
        Row after{};
        if (kAhead) {
            load(t + step, next);
            look(t + 2 * step, after);
        }
        const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
        auto zeros = [&] {
            const uint64_t zero[G::P] = {};
            for (int g = lane; g < row.groups; g += 32) row.store(g, zero);
            if (lane < row.edges) store_from_float(row.dx + row.edge(lane), 0.0f);
        };
        if (now.counts) {
            if (MODE == kClassDistill) class_inputs<MODE, 2>(p, t, row.x, top, now.in);
            ClassSum sum;
#pragma unroll
            for (int b = 0; b < J / B; ++b)
                if (32 * B * b < row.groups) sum.add_groups<E, B, false>(reinterpret_cast<const uint4(&)[B]>(now.raw[B * b]), p.cs);
            if (lane < row.edges) sum.add<false>(now.edge, p.cs);
            sum.over_warp<false>(p.cs);
            sum.settle();
            ClassTerms terms;
            const ClassNumbers numbers = class_numbers<MODE>(p, now.in, sum, inv, terms);
            class_account<MODE>(p, t, now.in, sum, terms, lane == 0, sums);
            if (GRAD && MODE == kClassDistill && numbers.factor == 0.0f) {
                zeros();                            // without a teacher, whatever the logits hold
            } else if (GRAD) {
                const uint64_t c2 = f32x2_pack(p.c, p.c), top2 = f32x2_pack(-sum.top, -sum.top), factor2 = f32x2_pack(numbers.factor, numbers.factor);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if (32 * j + lane < row.groups) {
                        uint64_t v[G::P];
#pragma unroll
                        for (int e = 0; e < G::P; ++e) v[e] = f32x2_mul(class_powers(G::pair(now.raw[j], e), top2, c2), factor2);
                        row.store(32 * j + lane, v);
                    }
                }
                if (lane < row.edges) store_from_float(row.dx + row.edge(lane), class_power(now.edge, sum.top, p.c) * numbers.factor);
            }
            if (GRAD) {
                __syncwarp();                       // the targets' values replace what was just written
                if (MODE == kClassPolicy) {
                    if (lane == 0) store_from_float(row.dx + now.in.target, numbers.at);
                } else {
                    for (int j = lane; j < p.K; j += 32)
                        if (top.id[j] >= 0) store_from_float(row.dx + top.id[j], class_top_value(p, top, j, now.in.top.twice, sum.top, numbers));
                    __syncwarp();
                }
            }
        } else {
            if (GRAD) zeros();
            if (lane == 0) class_dead_row<MODE>(p, t);
        }
        if (!kAhead) {
            load(t + step, next);
            look(t + 2 * step, after);
        }
        now = next;
        next = after;
    }
    short_finish<MODE>(p, inv, sums);
}

// R rows per warp and turn: their numbers are worked out at the same time, by 32 / R lanes each, which the sums reach by exchanging halves; a row's
// terms stay in registers for the gradient, 64 a lane at most.  Bound by waiting: a turn loads its rows' logits after their targets, nothing of the
// next turn but its targets is on the way, 16 warps an SM have no other work, and no unit is full (powers 31 %, ALU 37 %).  32768 rows of 1000
// bfloat16, policy loss 41 us (a warp per row: 53; its bytes take 20); of 200, 21 (33; 4); of 256, log-probabilities 9.8 (15.4; 2.6).  With rows for one
// CTA per SM or less a warp per row is faster (500 bfloat16, policy loss: 64 rows 7.1 us instead of 8.9, 600 rows 8.2 instead of 9.1, 2000 rows
// 11.5 instead of 11.2, 4000 rows 14.1 instead of 11.7).  Three CTAs per SM spill with a gradient (32768 x 1000: 55 us).
template <class E>
__host__ __device__ constexpr int bundle_rows(int J) {
    return J * ClassGroup<E>::N <= 16 ? 4 : 64 / (J * ClassGroup<E>::N);
}
__host__ __device__ constexpr int bundle_ctas(bool grad) { return grad ? 2 : 3; }          // per SM, in registers

template <class E, int MODE, bool GRAD, int J>
__global__ void __launch_bounds__(kShortWarps * 32, bundle_ctas(GRAD)) k_class_bundle(const __grid_constant__ ClassParams p) {
    using G = ClassGroup<E>;
    constexpr int R = bundle_rows<E>(J), W = 32 / R;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = lane / W;
    const bool writes = (lane & (W - 1)) == 0;      // lanes part * W ... belong to row `first + part`
    grid_dependency_wait();
    const ClassSpan span = MODE == kClassLogp ? class_warp_span(p) : ClassSpan{};
    struct Look {
        long long target;
        float w;
        bool counts;
    };
    auto look = [&](long long t) {
        Look l{0, 0.0f, false};
        if (t >= p.T) return l;
        l.counts = class_counts(p, t, MODE, &l.target, &l.w);
        if (MODE == kClassLogp) l.counts = l.counts && span.has(t);
        return l;
    };
    double sums[3] = {0.0, 0.0, 0.0};
    const long long step = static_cast<long long>(gridDim.x) * kShortWarps * R;
    long long first = (static_cast<long long>(blockIdx.x) * kShortWarps + warp) * R;
    Look now = look(first + part);
    const double inv = short_inverse_norm<MODE>(p);
    for (; first < p.T; first += step) {
        const long long t = first + part;
        const unsigned live = __ballot_sync(0xffffffffu, now.counts);
        uint4 raw[R][J];
        float edge[R], top[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool counts = live >> (r * W) & 1;
            const ClassRow<E> row(p.x, p.ld, nullptr, 0, first + r, p.V);
#pragma unroll
            for (int j = 0; j < J; ++j) raw[r][j] = counts && 32 * j + lane < row.groups ? row.load(32 * j + lane) : G::nothing();
            edge[r] = counts && lane < row.edges ? load_local(row.x + row.edge(lane)) : -INFINITY;
        }
        ClassInputs in{};
        in.target = now.target;
        in.w = now.w;
        if (now.counts) class_inputs<MODE>(p, t, static_cast<const E*>(p.x) + t * p.ld, ClassTop{}, in);
        const Look next = look(t + step);
        uint64_t term[R][J][G::P];
        float s[R];
        const uint64_t c2 = f32x2_pack(p.c, p.c);
#pragma unroll
        for (int r = 0; r < R; ++r) {               // -inf and no term: rows that do not count
            top[r] = warp_largest(fmaxf(G::template largest<J>(raw[r]), edge[r]));
            if (top[r] == -INFINITY) top[r] = 0.0f;
            const uint64_t top2 = f32x2_pack(-top[r], -top[r]);
            uint64_t two[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < G::P; ++i) {
                    term[r][j][i] = class_powers(G::pair(raw[r][j], i), top2, c2);
                    two[i & 1] = f32x2_add(two[i & 1], term[r][j][i]);
                }
            edge[r] = class_power(edge[r], top[r], p.c);
            float lo, hi;
            f32x2_unpack(f32x2_add(two[0], two[1]), lo, hi);
            s[r] = lo + hi + edge[r];
        }
        ClassSum sum;
        sum.top = top[0];
#pragma unroll
        for (int r = 1; r < R; ++r) sum.top = part == r ? top[r] : sum.top;
#pragma unroll
        for (int d = R / 2; d >= 1; d >>= 1)
#pragma unroll
            for (int r = 0; r < d; ++r) {           // the upper half of the lanes takes the upper half of the rows
                const bool up = part & d;
                const float give = up ? s[r] : s[r + d];
                s[r] = (up ? s[r + d] : s[r]) + __shfl_xor_sync(0xffffffffu, give, d * W);
            }
        sum.s = s[0];
#pragma unroll
        for (int d = W / 2; d >= 1; d >>= 1) sum.s += __shfl_xor_sync(0xffffffffu, sum.s, d);
        ClassTerms terms;
        const ClassNumbers numbers = class_numbers<MODE, W>(p, in, sum, inv, terms);
        if (now.counts) class_account<MODE>(p, t, in, sum, terms, writes, sums);
        else if (writes && t < p.T) class_dead_row<MODE>(p, t);
        if (GRAD) {
            const float own = now.counts ? numbers.factor : 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (first + r >= p.T) break;
                const float factor = __shfl_sync(0xffffffffu, own, r * W);
                const uint64_t factor2 = f32x2_pack(factor, factor);
                const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, first + r, p.V);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if (32 * j + lane < row.groups) {
                        uint64_t v[G::P];
#pragma unroll
                        for (int i = 0; i < G::P; ++i) v[i] = f32x2_mul(term[r][j][i], factor2);
                        row.store(32 * j + lane, v);
                    }
                }
                if (lane < row.edges) store_from_float(row.dx + row.edge(lane), edge[r] * factor);
            }
            __syncwarp();                           // the targets' values replace what was just written
            if (now.counts && writes) store_from_float(static_cast<E*>(p.dx) + t * p.ld_d + in.target, numbers.at);
        }
        now = next;
    }
#pragma unroll
    for (int d = W; d < 32; d *= 2)
        for (int i = 0; i < 3; ++i) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], d);
    short_finish<MODE>(p, inv, sums);
}

// norm_part[b] = sum of the weights of the rows that count among rows b * norm_rows ...
constexpr int kNormThreads = 256;

template <int MODE>
__global__ void __launch_bounds__(kNormThreads) k_class_norm(const __grid_constant__ ClassParams p, double* part) {
    __shared__ double warp_part[kNormThreads / 32];
    grid_dependency_release();
    const long long first = blockIdx.x * p.norm_rows, last = min(first + p.norm_rows, p.T);
    double sum = class_norm_part<MODE>(p, first, last, threadIdx.x, kNormThreads);
    sum = warp_sum64(sum);
    if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = 0.0;
        for (int w = 0; w < kNormThreads / 32; ++w) sum += warp_part[w];
        part[blockIdx.x] = sum;
    }
}

// ---- gradient of log-probabilities ---------------------------------------------------------------------
// Rows whose statistics are known: from the caller (lse, fp32) or from an earlier pass (top and s).  One read, one write: bound by HBM.  A CTA
// takes 16 KB of a row at a time, all loads on their way before the first power (with two groups a thread 444 us instead of 349), and steps
// through the pieces without a division.  8192 x 65536 bfloat16 337 us, 6.4 TB/s; under the power cap of a long run 373.
struct ClassGradParams {
    const void* x;
    long long ld;
    long long T;
    int V;
    const void* ids;
    int wide_ids;
    long long ignore;
    float c;
    double c64;
    float scale;
    const float* lse;
    const float2* stat;
    const float* g;
    void* dx;
    long long ld_d;
    int* status;                 // NULL: targets outside the classes have been reported
    int slices;                  // of a row
    int backwards;               // from the last row on: what was read last may still be in L2
};

constexpr int kClassGradThreads = 256;
constexpr int kClassGradGroups = 4;                 // per thread, all on their way before the first is worked on

template <class E>
__global__ void __launch_bounds__(kClassGradThreads) k_class_grad(const __grid_constant__ ClassGradParams p) {
    using G = ClassGroup<E>;
    constexpr int N = G::N, U = kClassGradGroups;
    const int tid = threadIdx.x, threads = blockDim.x;
    grid_dependency_wait();
    struct Numbers {             // of a row
        long long target;
        float g;
        float2 stat;
    };
    // slice `slice` of row t, and what comes gridDim.x pieces later
    auto row_of = [&](long long t) { return p.backwards ? p.T - 1 - t : t; };
    auto fetch = [&](long long t) {
        Numbers n{};
        if (t < p.T) {
            t = row_of(t);
            n.target = load_any_id(p.ids, p.wide_ids, t);
            n.g = p.g[t];
            n.stat = p.stat ? p.stat[t] : make_float2(p.lse[t], 0.0f);
        }
        return n;
    };
    const int rows = gridDim.x / p.slices, rest = gridDim.x % p.slices;
    long long next_t = blockIdx.x / p.slices;
    int next_slice = blockIdx.x % p.slices;
    Numbers next = fetch(next_t);
    while (next_t < p.T) {
        const Numbers now = next;
        const long long t = row_of(next_t);
        const int slice = next_slice;
        next_t += rows;
        next_slice += rest;
        if (next_slice >= p.slices) {
            next_slice -= p.slices;
            ++next_t;
        }
        next = fetch(next_t);
        const ClassRow<E> row(p.x, p.ld, p.dx, p.ld_d, t, p.V);
        const float gt = now.g * p.scale;
        bool live = now.target != p.ignore && gt != 0.0f;
        if (now.target != p.ignore && (now.target < 0 || now.target >= p.V)) {
            live = false;
            if (p.status && tid == 0) atomicExch(p.status, -4);
        }
        const int first = slice * threads * U + tid;
        const bool edges = slice == 0 && tid < row.edges;
        if (!live) {
            const uint64_t zero[G::P] = {};
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (first + u * threads < row.groups) row.store(first + u * threads, zero);
            if (edges) store_from_float(row.dx + row.edge(tid), 0.0f);
            continue;
        }
        const E* in = row.x + row.head + first * N;
        E* out = row.dx + row.head + first * N;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * threads < row.groups) raw[u] = *reinterpret_cast<const uint4*>(in + u * threads * N);
        float base, k;
        if (p.stat) {
            base = now.stat.x;
            k = -gt / now.stat.y;
        } else {                                    // lse / scale in place of the largest logit, the part below fp32 put into the factor
            const ClassBase own = class_base(now.stat.x, p.scale, p.c64);
            base = own.high;
            k = -gt * exp2_fast(kPowerLift - own.low);
        }
        const int where = static_cast<int>(now.target) - row.head;
        const uint64_t c2 = f32x2_pack(p.c, p.c), base2 = f32x2_pack(-base, -base), k2 = f32x2_pack(k, k);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int g = first + u * threads;
            if (g >= row.groups) break;
            uint64_t v[G::P];
#pragma unroll
            for (int j = 0; j < G::P; ++j) v[j] = f32x2_mul(class_powers(G::pair(raw[u], j), base2, c2), k2);
            if (where >= g * N && where < g * N + N) {
#pragma unroll
                for (int j = 0; j < G::P; ++j) {
                    const int at = where - g * N - 2 * j;
                    v[j] = f32x2_add(v[j], f32x2_pack(at == 0 ? gt : 0.0f, at == 1 ? gt : 0.0f));
                }
            }
            row.store_at(out + u * threads * N, v);
        }
        if (edges) {
            const int at = row.edge(tid);
            const float v = class_power(load_local(row.x + at), base, p.c) * k;
            store_from_float(row.dx + at, at == now.target ? v + gt : v);
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

// One CTA per pair, the two sequences by half of it each; the last CTA adds the pairs up.  Bound by latency: 4 us for a pair of 150 tokens.
__global__ void __launch_bounds__(kPairThreads) k_class_pair(const __grid_constant__ ClassPairParams p) {
    __shared__ double warp_part[kPairThreads / 32][2];
    __shared__ double total[3];
    __shared__ bool last_cta;
    const int tid = threadIdx.x, warp = tid >> 5, side = tid >= kPairThreads / 2, lane = tid & (kPairThreads / 2 - 1);
    grid_dependency_release();
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
        const float w = p.weights ? __ldg(p.weights + pair) : 1.0f;
        const double ref = p.ref ? static_cast<double>(__ldg(p.ref + pair)) - static_cast<double>(__ldg(p.ref + p.P + pair)) : 0.0;
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
        double s[2], rows[2];
        for (int j = 0; j < 2; ++j) {
            s[j] = 0.0;
            rows[j] = 0.0;
            for (int i = 0; i < kPairThreads / 64; ++i) {
                s[j] += warp_part[j * (kPairThreads / 64) + i][0];
                rows[j] += warp_part[j * (kPairThreads / 64) + i][1];
            }
            if (!p.average || rows[j] == 0.0) rows[j] = 1.0;
            s[j] /= rows[j];
        }
        if (tid == 0) {
            const double h = p.beta * (s[0] - s[1] - ref) - p.margin;
            // log sigmoid(h) = -softplus(-h), log sigmoid(-h) = -softplus(h); t = exp(-|h|) and what follows from it in fp32 (see logistic_terms)
            // An h that is infinite (a sequence without probability) or past fp32 has t = 0; a term without weight is left out, infinite or not.
            const float size = fabsf(static_cast<float>(h)), t = size > 104.0f ? 0.0f : expf(-size) * (1.0f - static_cast<float>(fabs(h) - size)),
                        one = 1.0f / (1.0f + t);
            const double soft = log1pf(t), plus = fmax(h, 0.0) + soft, minus = fmax(-h, 0.0) + soft;
            const float right = h >= 0.0 ? one : t * one, wrong = h >= 0.0 ? t * one : one;
            const double loss = (p.smoothing < 1.0 ? (1.0 - p.smoothing) * minus : 0.0) + (p.smoothing > 0.0 ? p.smoothing * plus : 0.0);
            p.pair_loss[pair] = w == 0.0f ? 0.0 : w * loss;
            p.h[pair] = static_cast<float>(h);
            if (p.seq_logp) {
                p.seq_logp[pair] = static_cast<float>(s[0]);
                p.seq_logp[p.P + pair] = static_cast<float>(s[1]);
            }
            total[0] = w == 0.0f ? 0.0 : w * inv * p.factor * p.beta * (p.smoothing * right - (1.0 - p.smoothing) * wrong);
        }
        __syncthreads();
        const float g = static_cast<float>((side ? -total[0] : total[0]) / rows[side]);
        // (added to 0: falling offsets may put a row into several sequences)
        for (long long t = a + lane; t < z; t += kPairThreads / 2) atomicAdd(p.coef + t, g);
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
