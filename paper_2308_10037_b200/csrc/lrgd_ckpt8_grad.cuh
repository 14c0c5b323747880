// Gradient of a C-class logistic layer from rows kept in 8 bits, on the tensor cores:
//
//   grad_w[c,j] (+)= sum_t (dz[t,c] * s[t,g]) * q[t,j]   for the columns j of group g,      grad_b[c] (+)= sum_t dz[t,c]
//
// As a matrix product, D[j,(c)] = sum over t of A[j,t] B[t,c] with A = q^T, B = dz * s: the sum index is the row t, and the scale
// differs from one group of 128 columns to the next, so B is formed per group.  An int8 is exact in bfloat16; the fp32 factor
// x = dz * s is cut into three bfloat16 terms, the upper eight bits of x, of what is left and of what is then left, which hold its
// 24 bits exactly whatever its size beside other rows' (two terms would leave 2^-16 of every factor).  The terms stand side by side as
// 3 * CP columns of B, products accumulate in fp32 in tensor memory, and the three sums of a class are added when they are read back.
// So every product is a floating-point one: a row loses no bits to another row of a larger dz or scale.  Integers of a common step
// per class and group (four bytes a factor on the int8 products, 40 us at the size below) did lose them: beside one
// masked row whose scale was 1e6 times the others' the sums were off by a thousandth, so that form was taken out.
// 16384 x 4096, 64 classes: 53 us, k_ckpt8_join (6) included; two classes 41 us; the floor is 11 (74 MB).
//
// A CTA takes two groups (256 columns), one block of up to 64 classes and a range of rows, 32 rows per stage.  The raw q of a
// stage comes by TMA (a ring of kTcRing stages; by plain word loads where q is not 16-byte aligned).  Two sets of eight warps
// convert, one the even stages and one the odd ones: a warp turns 8 rows x 128 columns of q into bfloat16 and a thread 8 rows of one
// class of dz into 2 x 3 terms, written K-major (8 consecutive t of one column or class are 16 bytes) into one of three operand
// buffers.  A seventeenth warp issues the tcgen05.mma of a stage when its eight warps have arrived, an eighteenth the copies of a
// later stage: the scales, one row per lane, are fetched once per stage there (every warp gathering its own cost a quarter of
// the kernel's shared-memory bandwidth).
// What bounds it: the latency of the converting warps, of which the registers leave room for four per scheduler.  With 64 classes a warp
// takes 3,100 clocks per stage of its own: 830 to form and cut dz * s, 590 to widen q, 300 to fetch its next dz, 230 in the flushes, the
// rest waiting and publishing; issue slots are 64 % busy.  Stages of 64 rows (fewer of them, but spilled registers) took 59 us.
// No barrier spans the CTA inside the loop: the warps meet on mbarriers, so that loads, conversion and products overlap.
// Every kTcFlush stages the sums move from tensor memory to registers: the tensor cores drop the bits below the accumulator's last
// place, an error that grows with the length of the chain (114 steps: 1.2e-6 of the result; 32 steps: 2.3e-7).
// The rows are split over CTAs to fill the GPU; k_ckpt8_join adds the parts in order.
#pragma once
#include <cuda.h>

#include "lrgd_ckpt8.cuh"

namespace lrgd {

constexpr int kTcWarps = 16;                       // converting warps; one more issues the products, another one the copies
constexpr int kTcThreads = (kTcWarps + 2) * 32;
constexpr int kTcFlush = 16;                       // stages between two flushes of the accumulators
constexpr int kTcRows = 32;                        // rows per stage
constexpr int kTcBlocks = kTcRows / 8;             // blocks of eight rows: 16 bytes of an operand's row
constexpr int kTcBuffers = 3;
constexpr int kTcMaxClasses = 64;
constexpr int kTcRing = 12;
constexpr int kTcHeader = 4096;                    // barriers and flags (1 KB), then the scales of the ring's stages
constexpr int kTcOperandA = kCkptGroup * kTcRows * 2;              // bytes per group and buffer
constexpr int kTcRaw = kTcRows * kCkptGroup;       // bytes of raw q per group and stage
constexpr int tc_smem_bytes(int cp, bool tma) {
    const int need = kTcHeader + (tma ? kTcRing * 2 * kTcRaw : 0) + kTcBuffers * 2 * (kTcOperandA + 3 * cp * kTcRows * 2) + 1024;
    return need > 120 * 1024 ? need : 120 * 1024;   // more than half an SM's: one CTA per SM, which takes all of its tensor memory
}

struct CkptGradParams {
    const signed char* q;
    long long ld_q;
    const float* s;
    long long T;
    int n;
    int groups;
    const void* dz;
    long long ld_dz;
    int C;
    int chunks;
    long long rows;            // rows per chunk, a multiple of kTcRows
    int accumulate;
    float* part_w;             // [chunks][C][n]
    float* part_b;             // [chunks][C]
    float* grad_w;             // [C][n]
    float* grad_b;             // [C], nullable
};

struct TcGradParams {
    CkptGradParams g;
    int cp;                    // classes per block: a multiple of 16
    int* status;
};

__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t addr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Arrives on the barrier when every tcgen05.mma this thread has issued so far is complete.
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
        : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
// Shared-memory operand, K-major without swizzle: 8 rows x 16 bytes (8 values of K) are 128 contiguous bytes; `k_stride` bytes to
// the next 8 values of K, 128 bytes to the next 8 rows.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t k_stride) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(k_stride >> 4) << 16 | uint64_t(128 >> 4) << 32 | uint64_t(1) << 46;
}

// Two int8 (byte `i` of two words) to two bfloat16: the low seven bits under the exponent of 128 give 128 + (q & 127); a q >= 0
// then has 128 too much, a negative one 256.  Exact.
template <int I>
__device__ __forceinline__ uint32_t int8_pair_to_bf16(uint32_t w0, uint32_t w1) {
    const uint32_t p = __byte_perm(w0, w1, I | (4 + I) << 8);      // bytes 0 and 2; the others are masked off
    const uint32_t m = (p & 0x007f007fu) | 0x43004300u, b = (p & 0x00800080u) | 0x43004300u;
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(m), "r"(b));
    return r;
}
// The upper halves of (x0, x1) as packed bfloat16, and what is left of the two.  Cut off, not rounded: three times eight bits hold the 24
// of an fp32 number exactly, and the largest numbers do not become infinite.
__device__ __forceinline__ uint32_t split_term(float& x0, float& x1) {
    const uint32_t a = __float_as_uint(x0), b = __float_as_uint(x1);
    x0 -= __uint_as_float(a & 0xffff0000u);
    x1 -= __uint_as_float(b & 0xffff0000u);
    return __byte_perm(a, b, 0x7632);
}

template <class E, bool TMA>
__global__ void __launch_bounds__(kTcThreads, 1) k_ckpt8_grad_tc(const __grid_constant__ CUtensorMap map, const __grid_constant__ TcGradParams tp) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const CkptGradParams& p = tp.g;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);              // [kTcRing] raw q and the scales of a stage have landed
    uint64_t* empty = full + kTcRing;                                // [kTcRing] the eight warps of the stage have read them
    uint64_t* ready = empty + kTcRing;                               // [kTcBuffers] an operand buffer is written
    uint64_t* done = ready + kTcBuffers;                             // [kTcBuffers] the products that read it are complete
    uint64_t* flushed = done + kTcBuffers;                           // the accumulators have been read out
    uint32_t* tmem_at = reinterpret_cast<uint32_t*>(flushed + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);
    volatile int* issued_at = abort_flag + 1;
    const int cp = tp.cp, ncols = 3 * cp;
    const int op_b = 3 * cp * kTcRows * 2;                           // bytes per group and buffer
    float* scales = reinterpret_cast<float*>(smem + 1024);           // [kTcRing][2 groups][kTcRows]
    unsigned char* ring = smem + kTcHeader;
    unsigned char* opa = ring + (TMA ? kTcRing * 2 * kTcRaw : 0);    // [kTcBuffers][2 groups]
    unsigned char* opb = opa + kTcBuffers * 2 * kTcOperandA;         // [kTcBuffers][2 groups]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g0 = blockIdx.x * 2, groups = min(2, p.groups - g0);
    const int c0 = blockIdx.z * cp, classes = min(cp, p.C - c0);
    const long long lo = blockIdx.y * p.rows, hi = min(p.T, lo + p.rows);
    const int stages = static_cast<int>((hi - lo + kTcRows - 1) / kTcRows);

    if (tid == 0) {
        for (int i = 0; i < kTcRing; ++i) {
            mbar_init(full + i, TMA ? 2 : 1);
            mbar_init(empty + i, kTcWarps / 2);
        }
        for (int i = 0; i < kTcBuffers; ++i) {
            mbar_init(ready + i, kTcWarps / 2);
            mbar_init(done + i, 1);
        }
        mbar_init(flushed, kTcWarps);
        *abort_flag = 0;
        *issued_at = 0;
        fence_mbar_init();
    }
    if (warp == 0) tmem_alloc(tmem_at, 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    grid_dependency_release();                                       // k_ckpt8_join may be launched; it waits for this kernel's end
    const uint32_t tmem = *tmem_at;
    bool ok = true;
    float acc[kTcMaxClasses / 2];                                    // sums of this thread's column, (warp >> 2) & 1 its group
#pragma unroll
    for (int i = 0; i < kTcMaxClasses / 2; ++i) acc[i] = 0.0f;
    float zsum = 0.0f;
    const int fg = (warp >> 2) & 1, fhalf = warp >> 3;
    auto flush = [&] {                                               // accumulators -> acc: class 16 * i + 8 * fhalf + k in acc[8 * i + k]
        tmem_fence_after();
        if (fg < groups) {
#pragma unroll
            for (int i = 0; i < kTcMaxClasses / 16; ++i)
                if (16 * i < cp) {
                    float a[8], b[8], d[8];
                    const uint32_t at = tmem + (uint32_t((warp & 3) * 32) << 16) + fg * ncols + 16 * i + 8 * fhalf;
                    tmem_load8(at, a);
                    tmem_load8(at + cp, b);
                    tmem_load8(at + 2 * cp, d);
#pragma unroll
                    for (int k = 0; k < 8; ++k) acc[8 * i + k] += a[k] + (b[k] + d[k]);
                }
        }
        tmem_fence_before();
    };
    const int set = warp >> 3, sw = warp & 7, stid = tid & 255;      // set of eight warps, place in it
    const int zk = stid / cp, zc = stid - zk * cp;                   // this thread's part of dz: class c0 + zc, rows 8 * zk .. + 7
    const bool z_on = zk < kTcBlocks;

    if (warp == kTcWarps) {
        if (lane == 0) {
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(ncols / 8) << 17) | (uint32_t(kCkptGroup / 16) << 24);
            const uint64_t a0 = operand_desc(smem_u32(opa), kCkptGroup * 16), b0 = operand_desc(smem_u32(opb), ncols * 16);
            int stage = 0, buf = 0, parity = 0, sums = 0;
            for (; stage < stages; ++stage) {
                if (!mbar_wait_bounded(ready + buf, parity, abort_flag)) { ok = false; break; }
                const bool fresh = stage % kTcFlush == 0;            // the sums so far are taken out first
                if (fresh && stage > 0 && !mbar_wait_bounded(flushed, sums++ & 1, abort_flag)) { ok = false; break; }
                tmem_fence_after();
                for (int gi = 0; gi < groups; ++gi) {
                    // descriptors count in 16 bytes; 16 rows of the sum are two blocks of K
                    const uint64_t a = a0 + ((buf * 2 + gi) * kTcOperandA >> 4), b = b0 + ((buf * 2 + gi) * op_b >> 4);
#pragma unroll
                    for (int k = 0; k < kTcRows / 16; ++k)
                        mma_bf16(tmem + gi * ncols, a + k * 2 * kCkptGroup, b + k * 2 * ncols, idesc, !fresh || k > 0);
                }
                mma_commit(done + buf);
                if (++buf == kTcBuffers) { buf = 0; parity ^= 1; }
            }
            *issued_at = stage;
        }
    } else if (warp == kTcWarps + 1) {
        const uint64_t policy = l2_policy_evict_first();
        // lane: one row of the stage, both groups' scales
        float s0 = 0.0f, s1 = 0.0f;
        auto load_scales = [&](int stage) {
            const long long t = lo + static_cast<long long>(stage) * kTcRows + lane;
            const float* sp = p.s + t * p.groups + g0;
            s0 = stage < stages && t < hi ? __ldg(sp) : 0.0f;
            s1 = stage < stages && t < hi && groups > 1 ? __ldg(sp + 1) : 0.0f;
        };
        auto fetch = [&](int stage, int slot) {
            if (TMA && lane == 0) {
                mbar_arrive_expect_tx(full + slot, uint32_t(groups * kTcRaw));
                for (int gi = 0; gi < groups; ++gi)
                    bulk_tensor_2d_g2s(ring + (slot * 2 + gi) * kTcRaw, &map, (g0 + gi) * kCkptGroup, int(lo) + stage * kTcRows, full + slot, policy);
            }
            scales[slot * 2 * kTcRows + lane] = s0;
            scales[slot * 2 * kTcRows + kTcRows + lane] = s1;
            __syncwarp();
            if (lane == 0) mbar_arrive(full + slot);
            load_scales(stage + 1);
        };
        load_scales(0);
        const int ahead = min(kTcRing, stages);
        for (int i = 0; i < ahead; ++i) fetch(i, i);
        int slot = 0, parity = 0, stage = 0;
        for (; stage + kTcRing < stages; ++stage) {
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(empty + slot, parity, abort_flag));
            if (!ok) break;
            fetch(stage + kTcRing, slot);
            if (++slot == kTcRing) { slot = 0; parity ^= 1; }
        }
        if (TMA)                                                     // every copy lands before the CTA ends, also after giving up
            for (int i = stage; i < min(stages, stage + kTcRing); ++i) mbar_wait_drain(full + i % kTcRing, (i / kTcRing) & 1);
    } else {
        const bool z_real = z_on && zc < classes;
        long long zt = lo + set * kTcRows + zk * 8;
        const E* zp = static_cast<const E*>(p.dz) + c0 + zc + zt * p.ld_dz;
        float z[8];
        auto load_dz = [&] {                                         // and on to this set's next stage
#pragma unroll
            for (int r = 0; r < 8; ++r) z[r] = 0.0f;
            if (z_real) {
                const E* q = zp;
                if (zt + 8 <= hi) {
#pragma unroll
                    for (int r = 0; r < 8; ++r, q += p.ld_dz) z[r] = load_as_float(q);
                } else {
#pragma unroll
                    for (int r = 0; r < 8; ++r, q += p.ld_dz)
                        if (zt + r < hi) z[r] = load_as_float(q);
                }
            }
            zp += 2 * kTcRows * p.ld_dz;
            zt += 2 * kTcRows;
        };
        // this warp's part of q: group qg, rows 8 * qk .. 8 * qk + 7, four columns per lane
        const int qg = sw & 1, qk = sw >> 1;
        uint32_t w[8];
        auto load_words = [&](int stage) {                           // q without alignment: the words that hold the four bytes
            const int col = (g0 + qg) * kCkptGroup + 4 * lane;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const long long t = lo + stage * kTcRows + qk * 8 + r;
                w[r] = 0;
                if (qg < groups && t < hi && col < p.n) {
                    const uintptr_t a = reinterpret_cast<uintptr_t>(p.q) + t * p.ld_q + col;
                    const int left = min(4, p.n - col), off = int(a & 3);
                    const uint32_t* base = reinterpret_cast<const uint32_t*>(a & ~uintptr_t(3));
                    const uint32_t w0 = __ldg(base), w1 = off + left > 4 ? __ldg(base + 1) : 0u;
                    w[r] = __funnelshift_r(w0, w1, 8 * off) & (0xffffffffu >> (32 - 8 * left));
                }
            }
        };
        load_dz();
        if (!TMA) load_words(set);
        auto wait = [&](uint64_t* bar, uint32_t parity) {            // one verdict for the warp
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, abort_flag));
            return ok;
        };
        // both sets take the sums out before the (even) stage `next` starts them afresh
        auto take_out = [&](int next) {
            if (next == 0 || next % kTcFlush != 0) return true;
            if (!wait(done + (next - 1) % kTcBuffers, ((next - 1) / kTcBuffers) & 1)) return false;
            flush();
            __syncwarp();
            if (lane == 0) mbar_arrive(flushed);
            return true;
        };
        int slot = set, slot_phase = 0, buf = set, use = 0;          // use: how often this buffer was filled before
        for (int stage = set; stage < stages; stage += 2) {
            if (use > 0 && !wait(done + buf, (use - 1) & 1)) break;  // the products of three stages ago have read this buffer
            if (!wait(full + slot, slot_phase)) break;
            if (TMA && qg < groups) {
                const uint32_t* raw = reinterpret_cast<const uint32_t*>(ring + (slot * 2 + qg) * kTcRaw) + qk * 8 * 32 + lane;
#pragma unroll
                for (int r = 0; r < 8; ++r) w[r] = raw[r * 32];
            }
            if (z_on) {
                const float4* rows = reinterpret_cast<const float4*>(scales + slot * 2 * kTcRows) + 2 * zk;
                zsum += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
#pragma unroll
                for (int gi = 0; gi < 2; ++gi) {
                    if (gi < groups) {
                        const float4 sa = rows[gi * (kTcRows / 4)], sb = rows[gi * (kTcRows / 4) + 1];
                        float x[8] = {z[0] * sa.x, z[1] * sa.y, z[2] * sa.z, z[3] * sa.w, z[4] * sb.x, z[5] * sb.y, z[6] * sb.z, z[7] * sb.w};
                        uint4* dst = reinterpret_cast<uint4*>(opb + (buf * 2 + gi) * op_b + zk * (ncols * 16)) + zc;
#pragma unroll
                        for (int term = 0; term < 3; ++term) {
                            uint4 o;
                            o.x = split_term(x[0], x[1]);
                            o.y = split_term(x[2], x[3]);
                            o.z = split_term(x[4], x[5]);
                            o.w = split_term(x[6], x[7]);
                            dst[term * cp] = o;
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + slot);                // raw rows and scales are in registers or used
            if (stage + 2 < stages) load_dz();
            slot += 2;
            if (slot >= kTcRing) { slot -= kTcRing; slot_phase ^= 1; }
            if (qg < groups) {
                // column 4 * lane + i becomes row i * 32 + lane of the operand, so that neighbouring lanes store neighbouring 16 bytes
                uint4* dst = reinterpret_cast<uint4*>(opa + (buf * 2 + qg) * kTcOperandA + qk * (kCkptGroup * 16)) + lane;
#define LRGD_COLUMN(I) \
    dst[I * 32] = make_uint4(int8_pair_to_bf16<I>(w[0], w[1]), int8_pair_to_bf16<I>(w[2], w[3]), int8_pair_to_bf16<I>(w[4], w[5]), int8_pair_to_bf16<I>(w[6], w[7]))
                LRGD_COLUMN(0);
                LRGD_COLUMN(1);
                LRGD_COLUMN(2);
                LRGD_COLUMN(3);
#undef LRGD_COLUMN
            }
            if (!TMA && stage + 2 < stages) load_words(stage + 2);
            if (!take_out(stage - set)) break;
            fence_proxy_async_smem();                                // what was just stored is read by the tensor cores
            __syncwarp();
            if (lane == 0) mbar_arrive(ready + buf);
            buf += 2;
            if (buf >= kTcBuffers) { buf -= kTcBuffers; ++use; }
        }
        if (ok && set == 1 && (stages & 1)) take_out(stages - 1);    // the last stage is the other set's
    }
    // all warps get here: every wait above is bounded.  Then the products still in flight, before their memory is used again.
    ok = __syncthreads_and(ok);
    const int issued = *issued_at;
    for (int b = 0; b < kTcBuffers; ++b) {
        const int uses = (issued + kTcBuffers - 1 - b) / kTcBuffers; // stages that committed to this barrier
        if (uses > 0 && !mbar_wait_drain(done + b, (uses - 1) & 1)) ok = false;
    }
    ok = __syncthreads_and(ok);
    if (ok) {
        // sums -> shared memory [class][256] -> rows of the part
        float* tile = reinterpret_cast<float*>(opa);
        float* bsum = tile + kTcMaxClasses * 256;                    // [2 sets][kTcBlocks][cp], each set 256 long
        if (warp < kTcWarps) {
            flush();
            if (fg < groups)
#pragma unroll
                for (int i = 0; i < kTcMaxClasses / 16; ++i)
                    if (16 * i < cp)
#pragma unroll
                        for (int k = 0; k < 8; ++k) tile[(16 * i + 8 * fhalf + k) * 256 + fg * 128 + 4 * lane + (warp & 3)] = acc[8 * i + k];
            bsum[tid] = z_on ? zsum : 0.0f;
        }
        __syncthreads();
        const bool direct = p.chunks == 1;
        const int width = min(256, p.n - g0 * kCkptGroup);
        float* out = direct ? p.grad_w : p.part_w + static_cast<long long>(blockIdx.y) * p.C * p.n;
        out += static_cast<long long>(c0) * p.n + g0 * kCkptGroup;
        if (!direct && p.n % 4 == 0) {                               // rows of the scratch start on 16 bytes
            for (int i = tid; i < classes * 64; i += kTcThreads)
                if ((i & 63) * 4 < width)
                    *reinterpret_cast<float4*>(out + static_cast<long long>(i >> 6) * p.n + (i & 63) * 4) = reinterpret_cast<const float4*>(tile)[i];
        } else {
            for (int i = tid; i < classes * 256; i += kTcThreads) {
                float* o = out + static_cast<long long>(i >> 8) * p.n + (i & 255);
                if ((i & 255) < width) *o = direct && p.accumulate ? *o + tile[i] : tile[i];
            }
        }
        if (blockIdx.x == 0 && tid < classes) {
            float sum = 0.0f;
            for (int k = 0; k < kTcBlocks; ++k) sum += bsum[k * cp + tid] + bsum[256 + k * cp + tid];
            if (!direct) p.part_b[static_cast<long long>(blockIdx.y) * p.C + c0 + tid] = sum;
            else if (p.grad_b) p.grad_b[c0 + tid] = p.accumulate ? p.grad_b[c0 + tid] + sum : sum;
        }
    } else if (tid == 0) {
        atomicExch(tp.status, kStatusTimeout);
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

// One class, X^T err of the binary model: bound by reading q, the pipeline above would only add its start and its conversions.
// Sixteen lanes take 256 columns of a row, sixteen neighbouring ones per lane (VEC: one 16-byte load), a warp two rows at a time,
// the CTA's warps take turns.  Scale and dz are one factor per lane and row.  The sums of the lanes and warps that share a column
// meet in shared memory in a fixed order.  The sums are fp32 in short chains (a lane adds every 32nd row of its CTA's, seven at
// 65536 x 256; then 32 lanes and warps, then the CTAs in 32 slices): 2 to 4e-7 of the result there (dz has both signs and the sums
// cancel), like a matrix product in fp32.
// Two CTAs of 16 warps with 64 registers a thread, no rows fetched ahead by hand:
// 16384 x 4096 17 us (3.9 TB/s), 65536 x 256 8.5 us; with two rows ahead 27 and 9.0 us, with four and one CTA per SM 52 and 12.
constexpr int kUnitWarps = 16;
constexpr int kUnitCtas = 2;                                         // per SM
constexpr int kUnitRows = 2 * kUnitWarps;                            // rows of a turn of the CTA

__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

template <class E, bool VEC>
__global__ void __launch_bounds__(kUnitWarps * 32, kUnitCtas) k_ckpt8_grad_unit(const __grid_constant__ CkptGradParams p) {
    __shared__ float sums[kUnitWarps][256];
    __shared__ float bias_sums[kUnitWarps];
    grid_dependency_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane & 15;
    const int c0 = blockIdx.x * 256 + (VEC ? sub * 16 : sub);        // columns c0 .. c0 + 15, or c0, c0 + 16, ...
    const int g0 = blockIdx.x * 2;
    const long long lo = blockIdx.y * p.rows, hi = min(p.T, lo + p.rows);
    uint64_t acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0ull;
    float zsum = 0.0f;
    const long long first = lo + warp * 2 + (lane >> 4);
    const signed char* row = p.q + first * p.ld_q + c0;
    const float* scale = p.s + first * p.groups + g0 + (VEC ? sub >> 3 : 0);
    const E* dz = static_cast<const E*>(p.dz) + first * p.ld_dz;
    const bool in = c0 < p.n, two = g0 + 1 < p.groups;
    for (long long t = first; t < hi; t += kUnitRows) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        float f0 = 0.0f, f1 = 0.0f;
        if constexpr (VEC) {
            if (in) {
                w = __ldcs(reinterpret_cast<const uint4*>(row));
                f0 = __ldg(scale);
            }
        } else {
            uint32_t b[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c0 + 16 * i < p.n) b[i / 4] |= static_cast<uint32_t>(static_cast<unsigned char>(__ldg(row + 16 * i))) << (8 * (i & 3));
            w = make_uint4(b[0], b[1], b[2], b[3]);
            f0 = __ldg(scale);
            if (two) f1 = __ldg(scale + 1);
        }
        const float z = load_as_float(dz);
        row += kUnitRows * p.ld_q;
        scale += kUnitRows * static_cast<long long>(p.groups);
        dz += kUnitRows * p.ld_dz;
        zsum += z;
        const float a = z * f0, b = VEC ? a : z * f1;
        const uint64_t fa = f32x2_pack(a, a), fb = f32x2_pack(b, b), bias = f32x2_pack(-8388736.0f, -8388736.0f);
        const uint32_t q[4] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u, w.z ^ 0x80808080u, w.w ^ 0x80808080u};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // q + 128 as the mantissa of 2^23 + q + 128
            const uint64_t x0 = f32x2_pack(__uint_as_float(__byte_perm(q[i], 0x4b000000u, 0x7540)), __uint_as_float(__byte_perm(q[i], 0x4b000000u, 0x7541)));
            const uint64_t x1 = f32x2_pack(__uint_as_float(__byte_perm(q[i], 0x4b000000u, 0x7542)), __uint_as_float(__byte_perm(q[i], 0x4b000000u, 0x7543)));
            acc[2 * i] = f32x2_fma(f32x2_add(x0, bias), i < 2 ? fa : fb, acc[2 * i]);
            acc[2 * i + 1] = f32x2_fma(f32x2_add(x1, bias), i < 2 ? fa : fb, acc[2 * i + 1]);
        }
    }
    // the two half-warps' rows, then the warps'
    zsum += __shfl_xor_sync(0xffffffffu, zsum, 16);
    if (lane == 0) bias_sums[warp] = zsum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float even, odd;
        f32x2_unpack(acc[i], even, odd);
        even += __shfl_xor_sync(0xffffffffu, even, 16);
        odd += __shfl_xor_sync(0xffffffffu, odd, 16);
        if (lane < 16) {
            sums[warp][VEC ? sub * 16 + 2 * i : sub + 32 * i] = even;
            sums[warp][VEC ? sub * 16 + 2 * i + 1 : sub + 32 * i + 16] = odd;
        }
    }
    __syncthreads();
    const bool direct = p.chunks == 1;
    const int col = blockIdx.x * 256 + threadIdx.x;
    if (threadIdx.x < 256 && col < p.n) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kUnitWarps; ++w) sum += sums[w][threadIdx.x];
        float* o = (direct ? p.grad_w : p.part_w + static_cast<long long>(blockIdx.y) * p.n) + col;
        *o = direct && p.accumulate ? *o + sum : sum;
    }
    if (blockIdx.x == 0 && threadIdx.x == 256) {
        float sum = 0.0f;
        for (int w = 0; w < kUnitWarps; ++w) sum += bias_sums[w];
        if (!direct) p.part_b[blockIdx.y] = sum;
        else if (p.grad_b) *p.grad_b = p.accumulate ? *p.grad_b + sum : sum;
    }
}

// Adds the parts in a fixed order.  Few parts (SLICES == 1): a thread adds those of four neighbouring values (VEC) in turn.  Many
// parts: slice y of a value takes parts y, y + SLICES, ..., and the slices are added in turn.
constexpr int kJoinThreads = 256;

template <int VEC, int SLICES>
__global__ void __launch_bounds__(kJoinThreads) k_ckpt8_join(const __grid_constant__ CkptGradParams p) {
    struct alignas(4 * VEC) Vec { float v[VEC]; };
    constexpr int kCols = kJoinThreads / SLICES;
    __shared__ Vec part_sum[SLICES][kCols];
    grid_dependency_wait();
    const long long count = static_cast<long long>(p.C) * p.n / VEC, all = count + (p.grad_b ? p.C : 0);
    const int x = threadIdx.x % kCols, y = threadIdx.x / kCols;
    for (long long i0 = static_cast<long long>(blockIdx.x) * kCols; i0 < all; i0 += static_cast<long long>(gridDim.x) * kCols) {
        const long long i = i0 + x;
        Vec sum{};
        if (i < count) {
            const Vec* part = reinterpret_cast<const Vec*>(p.part_w) + i;
#pragma unroll 4
            for (int c = y; c < p.chunks; c += SLICES) {
                const Vec v = part[c * count];
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum.v[k] += v.v[k];
            }
        } else if (i < all) {
            for (int c = y; c < p.chunks; c += SLICES) sum.v[0] += p.part_b[static_cast<long long>(c) * p.C + (i - count)];
        }
        if constexpr (SLICES > 1) {
            __syncthreads();                        // the sums of the values before these have been read
            part_sum[y][x] = sum;
            __syncthreads();
            if (y == 0)
#pragma unroll
                for (int k = 1; k < SLICES; ++k)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) sum.v[j] += part_sum[k][x].v[j];
        }
        if (y > 0) continue;
        if (i < count) {
            Vec* out = reinterpret_cast<Vec*>(p.grad_w) + i;
            if (p.accumulate) {
                const Vec h = *out;
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum.v[k] += h.v[k];
            }
            *out = sum;
        } else if (i < all) {
            float* out = p.grad_b + (i - count);
            *out = p.accumulate ? *out + sum.v[0] : sum.v[0];
        }
    }
}

}  // namespace lrgd
