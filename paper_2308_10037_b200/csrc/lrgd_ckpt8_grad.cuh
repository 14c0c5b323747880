// Gradient of a C-class logistic layer from rows kept in 8 bits, on the tensor cores:
//
//   grad_w[c,j] (+)= sum_t (dz[t,c] * s[t,g]) * q[t,j]   for the columns j of group g,      grad_b[c] (+)= sum_t dz[t,c]
//
// As a matrix product, D[j,(c)] = sum over t of A[j,t] B[t,c] with A = q^T, B = dz * s: the sum index is the row t, and the scale
// differs from one group of 128 columns to the next, so B is formed per group.  q is an int8 operand as it is: a TMA copy puts
// it where the tensor cores read it and nothing converts it.  For B the fp32 factor x = dz * s becomes a 31-bit integer
// I = rint(x * 2^k), cut into four signed bytes, I = d3 * 2^24 + d2 * 2^16 + d1 * 2^8 + d0, which stand side by side as 4 * CP
// columns of B.  The products are summed in 32-bit integers, exactly, and the four sums of a class are put together in fp64 when
// they are read back; the one rounding to fp32 is the last.  2^k belongs to a class, a group and a range of rows: it brings the
// largest |dz| of the class times the largest s of the group to 2^28 .. 2^30 (k_ckpt8_ranges finds the two), so the rounding of
// I (a half) is 2^-29 of that at most: nothing beside the fp32 rounding of the terms that carry the sum.
// Measured against three bfloat16 terms with fp32 sums (24 bits, but q converted and every operand twice as wide): 16384 x 4096,
// 64 classes, 52 us there, 40 us here, k_ckpt8_ranges (5) and k_ckpt8_join (6) included; the floor is 11 (74 MB).
//
// A CTA takes two groups (256 columns), one block of up to 64 classes and a range of rows, 32 rows per stage.  One warp copies q
// (TMA) and the scales into the slots of q, eleven to sixteen stages ahead; a set of one to four warps (16 classes each) writes the
// bytes of dz * s into a slot of B, K-major (16 consecutive t of one byte and class are 16 bytes), the sets taking the stages in
// turn; one thread per group issues the tcgen05.mma of the stage, whose completion frees both slots.  The parties meet on mbarriers
// alone.  Where q is not 16-byte aligned the set places its bytes.  The rows are split over CTAs to fill the GPU; k_ckpt8_join adds
// the parts in order.
// What bounds it (clock readings of one CTA): with 64 classes the converting warps, 1900 clocks for the 16 rows x 32 classes x 2
// groups of a warp and stage, four stages at a time; with few classes the issuing threads, about 500 clocks a stage: alone in
// its warp, every instruction of such a thread costs its latency (one thread for both groups took 670 to 900).
#pragma once
#include <cuda.h>

#include "lrgd_ckpt8.cuh"

namespace lrgd {

constexpr int kTcWarps = 16;                       // converting warps
constexpr int kTcThreads = (kTcWarps + 3) * 32;    // then a copying warp and two that issue the products, one group each
constexpr int kTcRows = 32;                        // rows per stage: K of one tcgen05.mma on bytes
constexpr int kTcMaxClasses = 64;
constexpr int kTcMaxSlots = 16;
constexpr int kTcHeader = 5120;                    // barriers, flags and exponents (1 KB), then the scales of the slots
constexpr int kTcTileA = kTcRows * kCkptGroup;     // bytes of q per group and slot
constexpr int64_t kTcMaxRows = 1 << 16;            // rows per CTA: 2^16 products of two bytes stay below 2^31
constexpr int kTcMaxSub = 32;
constexpr int kTcMaxSmem = 232448;                 // dynamic shared memory a CTA may ask for
// Slots: those of dz * s first, then what is left for q (eleven for 64 classes, sixteen for 32 and fewer; always more than those
// of dz * s, so that a slot of q comes round later than the slot of dz * s it was multiplied with).
constexpr int tc_slots_b(int cp) { return cp <= 16 ? 14 : 8; }
constexpr int tc_fixed_bytes(int cp) { return kTcHeader + tc_slots_b(cp) * 2 * 4 * cp * kTcRows + 1024; }
constexpr int tc_slots_a(int cp) {
    const int fit = (kTcMaxSmem - tc_fixed_bytes(cp)) / (2 * kTcTileA);
    return fit < kTcMaxSlots ? fit : kTcMaxSlots;
}
// (always more than half an SM's: one CTA per SM, which takes all of its tensor memory)
constexpr int tc_smem_bytes(int cp) { return tc_fixed_bytes(cp) + tc_slots_a(cp) * 2 * kTcTileA; }
static_assert(tc_slots_a(64) > tc_slots_b(64) && tc_slots_a(48) > tc_slots_b(48) && tc_slots_a(16) > tc_slots_b(16), "see above");
static_assert(tc_smem_bytes(16) > 120 * 1024, "one CTA per SM");

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
    int slots_a, slots_b;      // stages in flight, of q and of dz * s
    int sub;                   // parts of a chunk that k_ckpt8_ranges looks at one by one
    unsigned int* ranges;      // [chunks][sub][C + groups]: bits of the largest |dz| of a class and the largest |s| of a group
    int* status;
};

// Largest magnitudes, as bits (a NaN above an infinity above every number).  Block: 32 columns x 8 rows of dz or of s.
constexpr int kRangeThreads = 256;

template <class E>
__global__ void __launch_bounds__(kRangeThreads) k_ckpt8_ranges(const __grid_constant__ TcGradParams tp) {
    __shared__ unsigned int top[8][32];
    const CkptGradParams& p = tp.g;
    grid_dependency_release();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int dz_blocks = (p.C + 31) / 32;
    const bool is_dz = static_cast<int>(blockIdx.x) < dz_blocks;
    const int col = (is_dz ? blockIdx.x : blockIdx.x - dz_blocks) * 32 + x, cols = is_dz ? p.C : p.groups;
    const int chunk = blockIdx.y / tp.sub, part = blockIdx.y - chunk * tp.sub;
    const long long per = (p.rows + tp.sub - 1) / tp.sub;
    const long long lo = chunk * p.rows + part * per, hi = min(min(p.T, (chunk + 1) * p.rows), lo + per);
    unsigned int m = 0;
    if (col < cols) {
        if (is_dz) {
            const E* dz = static_cast<const E*>(p.dz) + col;
#pragma unroll 8
            for (long long t = lo + y; t < hi; t += 8) m = max(m, __float_as_uint(load_as_float(dz + t * p.ld_dz)) & 0x7fffffffu);
        } else {
            const float* s = p.s + col;
#pragma unroll 8
            for (long long t = lo + y; t < hi; t += 8) m = max(m, __float_as_uint(__ldg(s + t * p.groups)) & 0x7fffffffu);
        }
    }
    top[y][x] = m;
    __syncthreads();
    if (y == 0 && col < cols) {
#pragma unroll
        for (int k = 1; k < 8; ++k) m = max(m, top[k][x]);
        tp.ranges[static_cast<long long>(blockIdx.y) * (p.C + p.groups) + (is_dz ? 0 : p.C) + col] = m;
    }
}

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
__device__ __forceinline__ void mma_int8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
        : "memory");
}
__device__ __forceinline__ void tmem_load8(uint32_t addr, int (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Four bytes global -> shared, zeros where !real, and the arrival on `bar` of this thread when its copies so far have landed.
__device__ __forceinline__ void async_copy4(float* dst, const float* src, bool real) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ void async_copy_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Shared-memory operands.  A: rows of K are 128 contiguous bytes (the M index), 16-byte pieces exchanged within blocks of eight
// rows as the 128-byte swizzle does, 1024 bytes from one block of eight to the next.  B: K-major without swizzle, eight rows of 16 bytes
// are 128 contiguous bytes; `k_stride` bytes to the next 16 values of K, 128 bytes to the next eight rows.
__device__ __forceinline__ uint64_t desc_a(uint32_t addr) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(1024 >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
__device__ __forceinline__ uint64_t desc_b(uint32_t addr, uint32_t k_stride) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(k_stride >> 4) << 16 | uint64_t(128 >> 4) << 32 | uint64_t(1) << 46;
}

// Four integers to their four signed bytes: word d of `out` holds byte d of all four.
__device__ __forceinline__ void bytes_of_four(const int (&v)[4], uint32_t (&out)[4]) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (static_cast<uint32_t>(v[i]) + 0x80808080u) ^ 0x80808080u;      // digits in [-128, 127]
    const uint32_t lo01 = __byte_perm(x[0], x[1], 0x5140), hi01 = __byte_perm(x[0], x[1], 0x7362);
    const uint32_t lo23 = __byte_perm(x[2], x[3], 0x5140), hi23 = __byte_perm(x[2], x[3], 0x7362);
    out[0] = __byte_perm(lo01, lo23, 0x5410);
    out[1] = __byte_perm(lo01, lo23, 0x7632);
    out[2] = __byte_perm(hi01, hi23, 0x5410);
    out[3] = __byte_perm(hi01, hi23, 0x7632);
}

// Exponent k of the factor 2^k from the largest |dz| and |s| (bits); kNotFinite where a product of the two need not be finite.
constexpr int kNotFinite = 1 << 20;
__device__ __forceinline__ int factor_exponent(unsigned int dz, unsigned int s) {
    const int e = static_cast<int>(dz >> 23) + static_cast<int>(s >> 23) - 254;                       // product < 2^(e + 2)
    if (dz >= 0x7f800000u || s >= 0x7f800000u || e > 125) return kNotFinite;
    return min(28 - e, 126);
}

template <class E, bool TMA>
__global__ void __launch_bounds__(kTcThreads, 1) k_ckpt8_grad_tc(const __grid_constant__ CUtensorMap map, const __grid_constant__ TcGradParams tp) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const CkptGradParams& p = tp.g;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);              // [slots_a] q and the scales of a stage have landed
    uint64_t* done = full + kTcMaxSlots;                             // [slots_a] the products of the stage are complete
    uint64_t* ready = done + kTcMaxSlots;                            // [slots_b] both operands are in place
    uint64_t* last = ready + kTcMaxSlots;                            // [2 groups] all products are complete
    uint32_t* tmem_at = reinterpret_cast<uint32_t*>(last + 2);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_at + 1);
    int* exponent = reinterpret_cast<int*>(smem + 512);              // [2 groups][kTcMaxClasses]
    float* scales = reinterpret_cast<float*>(smem + 1024);           // [slots_a][2 groups][kTcRows]
    const int cp = tp.cp, ncols = 4 * cp;
    const int tile_b = ncols * kTcRows;                              // bytes per group and slot
    const int slots_a = tp.slots_a, slots_b = tp.slots_b;
    // sets of converting warps; at most one per slot of B, so that none is more than a turn of a ring ahead of another
    const int set_warps = cp / 16, sets = min(kTcWarps / set_warps, slots_b);
    unsigned char* opa = smem + kTcHeader;                           // [slots_a][2 groups]
    unsigned char* opb = opa + slots_a * 2 * kTcTileA;               // [slots_b][2 groups]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g0 = blockIdx.x * 2, groups = min(2, p.groups - g0);
    const int c0 = blockIdx.z * cp, classes = min(cp, p.C - c0);
    const long long lo = blockIdx.y * p.rows, hi = min(p.T, lo + p.rows);
    const int stages = static_cast<int>((hi - lo + kTcRows - 1) / kTcRows);

    grid_dependency_release();                                       // k_ckpt8_join may be launched; it waits for this kernel's end
    if (tid == 0) {
        for (int i = 0; i < slots_a; ++i) {
            mbar_init(full + i, 32 + (TMA ? 1 : 0));                 // the lanes that copy scales, and the copy of q
            mbar_init(done + i, groups);
        }
        for (int i = 0; i < slots_b; ++i) mbar_init(ready + i, set_warps);
        *abort_flag = 0;
        for (int i = 0; i < 2; ++i) mbar_init(last + i, 1);
        fence_mbar_init();
    }
    if (warp == 0) tmem_alloc(tmem_at, 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = *tmem_at;
    bool ok = true;
    float zsum = 0.0f;

    if (warp > kTcWarps) {
        const int gi = warp - kTcWarps - 1;
        if (lane == 0 && gi < groups) {
            // D int32, A and B int8, A with M contiguous
            const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (uint32_t(ncols / 8) << 17) | (uint32_t(kCkptGroup / 16) << 24);
            const uint64_t a0 = desc_a(smem_u32(opa + gi * kTcTileA)), b0 = desc_b(smem_u32(opb + gi * tile_b), ncols * 16);
            const uint32_t d = tmem + gi * ncols, step_b = 2 * tile_b >> 4;         // (descriptors count in 16 bytes)
            uint64_t a = a0, b = b0;
            int slot = 0, slot_b = 0, parity = 0;
#pragma unroll 1
            for (int stage = 0; stage < stages; ++stage) {
                if (!mbar_wait_bounded(ready + slot_b, parity, abort_flag)) { ok = false; break; }
                tmem_fence_after();
                mma_int8(d, a, b, idesc, stage > 0);
                mma_commit(done + slot);
                a += 2 * kTcTileA >> 4;
                b += step_b;
                if (++slot == slots_a) { slot = 0; a = a0; }
                if (++slot_b == slots_b) { slot_b = 0; b = b0; parity ^= 1; }
            }
            mma_commit(last + gi);                                   // all products of this thread, also after giving up
            if (!mbar_wait_drain(last + gi, 0)) ok = false;
        }
    } else if (warp == kTcWarps) {
        const uint64_t policy = l2_policy_evict_first();
        // lane: one row of a stage, both groups' scales (rows past the end: zeros)
        long long t = lo + lane;
        const float* sp = p.s + min(t, hi - 1) * p.groups + g0;
        int stage = 0, slot = 0, turn = 0;
        for (; stage < stages; ++stage) {
            if (turn > 0) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(done + slot, (turn - 1) & 1, abort_flag));
                if (!ok) break;
            }
            if (TMA && lane == 0) {
                mbar_arrive_expect_tx(full + slot, uint32_t(groups * kTcTileA));
                for (int gi = 0; gi < groups; ++gi)
                    bulk_tensor_2d_g2s(opa + (slot * 2 + gi) * kTcTileA, &map, (g0 + gi) * kCkptGroup, int(lo) + stage * kTcRows, full + slot, policy);
            }
            float* dst = scales + slot * 2 * kTcRows + lane;
            const bool in = t < hi;
            async_copy4(dst, in ? sp : p.s, in);
            if (groups > 1) async_copy4(dst + kTcRows, in ? sp + 1 : p.s, in);
            async_copy_arrive(full + slot);
            t += kTcRows;
            sp += static_cast<long long>(kTcRows) * p.groups;
            if (++slot == slots_a) { slot = 0; ++turn; }
        }
        // every copy lands before the CTA ends, also after giving up
        for (int i = max(0, stage - slots_a); i < stage; ++i) mbar_wait_drain(full + i % slots_a, (i / slots_a) & 1);
    } else {
        const int set = warp / set_warps, stid = tid - set * set_warps * 32;
        const int zk = stid / cp, zc = stid - zk * cp;               // this thread's part of dz: class c0 + zc, rows 16 * zk .. + 15
        const bool z_on = zk < kTcRows / 16, z_real = z_on && zc < classes;
        long long zt = lo + set * kTcRows + zk * 16;
        const E* zp = static_cast<const E*>(p.dz) + c0 + zc + zt * p.ld_dz;
        const uint32_t row_bytes = static_cast<uint32_t>(p.ld_dz) * sizeof(E);
        float z[16];
        auto load_dz = [&] {                                         // and on to this set's next stage
            // (a 32-bit factor: one multiply-add per address; ld_dz is at most 2^28)
            const char* q = reinterpret_cast<const char*>(zp);
            if (z_real && zt + 16 <= hi) {
#pragma unroll
                for (unsigned int r = 0; r < 16; ++r) z[r] = load_as_float(reinterpret_cast<const E*>(q + static_cast<uint64_t>(row_bytes) * r));
            } else {
#pragma unroll
                for (unsigned int r = 0; r < 16; ++r)
                    z[r] = z_real && zt + r < hi ? load_as_float(reinterpret_cast<const E*>(q + static_cast<uint64_t>(row_bytes) * r)) : 0.0f;
            }
            zp += sets * kTcRows * p.ld_dz;
            zt += sets * kTcRows;
        };
        load_dz();
        // exponents of the classes and groups of this CTA's rows
        grid_dependency_wait();                                      // k_ckpt8_ranges
        if (tid < 2 * kTcMaxClasses) {
            const int c = tid & (kTcMaxClasses - 1), gi = tid / kTcMaxClasses;
            int e = 0;
            if (c < classes && gi < groups) {
                const unsigned int* r = tp.ranges + static_cast<long long>(blockIdx.y) * tp.sub * (p.C + p.groups);
                unsigned int dz_top = 0, s_top = 0;
#pragma unroll 8
                for (int k = 0; k < tp.sub; ++k, r += p.C + p.groups) {
                    dz_top = max(dz_top, r[c0 + c]);
                    s_top = max(s_top, r[p.C + g0 + gi]);
                }
                e = factor_exponent(dz_top, s_top);
            }
            exponent[gi * kTcMaxClasses + c] = e;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kTcWarps * 32) : "memory");               // the converting warps
        float factor[2];
#pragma unroll
        for (int gi = 0; gi < 2; ++gi) {
            const int e = exponent[gi * kTcMaxClasses + (z_on ? zc : 0)];
            factor[gi] = e == kNotFinite ? 0.0f : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
        }
        // the stage's slot of q, and that of the stage which had its slot of B before
        int slot = set, turn = 0, slot_b = set;
        int before = set - slots_b, before_turn = 0;
        for (int stage = set < sets ? set : stages; stage < stages; stage += sets) {
            const bool in_time = before < 0 || mbar_wait_bounded(done + before, before_turn & 1, abort_flag);
            ok = __all_sync(0xffffffffu, in_time && mbar_wait_bounded(full + slot, turn & 1, abort_flag));
            if (!ok) break;
            if (z_on) {
                zsum += (((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]))) + (((z[8] + z[9]) + (z[10] + z[11])) + ((z[12] + z[13]) + (z[14] + z[15])));
#pragma unroll
                for (int gi = 0; gi < 2; ++gi) {
                    if (gi < groups) {
                        const float4* sp = reinterpret_cast<const float4*>(scales + (slot * 2 + gi) * kTcRows + zk * 16);
                        uint32_t word[4][4];                         // [four rows][byte]
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float4 s = sp[r];
                            const int v[4] = {__float2int_rn(z[4 * r] * s.x * factor[gi]), __float2int_rn(z[4 * r + 1] * s.y * factor[gi]),
                                              __float2int_rn(z[4 * r + 2] * s.z * factor[gi]), __float2int_rn(z[4 * r + 3] * s.w * factor[gi])};
                            bytes_of_four(v, word[r]);
                        }
                        uint4* dst = reinterpret_cast<uint4*>(opb + (slot_b * 2 + gi) * tile_b + zk * (ncols * 16)) + zc;
#pragma unroll
                        for (int d = 0; d < 4; ++d) dst[d * cp] = make_uint4(word[0][d], word[1][d], word[2][d], word[3][d]);
                    }
                }
            }
            if (!TMA) {
                // sixteen bytes at a time from the words that hold them, to where the copy would have put them
#pragma unroll 1
                for (int u = stid; u < kTcRows * 2 * 8; u += set_warps * 32) {
                    const int row = u >> 4, gi = (u >> 3) & 1, piece = u & 7;
                    const long long t = lo + static_cast<long long>(stage) * kTcRows + row;
                    const int col = (g0 + gi) * kCkptGroup + piece * 16, left = min(16, p.n - col);
                    uint32_t w[5] = {0u, 0u, 0u, 0u, 0u};
                    int off = 0;
                    if (gi < groups && t < hi && left > 0) {
                        const uintptr_t a = reinterpret_cast<uintptr_t>(p.q) + t * p.ld_q + col;
                        off = static_cast<int>(a & 3);
                        const uint32_t* base = reinterpret_cast<const uint32_t*>(a & ~uintptr_t(3));
#pragma unroll
                        for (int k = 0; k < 5; ++k)
                            if (4 * k < off + left) w[k] = __ldg(base + k);
                    }
                    uint32_t b[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int real = left - 4 * k;               // bytes of this word that belong to the row
                        b[k] = real <= 0 ? 0u : __funnelshift_r(w[k], w[k + 1], 8 * off) & (real >= 4 ? 0xffffffffu : (1u << (8 * real)) - 1u);
                    }
                    if (gi < groups)
                        *reinterpret_cast<uint4*>(opa + (slot * 2 + gi) * kTcTileA + row * 128 + ((piece ^ (row & 7)) << 4)) = make_uint4(b[0], b[1], b[2], b[3]);
                }
            }
            fence_proxy_async_smem();                                // what was just stored is read by the tensor cores
            __syncwarp();
            if (lane == 0) mbar_arrive(ready + slot_b);
            if (stage + sets < stages) load_dz();
            // (sets <= slots_b < slots_a)
            slot += sets;
            if (slot >= slots_a) { slot -= slots_a; ++turn; }
            before += sets;
            if (before >= slots_a) { before -= slots_a; ++before_turn; }
            slot_b += sets;
            if (slot_b >= slots_b) slot_b -= slots_b;
        }
    }
    // all warps get here: every wait above is bounded, and the products are complete
    ok = __syncthreads_and(ok);
    tmem_fence_after();
    if (ok) {
        const bool direct = p.chunks == 1;
        float* bsum = reinterpret_cast<float*>(opb);                 // [kTcWarps][32]
        if (warp < kTcWarps) {
            bsum[tid] = zsum;
            // this warp: 32 columns of one group, classes 16 * i + 8 * half ..
            const int gi = (warp >> 2) & 1, half = warp >> 3, col = (g0 + gi) * kCkptGroup + (warp & 3) * 32 + lane;
            float* out = (direct ? p.grad_w : p.part_w + static_cast<long long>(blockIdx.y) * p.C * p.n) + static_cast<long long>(c0) * p.n + col;
            if (gi < groups)
                for (int i = 0; 16 * i < cp; ++i) {
                    int d[4][8];
                    const uint32_t at = tmem + (uint32_t((warp & 3) * 32) << 16) + gi * ncols + 16 * i + 8 * half;
#pragma unroll
                    for (int k = 0; k < 4; ++k) tmem_load8(at + k * cp, d[k]);
                    tmem_load_wait();
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int c = 16 * i + 8 * half + k;
                        if (c < classes && col < p.n) {
                            const long long top = static_cast<long long>(d[3][k]) * 256 + d[2][k], low = static_cast<long long>(d[1][k]) * 256 + d[0][k];
                            const int e = exponent[gi * kTcMaxClasses + c];
                            // (top * 2^16 + low) / 2^e, rounded once to fp32
                            const double v = (static_cast<double>(top) * 65536.0 + static_cast<double>(low)) * __hiloint2double((1023 - e) << 20, 0);
                            float sum = e == kNotFinite ? __int_as_float(0x7fc00000) : static_cast<float>(v);
                            float* o = out + static_cast<long long>(c) * p.n;
                            *o = direct && p.accumulate ? *o + sum : sum;
                        }
                    }
                }
        }
        tmem_fence_before();
        __syncthreads();
        if (blockIdx.x == 0 && tid < classes) {
            float sum = 0.0f;
            for (int k = 0; k < sets; ++k)
                for (int b = 0; b < kTcRows / 16; ++b) sum += bsum[k * set_warps * 32 + b * cp + tid];
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
// meet in shared memory in a fixed order.  Two CTAs of 16 warps with 64 registers a thread, no rows fetched ahead by hand:
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
