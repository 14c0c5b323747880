// Rows kept between forward and backward in 8 bits.
//
//   save:      128 columns of a row share a scale:  a = max |x|,  s = a / 127,  q = rint(x * r), r = 127 * (1 / a)   (every
//              operation rounded to fp32; ties to even)
//   load:      x' = q * s
//
// |x' - x| <= a/254 within a group (plus the rounding of the two products).  A group whose a is below 1e-36 (127 / a would
// overflow) is kept as zeros; one with a NaN or an infinity gets the scale NaN, so that what is read back shows it.
#pragma once
#include "lrgd_route.cuh"

namespace lrgd {

constexpr int kCkptGroup = 128;
constexpr int kCkptThreads = 256;

struct CkptParams {
    const void* x;             // save: the rows
    void* back;                // load: the rows
    long long ld;
    signed char* q;
    long long ld_q;
    float* s;                  // [T][groups]
    long long T;
    int n;
    int groups;
};

// A warp takes 1024 columns of one row, all loaded before the first group is worked on (one group at a time left too few bytes in
// flight).  VEC: 16-byte loads and 8-byte accesses to q; otherwise element by element, neighbouring lanes on neighbouring columns.
// HBM-bound as long as a value costs few instructions: when saving, eight lanes share a group, so that its two divisions and the
// exchange of the maximum are spread over sixteen values a lane; maxima of bfloat16 pairs are taken packed; rounding and widening go
// through the mantissa of a float instead of the conversion unit.
// 16384 x 4096 bfloat16: save 33 us, load 30 us (203 MB each, 6.2 to 6.7 TB/s); with sixteen lanes a group when saving 46 us.
constexpr int kCkptSteps = 4;                               // when loading: pairs of groups, sixteen lanes each
constexpr int kSaveSteps = 2;                               // when saving: fours of groups, eight lanes each
constexpr int kCkptCols = kCkptSteps * 2 * kCkptGroup;      // columns of a row per warp
static_assert(kCkptCols == kSaveSteps * 4 * kCkptGroup, "both kernels cut a row the same way");

// fp32 pair -> packed bfloat16, to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// rint(v * r), at most 127, as the low byte: adding 1.5 * 2^23 leaves the integer (ties to even) in the mantissa's low bits.  The
// product is rounded first, as the definition has it: fused, one value in a million went to the other neighbour.
__device__ __forceinline__ uint32_t rint_byte(float v, float r) { return __float_as_uint(__fadd_rn(__fmul_rn(v, r), 12582912.0f)); }
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// byte I of w (signed) as a float: with the sign bit flipped it is q + 128, which is read as the mantissa of 2^23 + q + 128
template <int I>
__device__ __forceinline__ float byte_to_float(uint32_t flipped) {
    return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7540 | I)) - 8388736.0f;
}

// Eight values of a row: columns c0 .. c0 + 7 (VEC) or c0, c0 + 8, ..., c0 + 56
template <class E, bool VEC>
struct CkptLane {
    static constexpr int kWords = sizeof(E) == 4 ? 8 : 4;      // raw 32-bit words
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const E* row, int c0, int n) {      // zeros past the end
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
        if constexpr (VEC) {
            if (c0 < n) {
#pragma unroll
                for (int i = 0; i < kWords; i += 4) {
                    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(row + c0) + i / 4);
                    w[i] = a.x; w[i + 1] = a.y; w[i + 2] = a.z; w[i + 3] = a.w;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + 8 * i < n) {
                    if constexpr (sizeof(E) == 4) w[i] = __float_as_uint(__ldg(row + c0 + 8 * i));
                    else w[i / 2] |= static_cast<uint32_t>(__ldg(row + c0 + 8 * i)) << (16 * (i & 1));
                }
        }
    }
    __device__ __forceinline__ float value(int i) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    // bits of the largest magnitude: a NaN is above an infinity, which is above every number
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) t = max(t, w[i] & 0x7fffffffu);
            return t;
        } else {                                               // two 16-bit maxima
#pragma unroll
            for (int i = 0; i < 4; ++i) t = __vmaxu2(t, w[i] & 0x7fff7fffu);
            return max(t & 0xffff0000u, t << 16);
        }
    }
    __device__ __forceinline__ void store(signed char* out, int c0, int n, float inv, bool lost) const {
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = rint_byte(value(i), inv);
        if constexpr (VEC) {
            const uint32_t a = pack_bytes(q[0], q[1], q[2], q[3]), b = pack_bytes(q[4], q[5], q[6], q[7]);
            if (c0 < n) *reinterpret_cast<uint2*>(out + c0) = lost ? make_uint2(0u, 0u) : make_uint2(a, b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + 8 * i < n) out[c0 + 8 * i] = lost ? 0 : static_cast<signed char>(q[i]);
        }
    }
};

template <class E, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_save(const __grid_constant__ CkptParams p) {
    const int lane = threadIdx.x & 31, sub = lane & 7;
    const int first = blockIdx.y * (4 * kSaveSteps), mine = lane >> 3;       // groups first + 4 * k + mine
    const long long warps = static_cast<long long>(gridDim.x) * (kCkptThreads / 32);
    for (long long t = static_cast<long long>(blockIdx.x) * (kCkptThreads / 32) + (threadIdx.x >> 5); t < p.T; t += warps) {
        const E* row = static_cast<const E*>(p.x) + t * p.ld;
        signed char* out = p.q + t * p.ld_q;
        float* scales = p.s + t * p.groups;
        CkptLane<E, VEC> x[kSaveSteps][2];                     // the two halves of the group
        const int c0 = (first + mine) * kCkptGroup + (VEC ? sub * 8 : sub);
#pragma unroll
        for (int k = 0; k < kSaveSteps; ++k) {
            x[k][0].load(row, c0 + 4 * k * kCkptGroup, p.n);
            x[k][1].load(row, c0 + 4 * k * kCkptGroup + kCkptGroup / 2, p.n);
        }
#pragma unroll
        for (int k = 0; k < kSaveSteps; ++k) {
            const int g = first + 4 * k + mine, c = c0 + 4 * k * kCkptGroup;
            if (first + 4 * k >= p.groups) break;              // the same for the whole warp
            uint32_t top = max(x[k][0].top(), x[k][1].top());
#pragma unroll
            for (int m = 4; m >= 1; m >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
            const float a = __uint_as_float(top);
            const bool lost = top >= 0x7f800000u, none = a < 1e-36f;
            const float inv = none ? 0.0f : __fmul_rn(__frcp_rn(a), 127.0f);
            x[k][0].store(out, c, p.n, inv, lost);
            x[k][1].store(out, c + kCkptGroup / 2, p.n, inv, lost);
            // (the cap matters for the largest finite values alone: 127 times a scale that was rounded up would be infinite)
            if (sub == 0 && g < p.groups) scales[g] = lost ? __int_as_float(0x7fc00000) : none ? 0.0f : fminf(a / 127.0f, __fdiv_rz(3.402823466e38f, 127.0f));
        }
    }
}

template <class E, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_load(const __grid_constant__ CkptParams p) {
    const int lane = threadIdx.x & 31, sub = lane & 15;
    const int first = blockIdx.y * (2 * kCkptSteps) + (lane >> 4);
    const long long warps = static_cast<long long>(gridDim.x) * (kCkptThreads / 32);
    for (long long t = static_cast<long long>(blockIdx.x) * (kCkptThreads / 32) + (threadIdx.x >> 5); t < p.T; t += warps) {
        const signed char* row = p.q + t * p.ld_q;
        E* out = static_cast<E*>(p.back) + t * p.ld;
        uint2 w[kCkptSteps];
        float s[kCkptSteps];
#pragma unroll
        for (int k = 0; k < kCkptSteps; ++k) {
            const int g = first + 2 * k, c0 = g * kCkptGroup + (VEC ? sub * 8 : sub);
            w[k] = make_uint2(0u, 0u);
            s[k] = g < p.groups ? __ldg(p.s + t * p.groups + g) : 0.0f;
            if constexpr (VEC) {
                if (c0 < p.n) w[k] = __ldcs(reinterpret_cast<const uint2*>(row + c0));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + 16 * i < p.n) (i < 4 ? w[k].x : w[k].y) |= static_cast<uint32_t>(static_cast<unsigned char>(__ldg(row + c0 + 16 * i))) << (8 * (i & 3));
            }
        }
#pragma unroll
        for (int k = 0; k < kCkptSteps; ++k) {
            const int c0 = (first + 2 * k) * kCkptGroup + (VEC ? sub * 8 : sub);
            const uint32_t a = w[k].x ^ 0x80808080u, b = w[k].y ^ 0x80808080u;
            const float v[8] = {byte_to_float<0>(a) * s[k], byte_to_float<1>(a) * s[k], byte_to_float<2>(a) * s[k], byte_to_float<3>(a) * s[k],
                                byte_to_float<0>(b) * s[k], byte_to_float<1>(b) * s[k], byte_to_float<2>(b) * s[k], byte_to_float<3>(b) * s[k]};
            if constexpr (VEC) {
                if (c0 < p.n) {
                    if constexpr (sizeof(E) == 4) {
                        reinterpret_cast<float4*>(out + c0)[0] = make_float4(v[0], v[1], v[2], v[3]);
                        reinterpret_cast<float4*>(out + c0)[1] = make_float4(v[4], v[5], v[6], v[7]);
                    } else {
                        *reinterpret_cast<uint4*>(out + c0) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + 16 * i < p.n) store_from_float(out + c0 + 16 * i, v[i]);
            }
        }
    }
}

}  // namespace lrgd
