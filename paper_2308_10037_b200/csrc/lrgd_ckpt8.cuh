// Rows kept between forward and backward in 8 bits.
//
//   save:      128 columns of a row share a scale:  a = max |x|,  s = a / 127,  q = rint(x * (127 / a))   (ties to even)
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

__device__ __forceinline__ uint32_t half_warp_max_u32(uint32_t v) {
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, m));
    return v;
}

// Sixteen lanes hold a group, eight values each.  VEC: eight neighbouring columns by 16-byte loads and one 8-byte store;
// otherwise columns sixteen apart, element by element.
template <class E, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_save(const __grid_constant__ CkptParams p) {
    const int lane = threadIdx.x & 31, sub = lane & 15;
    const long long units = p.T * p.groups;
    const long long step = static_cast<long long>(gridDim.x) * (kCkptThreads / 16);
    for (long long u0 = static_cast<long long>(blockIdx.x) * (kCkptThreads / 16) + (threadIdx.x >> 5) * 2; u0 < units; u0 += step) {
        const long long u = u0 + (lane >> 4);
        const bool on = u < units;
        const long long t = on ? u / p.groups : 0;
        const int g = on ? static_cast<int>(u - t * p.groups) : 0;
        const int c0 = g * kCkptGroup + (VEC ? sub * 8 : sub);
        const E* src = static_cast<const E*>(p.x) + t * p.ld + c0;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if constexpr (VEC) {
            if (on && c0 < p.n) {
                if constexpr (sizeof(E) == 4) {
                    const float4 a = __ldcs(reinterpret_cast<const float4*>(src)), b = __ldcs(reinterpret_cast<const float4*>(src) + 1);
                    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
                } else {
                    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(src));
                    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[2 * i] = __uint_as_float(w[i] << 16);
                        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (on && c0 + 16 * i < p.n) v[i] = load_as_float(src + 16 * i);
        }
        // the largest magnitude as bits: a NaN is above an infinity, which is above every number
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        top = half_warp_max_u32(top);
        const float a = __uint_as_float(top);
        const bool lost = top >= 0x7f800000u, none = a < 1e-36f;
        const float inv = lost || none ? 0.0f : 127.0f / a;
        int q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = lost ? 0 : __float2int_rn(v[i] * inv);
        signed char* dst = p.q + t * p.ld_q + c0;
        if constexpr (VEC) {
            if (on && c0 < p.n) {
                uint2 o;
                o.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | static_cast<uint32_t>(q[3]) << 24;
                o.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | static_cast<uint32_t>(q[7]) << 24;
                *reinterpret_cast<uint2*>(dst) = o;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (on && c0 + 16 * i < p.n) dst[16 * i] = static_cast<signed char>(q[i]);
        }
        // (the cap matters for the largest finite values alone: 127 times a scale that was rounded up would be infinite)
        if (on && sub == 0) p.s[u] = lost ? __int_as_float(0x7fc00000) : none ? 0.0f : fminf(a / 127.0f, __fdiv_rz(3.402823466e38f, 127.0f));
    }
}

template <class E, bool VEC>
__global__ void __launch_bounds__(kCkptThreads) k_ckpt8_load(const __grid_constant__ CkptParams p) {
    const int lane = threadIdx.x & 31, sub = lane & 15;
    const long long units = p.T * p.groups;
    const long long step = static_cast<long long>(gridDim.x) * (kCkptThreads / 16);
    for (long long u = static_cast<long long>(blockIdx.x) * (kCkptThreads / 16) + (threadIdx.x >> 4); u < units; u += step) {
        const long long t = u / p.groups;
        const int g = static_cast<int>(u - t * p.groups);
        const int c0 = g * kCkptGroup + (VEC ? sub * 8 : sub);
        const signed char* src = p.q + t * p.ld_q + c0;
        E* dst = static_cast<E*>(p.back) + t * p.ld + c0;
        const float s = __ldg(p.s + u);
        if constexpr (VEC) {
            if (c0 < p.n) {
                const uint2 w = __ldcs(reinterpret_cast<const uint2*>(src));
                E o[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    store_from_float(&o[i], static_cast<float>(static_cast<signed char>(w.x >> (8 * i))) * s);
                    store_from_float(&o[4 + i], static_cast<float>(static_cast<signed char>(w.y >> (8 * i))) * s);
                }
                if constexpr (sizeof(E) == 4) {
                    reinterpret_cast<float4*>(dst)[0] = make_float4(o[0], o[1], o[2], o[3]);
                    reinterpret_cast<float4*>(dst)[1] = make_float4(o[4], o[5], o[6], o[7]);
                } else {
                    *reinterpret_cast<uint4*>(dst) = make_uint4(o[0] | uint32_t(o[1]) << 16, o[2] | uint32_t(o[3]) << 16,
                                                                o[4] | uint32_t(o[5]) << 16, o[6] | uint32_t(o[7]) << 16);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + 16 * i < p.n) store_from_float(dst + 16 * i, static_cast<float>(src[16 * i]) * s);
        }
    }
}

}  // namespace lrgd
