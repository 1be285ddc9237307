// The rotation of a channel pair, shared by the kernels that turn queries and keys: one arithmetic, so that a key turned on its way into
// the cache has the bits of one turned by wide_rope.
#pragma once

#include "internal.h"
#include "ptx.cuh"

#ifdef __CUDACC__
// A frequency (radians a position) as turns a position, a 64-bit fraction.  The product with an integer position wraps modulo one
// turn for free in 64-bit integer arithmetic (error: position * 2^-53 of the frequency).
__device__ __forceinline__ unsigned long long wide_rope_turn(double inv_freq) {
    double f = inv_freq * 0.15915494309189533577;   // 1 / (2 pi)
    f -= floor(f);
    return static_cast<unsigned long long>(f * 18446744073709551616.0);
}
// cosine and sine of the angle of a position: only the reduced angle, in half turns, is rounded to fp32
__device__ __forceinline__ float2 wide_rope_angle(long long pos, unsigned long long turn) {
    const unsigned long long phase = static_cast<unsigned long long>(pos) * turn;
    const float half_turns = static_cast<float>(static_cast<int>(phase >> 32)) * 4.656612873077393e-10f;   // 2^-31
    float2 v;
    sincospif(half_turns, &v.y, &v.x);
    return v;
}
// (u, w) -> (u cos - w sin, u sin + w cos), each product sum with one rounding of the second product
__device__ __forceinline__ float wide_rope_low(float u, float w, float2 c) { return __fmaf_rn(u, c.x, -__fmul_rn(w, c.y)); }
__device__ __forceinline__ float wide_rope_high(float u, float w, float2 c) { return __fmaf_rn(u, c.y, __fmul_rn(w, c.x)); }

namespace {

template <typename T> struct Vec8;   // 8 channels as the memory holds them
template <> struct Vec8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p, bool) const { *reinterpret_cast<uint4*>(p) = v; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    // in two halves, neighbouring lanes would leave each other's half of every 32-byte sector to a second access
    // (4099 tokens of 40 heads in fp32: 33.8 us in halves, 29.0 whole)
    __device__ __forceinline__ void load(const float* p, bool wide) {
        if (wide) {
            wptx::ld_global_256(p, a, b);
        } else {
            a = reinterpret_cast<const float4*>(p)[0];
            b = reinterpret_cast<const float4*>(p)[1];
        }
    }
    __device__ __forceinline__ void store(float* p, bool wide) const {
        if (wide) {
            wptx::st_global_256(p, a, b);
        } else {
            reinterpret_cast<float4*>(p)[0] = a;
            reinterpret_cast<float4*>(p)[1] = b;
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        a = make_float4(x[0], x[1], x[2], x[3]);
        b = make_float4(x[4], x[5], x[6], x[7]);
    }
};

}  // namespace
#endif
