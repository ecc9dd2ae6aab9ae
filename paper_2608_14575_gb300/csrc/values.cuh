// Values of the operators' types, 16 bytes of them or one.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "hwr.h"

namespace hwr {

template <int DT>
struct Vec {
    static constexpr int N = DT == HWR_F32 ? 4 : 8;      // values of 16 bytes
    __device__ static void unpack(const uint4 &u, float (&f)[N]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == HWR_F32) {
                f[i] = __uint_as_float(w[i]);
            } else if (DT == HWR_BF16) {
                f[(2 * i) % N] = __uint_as_float(w[i] << 16);
                f[(2 * i + 1) % N] = __uint_as_float(w[i] & 0xffff0000u);
            } else {
                const float2 v = __half22float2(*(const __half2 *)&w[i]);
                f[(2 * i) % N] = v.x;
                f[(2 * i + 1) % N] = v.y;
            }
        }
    }
    __device__ static uint4 pack(const float (&f)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == HWR_F32) {
                w[i] = __float_as_uint(f[i]);
            } else if (DT == HWR_BF16) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(f[(2 * i) % N], f[(2 * i + 1) % N]);
                w[i] = *(const uint32_t *)&v;
            } else {
                const __half2 v = __floats2half2_rn(f[(2 * i) % N], f[(2 * i + 1) % N]);
                w[i] = *(const uint32_t *)&v;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static uint4 lowest() {                   // -inf throughout
        const uint32_t w = DT == HWR_F32 ? 0xff800000u : DT == HWR_BF16 ? 0xff80ff80u : 0xfc00fc00u;
        return make_uint4(w, w, w, w);
    }
    __device__ static float largest(const uint4 &u) {    // (NaN left out)
        if (DT == HWR_F32)
            return fmaxf(fmaxf(__uint_as_float(u.x), __uint_as_float(u.y)), fmaxf(__uint_as_float(u.z), __uint_as_float(u.w)));
        if (DT == HWR_BF16) {
            const auto two = [](uint32_t w) { return *(const __nv_bfloat162 *)&w; };
            const __nv_bfloat162 m = __hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w)));
            return fmaxf(__low2float(m), __high2float(m));
        }
        const auto two = [](uint32_t w) { return *(const __half2 *)&w; };
        const __half2 m = __hmax2(__hmax2(two(u.x), two(u.y)), __hmax2(two(u.z), two(u.w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ static float load(const void *p, int i) {
        if (DT == HWR_F32) return ((const float *)p)[i];
        if (DT == HWR_BF16) return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
        return __half2float(((const __half *)p)[i]);
    }
    __device__ static void store(void *p, int i, float v) {
        if (DT == HWR_F32) ((float *)p)[i] = v;
        else if (DT == HWR_BF16) ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(v);
        else ((__half *)p)[i] = __float2half_rn(v);
    }
};

// Two fp32 values in one register pair, for the packed additions and multiplications.  A
// product that is added to may lose its rounding (the assembler makes one instruction of
// both, a few results in a million show): not for values whose every bit counts.
struct Two {
    uint64_t v;
    Two() = default;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Two(uint64_t v) : v(v) {}
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Two operator+(Two a, Two b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.v), "l"(b.v));
    return Two(r);
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.v), "l"(b.v));
    return Two(r);
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a.v), "l"(b.v), "l"(c.v));
    return Two(r);
}

}  // namespace hwr
