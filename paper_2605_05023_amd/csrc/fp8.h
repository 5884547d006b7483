// fp8.h -- the two 8-bit floating point formats of the block cache: device
// conversions and the power-of-two scales.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace attn {

template <bool E5M2>
struct Fp8 {
    // largest finite value, 1.75 * 2^8 and 1.75 * 2^15; kTop: it is 0.875 * 2^kTop
    static constexpr float kMax = E5M2 ? 57344.0f : 448.0f;
    static constexpr int kTop = E5M2 ? 16 : 9;

    // Bytes 2 HI and 2 HI + 1 of w as floats.
    template <int HI>
    static __device__ __forceinline__ void unpack(uint32_t w, float* a, float* b)
    {
        if constexpr (E5M2) {
            const auto f = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, HI != 0);
            *a = f[0];
            *b = f[1];
        } else {
            const auto f = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI != 0);
            *a = f[0];
            *b = f[1];
        }
    }

    // Four floats to bytes, to nearest even, limited to +-kMax; NaN stays NaN.
    static __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d)
    {
        return round(limit(a), limit(b), limit(c), limit(d));
    }

    // The same of floats within +-kMax.
    static __device__ __forceinline__ uint32_t round(float a, float b, float c, float d)
    {
        if constexpr (E5M2) {
            const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, lo, true);
        } else {
            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
            return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
        }
    }

    static __device__ __forceinline__ float limit(float x)
    {
        return __builtin_fabsf(x) > kMax ? __builtin_copysignf(kMax, x) : x;
    }

    // The smallest 2^e, e >= -120, with amax <= kMax 2^e (amax finite, >= 0):
    // amax = m 2^x with m in [0.5, 1) is at most 0.875 2^(kTop + e) iff
    // e >= x - kTop, or one more where m > 0.875.
    static __device__ __forceinline__ float scale_for(float amax)
    {
        const uint32_t bits = __builtin_bit_cast(uint32_t, amax);
        int e = (int)(bits >> 23) - 126 - kTop + ((bits & 0x7fffffu) > 0x600000u);
        e = e < -120 ? -120 : e;  // (zero and subnormal amax end here too)
        return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
    }
};

}  // namespace attn
