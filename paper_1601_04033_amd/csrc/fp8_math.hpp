// Quantization and matrix-instruction helpers shared by the 8-bit kernels.
#pragma once

#include "client_kernels.hpp"

namespace fasgd {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int FORMAT> constexpr int kFmaxExponent = FORMAT == FP8_E4M3 ? 9 : 16;

// The smallest e >= -126 with amax <= 448 2^e (e4m3) or 57344 2^e (e5m2);
// both limits are 0.875 times a power of two.  0 for amax = 0.
__device__ __forceinline__ int block_exponent(float amax, int fmax_exponent)
{
    const uint32_t bits = __float_as_uint(amax);
    if (bits == 0) return 0;
    const int e = static_cast<int>(bits >> 23) - 126 - fmax_exponent + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ v8i join_chunks(const v4i& lo, const v4i& hi)
{
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// |x|, 0 for what is not finite
__device__ __forceinline__ float finite_abs(float x)
{
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    return bits < 0x7f800000u ? __uint_as_float(bits) : 0.0f;
}

// Four values times 2^-e, within the format's range, rounded to nearest even.
// What is not finite becomes NaN.
template <int FORMAT> __device__ __forceinline__ uint32_t pack4(float x0, float x1, float x2, float x3, float s)
{
    const float x[4] = {x0, x1, x2, x3};
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        y[i] = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : x[i] * s;
    int v = 0;
    if constexpr (FORMAT == FP8_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(y[0], y[1], v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(y[2], y[3], v, true);
    }
    return static_cast<uint32_t>(v);
}

// Largest value of each group of 16 lanes, in all of them.
__device__ __forceinline__ float max_of_16(float x)
{
    x = fmaxf(x, dpp<0xB1>(x));    // quad_perm 1 0 3 2
    x = fmaxf(x, dpp<0x4E>(x));    // quad_perm 2 3 0 1
    x = fmaxf(x, dpp<0x141>(x));   // row_half_mirror
    return fmaxf(x, dpp<0x140>(x));    // row_mirror
}

#if defined(__HIP_DEVICE_COMPILE__)     // the host pass does not know buffer resources
// A buffer of the bytes from p on, as many of `bytes` as 32 bits can say;
// what is read past its end is 0.
__device__ __forceinline__ auto buffer(const uint8_t* p, int64_t bytes)
{
    constexpr int kRaw = 0x00020000;    // raw buffer, 32-bit data
    const uint32_t n = bytes < 0xffffffffll ? static_cast<uint32_t>(bytes) : 0xffffffffu;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, static_cast<int>(n), kRaw);
}
#endif

// 8 values (dwords lo and hi) times 2^(scale - 127), as bf16: exact.
template <int FORMAT> __device__ __forceinline__ v8bf widen(int lo, int hi, float scale)
{
    v2bf x[4];
    if constexpr (FORMAT == FP8_E4M3) {
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    } else {
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
    }
    return v8bf{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

}  // namespace fasgd
