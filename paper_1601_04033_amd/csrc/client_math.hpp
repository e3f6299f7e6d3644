// Element types, vector access and the dropout draw of the client's kernels.
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_math.hpp"

namespace fasgd {

struct bf16 {
    uint16_t bits;
};
struct f16 {
    _Float16 value;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }
__device__ __forceinline__ float to_float(f16 x) { return static_cast<float>(x.value); }

// Rounded to nearest even; NaN stays NaN.
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x)
{
    return bf16{__builtin_bit_cast(uint16_t, static_cast<__bf16>(x))};
}
template <> __device__ __forceinline__ f16 from_float<f16>(float x) { return f16{static_cast<_Float16>(x)}; }

// N consecutive elements at any alignment of their type: gfx950 takes vector
// accesses at any byte address, so rows of odd length cost no more
// instructions than aligned ones.
template <typename T, int N> struct Pack {
    T v[N];
};
template <typename T, int N> __device__ __forceinline__ Pack<T, N> load_pack(const T* p)
{
    Pack<T, N> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
template <typename T, int N> __device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r)
{
    __builtin_memcpy(p, &r, sizeof r);
}

// x of this lane and of the lane LANES (16 or 32) away, in some order: what a
// sum or a maximum over lanes joins, without a pass through LDS.
struct Pair {
    float x, y;
};
template <int LANES> __device__ __forceinline__ Pair across(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto r = LANES == 16 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                               : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// x of the lane that CTRL (a data-parallel primitive's code) names.
template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// Key and counter words of one dropout (include/fasgd_client.h).
struct DropKey {
    uint32_t key0, key1;        // seed low / high words
    uint32_t ctr1;              // 0x40000000 | site << 16
    uint32_t ctr_T, ctr_client;
    uint32_t thr;               // kept iff the 16-bit draw is >= thr
    float scale;                // 65536 / (65536 - thr)
    int64_t chunk_base;         // index_base / 8
};

// Keep bits of the 8 elements of one chunk: bit 7 - e is element 8 chunk + e.
// One Philox call serves 8 elements, 16 bits each; at 32 bits each the
// draws, not the memory, would bound a pass over 16-bit elements.
__device__ __forceinline__ uint32_t keep_bits(const DropKey& k, uint64_t chunk)
{
    uint32_t key0 = k.key0, key1 = k.key1;
#if defined(__HIP_DEVICE_COMPILE__)
    // The rounds' keys are added up here each time, by the scalar unit: taken
    // out of a loop over rows they are 20 registers, which the compiler spills
    // to lanes of vector registers and reads back with as many vector
    // instructions (16,384 x 4,096 bf16, forward 137 against 123 us).
    asm volatile("" : "+s"(key0), "+s"(key1));
#endif
    const uint4 w = philox4x32_10(make_uint4(static_cast<uint32_t>(chunk), k.ctr1 | static_cast<uint32_t>(chunk >> 32),
                                             k.ctr_T, k.ctr_client),
                                  key0, key1);
    // a draw is compared in the upper half of a word (kept: not below), so
    // thr = 65536 (nothing is kept) needs its own answer
    const uint32_t t = k.thr << 16, none = k.thr >> 16;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits = bits + bits + ((u[i] << 16) >= t ? 1u : 0u);
        bits = bits + bits + (u[i] >= t ? 1u : 0u);
    }
    return none ? 0u : bits;
}

// Keep bits of the N <= 8 elements from matrix index i on: bit N - 1 - j is
// element i + j.
template <int N> __device__ __forceinline__ uint32_t keep_run(const DropKey& k, int64_t i)
{
    const uint64_t chunk = static_cast<uint64_t>(k.chunk_base) + static_cast<uint64_t>(i >> 3);
    const int off = static_cast<int>(i & 7);
    uint32_t bits = keep_bits(k, chunk) << 8;
    if (off + N > 8) bits |= keep_bits(k, chunk + 1);
    return bits >> (16 - N - off);
}

// a x + y with the product rounded to fp32 before the sum: a x alone (y = 0)
// is then the fp32 product, not a wider one that a 16-bit store would round
// differently at ties.
__device__ __forceinline__ float scaled_sum(float a, float x, float y)
{
#pragma clang fp contract(off)
    const float t = a * x;
    return t + y;
}

// x where bit `at` of bits is set, else 0 (whatever x is).
__device__ __forceinline__ float kept(float x, uint32_t bits, int at)
{
    const int mask = static_cast<int>(bits << (31 - at)) >> 31;
    return __int_as_float(__float_as_int(x) & mask);
}

}  // namespace fasgd
