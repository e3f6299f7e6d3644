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

// Key and counter words of one dropout (include/fasgd_client.h).
struct DropKey {
    uint32_t key0, key1;        // seed low / high words
    uint32_t ctr1;              // 0x40000000 | site << 16
    uint32_t ctr_T, ctr_client;
    uint32_t thr;               // kept iff the 16-bit draw is >= thr
    float scale;                // 65536 / (65536 - thr)
    int64_t chunk_base;         // index_base / 8
};

// Keep bits of the 8 elements of one chunk: bit e is element 8 chunk + e.
// One Philox call serves 8 elements, 16 bits each; at 32 bits each the
// draws, not the memory, would bound a pass over 16-bit elements.
__device__ __forceinline__ uint32_t keep_bits(const DropKey& k, uint64_t chunk)
{
    const uint4 w = philox4x32_10(make_uint4(static_cast<uint32_t>(chunk), k.ctr1 | static_cast<uint32_t>(chunk >> 32),
                                             k.ctr_T, k.ctr_client),
                                  k.key0, k.key1);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= ((u[i] & 0xffffu) >= k.thr ? 1u : 0u) << (2 * i);
        bits |= ((u[i] >> 16) >= k.thr ? 1u : 0u) << (2 * i + 1);
    }
    return bits;
}

}  // namespace fasgd
