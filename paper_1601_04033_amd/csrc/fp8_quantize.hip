// client_fp8_quantize: a matrix in 8-bit floating point with one power-of-two
// scale per block of 128, in row form, transposed, or both from one read.
#include "client_kernels.hpp"

namespace fasgd {
namespace {

constexpr int kTile = kFp8Block;

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

// |x|, 0 for what is not finite
__device__ __forceinline__ float finite_abs(float x)
{
    const uint32_t bits = __float_as_uint(x) & 0x7fffffffu;
    return bits < 0x7f800000u ? __uint_as_float(bits) : 0.0f;
}

// Four values, already scaled into the format's range, rounded to nearest
// even.  What was not finite becomes NaN.
template <int FORMAT> __device__ __forceinline__ uint32_t pack4(const float (&x)[4])
{
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        y[i] = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : x[i];
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

template <int FORMAT> constexpr int kFmaxExponent = FORMAT == FP8_E4M3 ? 9 : 16;

// One 128 x 128 tile per block of 256 threads; thread (tr, tc) holds rows
// 8 tr .. + 7 of columns 8 tc .. + 7, so that it has 8 consecutive bytes for
// either form.
template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void quantize(QuantizeArgs a)
{
    __shared__ float row_max[kTile][16];
    __shared__ float col_max[kTile][16];
    __shared__ float whole_max[4];
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;
    const int tiles_c = static_cast<int>((a.cols + kTile - 1) / kTile);
    const int tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const int64_t r0 = static_cast<int64_t>(tile_r) * kTile + tr * 8;
    const int64_t c0 = static_cast<int64_t>(tile_c) * kTile + tc * 8;
    const T* x = static_cast<const T*>(a.x);
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        Pack<T, 8> p;
        if (r0 + i < a.rows && c0 + 8 <= a.cols) {
            p = load_pack<T, 8>(x + (r0 + i) * a.ldx + c0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                p.v[j] = r0 + i < a.rows && c0 + j < a.cols ? x[(r0 + i) * a.ldx + c0 + j] : from_float<T>(0.0f);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = to_float(p.v[j]);
    }
    float rm[8], cm[8], all = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) rm[i] = cm[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = finite_abs(v[i][j]);
            rm[i] = fmaxf(rm[i], f);
            cm[j] = fmaxf(cm[j], f);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row_max[tr * 8 + i][tc] = rm[i];
        col_max[tc * 8 + i][tr] = cm[i];
        all = fmaxf(all, rm[i]);
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) all = fmaxf(all, __shfl_xor(all, k));
    if ((threadIdx.x & 63) == 0) whole_max[threadIdx.x >> 6] = all;
    __syncthreads();
    int er[8], ec[8];
    if (a.whole) {
        const float m = fmaxf(fmaxf(whole_max[0], whole_max[1]), fmaxf(whole_max[2], whole_max[3]));
        const int e = block_exponent(m, kFmaxExponent<FORMAT>);
#pragma unroll
        for (int i = 0; i < 8; ++i) er[i] = ec[i] = e;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float r = 0.0f, c = 0.0f;
            for (int k = 0; k < 16; ++k) {
                r = fmaxf(r, row_max[tr * 8 + i][k]);
                c = fmaxf(c, col_max[tc * 8 + i][k]);
            }
            er[i] = block_exponent(r, kFmaxExponent<FORMAT>);
            ec[i] = block_exponent(c, kFmaxExponent<FORMAT>);
        }
    }
    if (a.row.data) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= a.rows) continue;
            const float s = exp2_int(-er[i]);
            uint2 q;
            q.x = pack4<FORMAT>({v[i][0] * s, v[i][1] * s, v[i][2] * s, v[i][3] * s});
            q.y = pack4<FORMAT>({v[i][4] * s, v[i][5] * s, v[i][6] * s, v[i][7] * s});
            *reinterpret_cast<uint2*>(a.row.data + (r0 + i) * a.row.ld + c0) = q;
            if (tc == 0) a.row.scales[tile_c * a.row.lds + r0 + i] = static_cast<uint8_t>(er[i] + 127);
        }
    }
    if (a.col.data) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c0 + j >= a.cols) continue;
            const float s = exp2_int(-ec[j]);
            uint2 q;
            q.x = pack4<FORMAT>({v[0][j] * s, v[1][j] * s, v[2][j] * s, v[3][j] * s});
            q.y = pack4<FORMAT>({v[4][j] * s, v[5][j] * s, v[6][j] * s, v[7][j] * s});
            *reinterpret_cast<uint2*>(a.col.data + (c0 + j) * a.col.ld + r0) = q;
            if (tr == 0) a.col.scales[tile_r * a.col.lds + c0 + j] = static_cast<uint8_t>(ec[j] + 127);
        }
    }
}

template <typename T> hipError_t launch_type(const QuantizeArgs& a, int format, hipStream_t s)
{
    const unsigned grid = static_cast<unsigned>(((a.cols + kTile - 1) / kTile) * ((a.rows + kTile - 1) / kTile));
    if (format == FP8_E4M3) quantize<T, FP8_E4M3><<<grid, 256, 0, s>>>(a);
    else quantize<T, FP8_E5M2><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, int dtype, hipStream_t s)
{
    const int format = a.row.data ? a.row.format : a.col.format;
    if (dtype == DTYPE_F32) return launch_type<float>(a, format, s);
    if (dtype == DTYPE_BF16) return launch_type<bf16>(a, format, s);
    return launch_type<f16>(a, format, s);
}

}  // namespace fasgd
