// client_fp8_quantize: a matrix in 8-bit floating point with one power-of-two
// scale per block of 128, in row form, transposed, or both from one read.
//
// Bound by memory: x is read once, and each form written in whole lines.
#include "fp8_math.hpp"

namespace fasgd {
namespace {

constexpr int kTile = kFp8Block;

// 8 elements of a row from column c on, 0 past its end.
template <typename T> __device__ __forceinline__ Pack<T, 8> load8(const T* row, int64_t c, int64_t cols)
{
    if (c + 8 <= cols) return load_pack<T, 8>(row + c);
    Pack<T, 8> p;
#pragma unroll
    for (int j = 0; j < 8; ++j) p.v[j] = c + j < cols ? row[c + j] : from_float<T>(0.0f);
    return p;
}

// Row form alone: 16 lanes hold a block of a row, so its largest magnitude is
// theirs, and any number of rows fills its waves.
template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void quantize_rows(QuantizeArgs a)
{
    const int lane = threadIdx.x & 15;
    const int64_t blocks = (a.cols + kTile - 1) / kTile;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
    if (i >= a.rows * blocks) return;
    const int64_t r = i / blocks, kb = i % blocks, c = kb * kTile + lane * 8;
    const Pack<T, 8> p = load8(static_cast<const T*>(a.x) + r * a.ldx, c, a.cols);
    float v[8], m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = to_float(p.v[j]);
        m = fmaxf(m, finite_abs(v[j]));
    }
    const int e = block_exponent(max_of_16(m), kFmaxExponent<FORMAT>);
    const float s = exp2_int(-e);
    uint2 q;
    q.x = pack4<FORMAT>(v[0], v[1], v[2], v[3], s);
    q.y = pack4<FORMAT>(v[4], v[5], v[6], v[7], s);
    *reinterpret_cast<uint2*>(a.row.data + r * a.row.ld + c) = q;
    if (lane == 0) a.row.scales[kb * a.row.lds + r] = static_cast<uint8_t>(e + 127);
}

// One 128 x 128 tile per block of 512 threads; thread (tr, tc) holds rows
// 4 tr .. + 3 of columns 8 tc .. + 7 (few enough registers for 4 waves per
// SIMD; with 8 rows a thread the writes waited for the reads).  The
// transposed form passes through LDS, so that it too is written in 16-byte
// pieces of whole lines.
template <typename T, int FORMAT>
__global__ __launch_bounds__(512, 4) void quantize_tile(QuantizeArgs a)
{
    constexpr int R = 4, kWaves = 8;
    __shared__ float col_max[kWaves][kTile];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kTile * kTile];
    __shared__ float whole_max[kWaves];
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int tiles_c = static_cast<int>((a.cols + kTile - 1) / kTile);
    const int tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const int64_t r0 = static_cast<int64_t>(tile_r) * kTile + tr * R;
    const int64_t c0 = static_cast<int64_t>(tile_c) * kTile + tc * 8;
    const T* x = static_cast<const T*>(a.x);
    Pack<T, 8> p[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (r0 + i < a.rows) {
            p[i] = load8(x + (r0 + i) * a.ldx, c0, a.cols);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) p[i].v[j] = from_float<T>(0.0f);
        }
    }
    float rm[R], cm[8];
#pragma unroll
    for (int i = 0; i < R; ++i) rm[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) cm[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = finite_abs(to_float(p[i].v[j]));
            rm[i] = fmaxf(rm[i], f);
            cm[j] = fmaxf(cm[j], f);
        }
    int er[R], ec[8];
    if (a.whole) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) m = fmaxf(m, rm[i]);
        m = max_of_16(m);
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        if ((threadIdx.x & 63) == 0) whole_max[wave] = m;
        __syncthreads();
        m = whole_max[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, whole_max[w]);
        const int e = block_exponent(m, kFmaxExponent<FORMAT>);
#pragma unroll
        for (int i = 0; i < R; ++i) er[i] = e;
#pragma unroll
        for (int j = 0; j < 8; ++j) ec[j] = e;
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) er[i] = block_exponent(max_of_16(rm[i]), kFmaxExponent<FORMAT>);
        if (a.col.data) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                cm[j] = fmaxf(cm[j], __shfl_xor(cm[j], 16));
                cm[j] = fmaxf(cm[j], __shfl_xor(cm[j], 32));
            }
            if ((threadIdx.x & 63) < 16) {
#pragma unroll
                for (int j = 0; j < 8; ++j) col_max[wave][tc * 8 + j] = cm[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) cm[j] = col_max[0][tc * 8 + j];
#pragma unroll
            for (int w = 1; w < kWaves; ++w)
#pragma unroll
                for (int j = 0; j < 8; ++j) cm[j] = fmaxf(cm[j], col_max[w][tc * 8 + j]);
#pragma unroll
            for (int j = 0; j < 8; ++j) ec[j] = block_exponent(cm[j], kFmaxExponent<FORMAT>);
        }
    }
    if (a.row.data) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float s = exp2_int(-er[i]);
            uint2 q;
            q.x = pack4<FORMAT>(to_float(p[i].v[0]), to_float(p[i].v[1]), to_float(p[i].v[2]), to_float(p[i].v[3]), s);
            q.y = pack4<FORMAT>(to_float(p[i].v[4]), to_float(p[i].v[5]), to_float(p[i].v[6]), to_float(p[i].v[7]), s);
            if (r0 + i >= a.rows) continue;
            *reinterpret_cast<uint2*>(a.row.data + (r0 + i) * a.row.ld + c0) = q;
            if (tc == 0) a.row.scales[tile_c * a.row.lds + r0 + i] = static_cast<uint8_t>(er[i] + 127);
        }
    }
    if (!a.col.data) return;
    // a column's 16-byte pieces are turned by its place among 8, so that
    // neither side meets in one bank
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t q = pack4<FORMAT>(to_float(p[0].v[j]), to_float(p[1].v[j]), to_float(p[2].v[j]),
                                         to_float(p[3].v[j]), exp2_int(-ec[j]));
        const int piece = (tr >> 2) ^ (tc & 7);
        *reinterpret_cast<uint32_t*>(turned + (tc * 8 + j) * kTile + piece * 16 + (tr & 3) * 4) = q;
        if (tr == 0 && c0 + j < a.cols) a.col.scales[tile_r * a.col.lds + c0 + j] = static_cast<uint8_t>(ec[j] + 127);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = k * 64 + (threadIdx.x >> 3), piece = threadIdx.x & 7;
        const int64_t col = static_cast<int64_t>(tile_c) * kTile + c;
        if (col >= a.cols) continue;
        const uint4 q = *reinterpret_cast<const uint4*>(turned + c * kTile + (piece ^ (c >> 3 & 7)) * 16);
        *reinterpret_cast<uint4*>(a.col.data + col * a.col.ld + static_cast<int64_t>(tile_r) * kTile + piece * 16) = q;
    }
}

template <typename T, int FORMAT> hipError_t launch_format(const QuantizeArgs& a, hipStream_t s)
{
    const int64_t tiles_c = (a.cols + kTile - 1) / kTile, tiles_r = (a.rows + kTile - 1) / kTile;
    if (!a.col.data && !a.whole)
        quantize_rows<T, FORMAT><<<static_cast<unsigned>((a.rows * tiles_c + 15) / 16), 256, 0, s>>>(a);
    else
        quantize_tile<T, FORMAT><<<static_cast<unsigned>(tiles_c * tiles_r), 512, 0, s>>>(a);
    return hipGetLastError();
}

template <typename T> hipError_t launch_type(const QuantizeArgs& a, int format, hipStream_t s)
{
    return format == FP8_E4M3 ? launch_format<T, FP8_E4M3>(a, s) : launch_format<T, FP8_E5M2>(a, s);
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
