// client_fp8_quantize: a matrix in 8-bit floating point with one power-of-two
// scale per block of 128, in row form, transposed, or both from one read.
//
// Bound by memory: x is read once, and each form written in whole lines.
// 8,192 x 16,384 bf16, both forms: 106 us, 5.1 TB/s; rows alone 4,099 x 5,003
// fp16: 13 us, 4.6 TB/s.  A matrix of a few tiles costs 5 to 7 us, the chain
// of one tile's steps.
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
    const int64_t i = a.first + static_cast<int64_t>(blockIdx.x) * 16 + (threadIdx.x >> 4);
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

// Magnitudes of 8 neighbouring elements as unsigned integers, whose order is
// that of the magnitudes (infinity and NaN above all others): 16-bit types two
// to a register, compared two at a time.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Magnitudes {
    u16x2 m[4];
    __device__ static constexpr uint32_t kInfinity = __is_same(T, bf16) ? 0x7f80u : 0x7c00u;
    __device__ void of(const Pack<T, 8>& p)
    {
        uint32_t w[4];
        __builtin_memcpy(w, &p, sizeof w);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu);
    }
    __device__ void join(const Magnitudes& o)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = __builtin_elementwise_max(m[i], o.m[i]);
    }
    __device__ uint32_t largest() const
    {
        const u16x2 x = __builtin_elementwise_max(__builtin_elementwise_max(m[0], m[1]), __builtin_elementwise_max(m[2], m[3]));
        return x[0] > x[1] ? x[0] : x[1];
    }
    __device__ static float value(uint32_t bits) { return to_float(__builtin_bit_cast(T, static_cast<uint16_t>(bits))); }
    __device__ float at(int j) const { return value(m[j / 2][j % 2]); }
};
template <> struct Magnitudes<float> {
    uint32_t m[8];
    __device__ static constexpr uint32_t kInfinity = 0x7f800000u;
    __device__ void of(const Pack<float, 8>& p)
    {
        __builtin_memcpy(m, &p, sizeof m);
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] &= 0x7fffffffu;
    }
    __device__ void join(const Magnitudes& o)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = m[i] > o.m[i] ? m[i] : o.m[i];
    }
    __device__ uint32_t largest() const
    {
        uint32_t x = m[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) x = x > m[i] ? x : m[i];
        return x;
    }
    __device__ static float value(uint32_t bits) { return __uint_as_float(bits); }
    __device__ float at(int j) const { return __uint_as_float(m[j]); }
};

// Four finite values times s, within the format's range, rounded to nearest even.
template <int FORMAT> __device__ __forceinline__ uint32_t pack4_finite(float x0, float x1, float x2, float x3, float s)
{
    int v = 0;
    if constexpr (FORMAT == FP8_E4M3) {
        v = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * s, x1 * s, v, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(x2 * s, x3 * s, v, true);
    } else {
        v = __builtin_amdgcn_cvt_pk_bf8_f32(x0 * s, x1 * s, v, false);
        v = __builtin_amdgcn_cvt_pk_bf8_f32(x2 * s, x3 * s, v, true);
    }
    return static_cast<uint32_t>(v);
}

// One 128 x 128 tile per block of 512 threads; thread (tr, tc) holds rows
// 4 tr .. + 3 of columns 8 tc .. + 7: few enough registers for 2 or 3 blocks
// per CU, which read while others write.  A tile that
// holds an infinity or a NaN takes its maxima again, of the finite values.
// The transposed form passes through LDS, so that it too is written in
// 16-byte pieces of whole lines.
template <typename T, int FORMAT>
__global__ __launch_bounds__(512, sizeof(T) == 4 ? 4 : 6) void quantize_tile(QuantizeArgs a)
{
    constexpr int R = 4, kWaves = 8;
    __shared__ float col_max[kWaves][kTile];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kTile * kTile];
    __shared__ float whole_max[kWaves];
    __shared__ __attribute__((aligned(16))) int col_exponent[kTile];
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int tiles_c = static_cast<int>((a.cols + kTile - 1) / kTile);
    const int tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const int64_t r0 = static_cast<int64_t>(tile_r) * kTile + tr * R;
    const int64_t c0 = static_cast<int64_t>(tile_c) * kTile + tc * 8;
    const T* x = static_cast<const T*>(a.x);
    Pack<T, 8> p[R];
    if (static_cast<int64_t>(tile_r + 1) * kTile <= a.rows && static_cast<int64_t>(tile_c + 1) * kTile <= a.cols) {
#pragma unroll
        for (int i = 0; i < R; ++i) p[i] = load_pack<T, 8>(x + (r0 + i) * a.ldx + c0);
    } else {
        // a row past the end is read as the last one, so that a thread's loads are under way together
        const bool whole = c0 + 8 <= a.cols;
        if (whole) {
#pragma unroll
            for (int i = 0; i < R; ++i) p[i] = load_pack<T, 8>(x + (r0 + i < a.rows ? r0 + i : a.rows - 1) * a.ldx + c0);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool in = r0 + i < a.rows;
            if (whole && in) continue;
            if (!whole && in && c0 < a.cols) {
                p[i] = load8(x + (r0 + i) * a.ldx, c0, a.cols);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) p[i].v[j] = from_float<T>(0.0f);
            }
        }
    }
    float rm[R], cm[8];     // largest magnitudes: a thread's, then the tile's
    Magnitudes<T> all;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        Magnitudes<T> m;
        m.of(p[i]);
        rm[i] = Magnitudes<T>::value(m.largest());
        if (i == 0) all = m;
        else all.join(m);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) cm[j] = all.at(j);
    auto join16 = [](float m) {     // over the lanes 16, 32 and 48 away
        const Pair p = across<16>(m);
        const Pair q = across<32>(fmaxf(p.x, p.y));
        return fmaxf(q.x, q.y);
    };
    // the column maxima of a wave's 16 rows go to LDS, or the wave's maximum
    auto share = [&] {
        if (a.whole) {
            const float m = join16(max_of_16(fmaxf(fmaxf(rm[0], rm[1]), fmaxf(rm[2], rm[3]))));
            if ((threadIdx.x & 63) == 0) whole_max[wave] = m;
            return;
        }
        float m[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) m[j] = join16(cm[j]);
        if ((threadIdx.x & 63) < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) col_max[wave][tc * 8 + j] = m[j];
        }
    };
    const bool joined = a.whole || a.col.data;
    if (joined) share();
    const bool finite = __syncthreads_or(all.largest() >= Magnitudes<T>::kInfinity) == 0;
    if (!finite) {
#pragma unroll
        for (int j = 0; j < 8; ++j) cm[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rm[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = finite_abs(to_float(p[i].v[j]));
                rm[i] = fmaxf(rm[i], f);
                cm[j] = fmaxf(cm[j], f);
            }
        }
        if (joined) share();
        __syncthreads();
    }
    int er[R], ec[8];
    if (a.whole) {
        float m = whole_max[0];
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
        if (a.col.data && threadIdx.x < kTile) {
            // once a column: in every thread these were a quarter of its work
            float m = col_max[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) m = fmaxf(m, col_max[w][threadIdx.x]);
            col_exponent[threadIdx.x] = block_exponent(m, kFmaxExponent<FORMAT>);
        }
    }
    auto pack = [&](T x0, T x1, T x2, T x3, float s) {
        return finite ? pack4_finite<FORMAT>(to_float(x0), to_float(x1), to_float(x2), to_float(x3), s)
                      : pack4<FORMAT>(to_float(x0), to_float(x1), to_float(x2), to_float(x3), s);
    };
    if (a.row.data) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float s = exp2_int(-er[i]);
            uint2 q;
            q.x = pack(p[i].v[0], p[i].v[1], p[i].v[2], p[i].v[3], s);
            q.y = pack(p[i].v[4], p[i].v[5], p[i].v[6], p[i].v[7], s);
            if (r0 + i >= a.rows) continue;
            *reinterpret_cast<uint2*>(a.row.data + (r0 + i) * a.row.ld + c0) = q;
            if (tc == 0) a.row.scales[tile_c * a.row.lds + r0 + i] = static_cast<uint8_t>(er[i] + 127);
        }
    }
    if (!a.col.data) return;
    if (!a.whole) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) ec[j] = col_exponent[tc * 8 + j];
    }
    // a column's 16-byte pieces are turned by its place among 8, so that
    // neither side meets in one bank
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t q = pack(p[0].v[j], p[1].v[j], p[2].v[j], p[3].v[j], exp2_int(-ec[j]));
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
    if (a.col.data || a.whole) {
        quantize_tile<T, FORMAT><<<static_cast<unsigned>(tiles_c * tiles_r), 512, 0, s>>>(a);
        return hipGetLastError();
    }
    QuantizeArgs q = a;
    const int64_t blocks = (a.rows * tiles_c + 15) / 16;
    hipError_t e = hipSuccess;
    for (int64_t b = 0; b < blocks && e == hipSuccess; b += kLaunchBlocks) {
        q.first = b * 16;
        quantize_rows<T, FORMAT><<<static_cast<unsigned>(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks), 256, 0, s>>>(q);
        e = hipGetLastError();
    }
    return e;
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
