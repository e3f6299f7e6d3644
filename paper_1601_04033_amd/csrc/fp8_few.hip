// 8-bit products that read their operands straight into registers: few rows
// on one side (up to 16: single tokens and small batches through a linear
// layer, or a layer of few outputs), and products so small that latency is
// all they cost.
//
// Bound by reading the larger operand once.  A block takes 16 or 32 of its
// rows, its 8 waves take the contraction's blocks of 128 in turn and read
// fragments straight from memory (16 rows of 128 bytes: whole lines), each
// value once; the few rows come from the caches.  The waves' sums are joined
// through LDS, so one launch writes the result, unless the larger operand's
// rows are too few for the CUs and long: then blocks take parts of the
// contraction, joined in order by a second launch.  1 x 4,096 x 16,384 (67 MB):
// 17.2 us, 3.9 TB/s, with weights that are in no cache (a ring of layers), 15.8
// where one layer follows itself, of which about 4 are the launch and x's
// quantization; 1 x 14,592 x 12,032 (176 MB): 39 and 34 us, 4.5 and 5.1 TB/s.
// Few unquantized activations (128 blocks of 128) are quantized on the way:
// every block does it again, into LDS, while its first loads of the larger
// operand are under way, which costs less than a launch before this one.
#include <string.h>

#include "fp8_math.hpp"

namespace fasgd {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;

struct Few {
    Fp8View big, few;
    const void* x;          // activations in place of few.data (FUSED)
    int64_t ldx;
    void* c;                // element (row of big, row of few) at c[r * stride_big + m * stride_few]
    int64_t stride_big, stride_few;
    int32_t c_dtype;
    int32_t accumulate;
    int32_t steps;          // blocks of 128 a split takes
    int64_t part;           // elements between the splits' products (0: one split)
};

#if defined(__HIP_DEVICE_COMPILE__)     // the host pass does not know buffer resources

// Rows of an operand from `row` on, 16 to a tile: lane l holds row l % 16 of
// a tile, and of a block of 128 the 16-byte chunks l / 16 of its two halves
// (both sides agree, so which of the contraction's values these are does not
// matter).  A row past the operand's end reads as 0.  Through buffers a load's
// address costs one scalar addition, and no register that a load under way
// still needs.
// Of the contraction the blocks from kb0 on.
struct Rows {
    static constexpr uint32_t kOutside = 0xf0000000u;
    __amdgpu_buffer_rsrc_t data;
    const uint8_t* scales;
    int64_t lds, scales_left;
    uint32_t ld, at;
    int lane;
    __device__ Rows(const Fp8View& v, int64_t row, int64_t kb0, int lane_)
        : data(buffer(v.data + row * v.ld + kb0 * kFp8Block, (v.rows - row) * v.ld - kb0 * kFp8Block)),
          scales(v.scales + kb0 * v.lds + row), lds(v.lds), scales_left(v.lds - row), ld(static_cast<uint32_t>(v.ld)),
          at((lane_ & 15) * static_cast<uint32_t>(v.ld) + (lane_ >> 4) * 16), lane(lane_)
    {
    }
    // (Non-temporal loads were slower, with the weights in the last-level cache
    // and in none: 1 x 14,592 x 12,032 46 against 34 and 48 against 39 us.)
    __device__ v8i read(int tile, int kb, bool in) const
    {
        const uint32_t p = in ? at + tile * 16 * ld : kOutside;
        const auto lo = __builtin_amdgcn_raw_buffer_load_b128(data, p, kb * kFp8Block, 0);
        const auto hi = __builtin_amdgcn_raw_buffer_load_b128(data, p + 64, kb * kFp8Block, 0);
        return join_chunks(__builtin_bit_cast(v4i, lo), __builtin_bit_cast(v4i, hi));
    }
    // the lane's row's scale with its three neighbours', and the scale alone:
    // a byte by itself would be widened, and so waited for, where the loop's
    // next loads begin
    __device__ uint32_t read_scale(int tile, int kb, bool in) const
    {
        return __builtin_amdgcn_raw_buffer_load_b32(buffer(scales + kb * lds, scales_left), in ? tile * 16 + (lane & 12) : kOutside, 0, 0);
    }
    __device__ int scale(uint32_t four) const { return four >> (lane & 3) * 8 & 0xff; }
};

#endif

// Activations in LDS: rows of k rounded up to 128 and 16 bytes (so that 16
// rows lie in different banks), then the scales, 16 to a block of 128.
struct Held {
    uint8_t* data;
    uint8_t* scales;
    int stride;
};
inline int held_stride(int64_t k) { return static_cast<int>((k + kFp8Block - 1) / kFp8Block * kFp8Block) + 16; }
inline size_t held_bytes(int64_t rows, int64_t k)
{
    return static_cast<size_t>(rows) * held_stride(k) + static_cast<size_t>((k + kFp8Block - 1) / kFp8Block) * 16;
}

// x quantized in e4m3 into LDS, 16 threads to a block of a row.  `first` is
// what a thread takes of the first blocks, loaded before anything else: 8
// elements, used where the row's end does not cut them.
// Whole registers until then: taken apart where they are loaded, they would be
// waited for there.
template <typename T> using Words = Pack<uint32_t, 2 * sizeof(T)>;
template <typename T> __device__ __forceinline__ Words<T> load_x(const Few& p, int i, int blocks)
{
    const int r = i / blocks, c = i % blocks * kFp8Block + (threadIdx.x & 15) * 8, k = static_cast<int>(p.few.k);
    Words<T> w;
    if (k >= 8) __builtin_memcpy(&w, static_cast<const T*>(p.x) + r * p.ldx + (c < k - 8 ? c : k - 8), sizeof w);
    return w;
}
template <typename T>
__device__ __forceinline__ void hold(const Few& p, const Held& h, int blocks, const Words<T>& first)
{
    const int lane = threadIdx.x & 15, rows = static_cast<int>(p.few.rows), k = static_cast<int>(p.few.k);
    auto item = [&](int i, const Words<T>& w) {
        Pack<T, 8> q;
        __builtin_memcpy(&q, &w, sizeof q);
        const int r = i / blocks, kb = i % blocks, c = kb * kFp8Block + lane * 8;
        if (c + 8 > k) {
            const T* x = static_cast<const T*>(p.x) + r * p.ldx;
#pragma unroll
            for (int j = 0; j < 8; ++j) q.v[j] = c + j < k ? x[c + j] : from_float<T>(0.0f);
        }
        float v[8], m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = to_float(q.v[j]);
            m = fmaxf(m, finite_abs(v[j]));
        }
        const int e = block_exponent(max_of_16(m), kFmaxExponent<FP8_E4M3>);
        const float s = exp2_int(-e);
        uint2 out;
        out.x = pack4<FP8_E4M3>(v[0], v[1], v[2], v[3], s);
        out.y = pack4<FP8_E4M3>(v[4], v[5], v[6], v[7], s);
        *reinterpret_cast<uint2*>(h.data + r * h.stride + c) = out;
        if (lane == 0) h.scales[kb * 16 + r] = static_cast<uint8_t>(e + 127);
    };
    int i = threadIdx.x >> 4;
    if (i < rows * blocks) item(i, first);      // apart from the rest, whose loads are waited for with all others
    for (i += kThreads / 16; i < rows * blocks; i += kThreads / 16) item(i, load_x<T>(p, i, blocks));
}

template <int FORMAT> __device__ __forceinline__ void widen_rows(const v8i& f, int scale, v8bf (&w)[4])
{
    const float s = __uint_as_float(static_cast<uint32_t>(scale) << 23);
#pragma unroll
    for (int t = 0; t < 4; ++t) w[t] = widen<FORMAT>(f[2 * t], f[2 * t + 1], s);
}

// MT tiles of 16 few rows, NT tiles of 16 of the larger operand's rows.
// X: the activations' type (FUSED), else unused.
template <typename X, bool FUSED, bool WIDE, int FBIG, int FFEW, int MT, int NT>
__global__ __launch_bounds__(kThreads, 4) void product_few(Few p, int held_stride)
{
#if defined(__HIP_DEVICE_COMPILE__)
    // blocks of 128 loaded while as many are multiplied, within 128 registers
    constexpr int kAhead = (FUSED ? 4 : 2) / (NT * MT);
    extern __shared__ __attribute__((aligned(16))) uint8_t dynamic[];
    __shared__ __attribute__((aligned(16))) float sums[kWaves][NT][MT][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * (16 * NT), m0 = static_cast<int64_t>(blockIdx.y) * (16 * MT);
    const int kb0 = blockIdx.z * p.steps, left = static_cast<int>((p.big.k + kFp8Block - 1) / kFp8Block) - kb0;
    const int blocks = left < p.steps ? left : p.steps;
    if constexpr (FUSED) {      // of x the columns of these blocks
        p.x = static_cast<const X*>(p.x) + static_cast<int64_t>(kb0) * kFp8Block;
        const int64_t k = p.few.k - static_cast<int64_t>(kb0) * kFp8Block, most = static_cast<int64_t>(blocks) * kFp8Block;
        p.few.k = k < most ? k : most;
    }
    v4f acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    constexpr int kFew = FUSED ? 1 : MT;
    struct Group {
        v8i big[kAhead][NT], few[kAhead][kFew];
        uint32_t scale_big[kAhead][NT], scale_few[kAhead][kFew];
    };
    const Rows big(p.big, r0, kb0, lane), few_rows(FUSED ? p.big : p.few, FUSED ? r0 : m0, kb0, lane);
    // A block past the last is loaded from outside the buffers, which moves
    // nothing (read as the last block it cost as much again: 1 x 4,096 x 16,384
    // 22 against 16 us), and not multiplied: with the same loads on every way
    // the waits are for what is needed.
    auto load = [&](Group& g, int k) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool in = k + u * kWaves < blocks;
            const int kb = in ? k + u * kWaves : 0;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                g.scale_big[u][n] = big.read_scale(n, kb, in);
                g.big[u][n] = big.read(n, kb, in);
            }
            if constexpr (!FUSED) {
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    g.scale_few[u][m] = few_rows.read_scale(m, kb, in);
                    g.few[u][m] = few_rows.read(m, kb, in);
                }
            }
        }
        // the compiler would put a scale's load where it is used, and wait there for all loads
        __builtin_amdgcn_sched_barrier(0);
    };
    Held h;
    h.data = dynamic;
    h.stride = held_stride;
    h.scales = dynamic + p.few.rows * held_stride;
    const int held_row = (lane & 15) < p.few.rows ? lane & 15 : static_cast<int>(p.few.rows) - 1;
    auto multiply = [&](const Group& g, int k) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int kb = k + u * kWaves;
            if (kb >= blocks) break;
            v8i few[MT];
            int scale_few[MT], scale_big[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) scale_big[n] = big.scale(g.scale_big[u][n]);
            if constexpr (FUSED) {
                const uint8_t* q = h.data + held_row * h.stride + kb * kFp8Block + (lane >> 4) * 16;
                few[0] = join_chunks(*reinterpret_cast<const v4i*>(q), *reinterpret_cast<const v4i*>(q + 64));
                scale_few[0] = h.scales[kb * 16 + held_row];
            } else {
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    few[m] = g.few[u][m];
                    scale_few[m] = few_rows.scale(g.scale_few[u][m]);
                }
            }
            if constexpr (WIDE) {
                v8bf wb[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) widen_rows<FBIG>(g.big[u][n], scale_big[n], wb[n]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    v8bf wf[4];
                    widen_rows<FFEW>(few[m], scale_few[m], wf);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int t = 0; t < 4; ++t)
                            acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[n][t], wf[t], acc[n][m], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int m = 0; m < MT; ++m)
                        acc[n][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                            g.big[u][n], few[m], acc[n][m], FBIG, FFEW, 0, scale_big[n], 0, scale_few[m]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    Group g[2];
    constexpr int kStep = kWaves * kAhead;
    auto run = [&] {    // with g[0] and g[1] under way
        for (int k = wave; k < blocks; k += 2 * kStep) {
            multiply(g[0], k);
            load(g[0], k + 2 * kStep);
            if (k + kStep >= blocks) break;
            multiply(g[1], k + kStep);
            load(g[1], k + 3 * kStep);
        }
    };
    if constexpr (FUSED) {
        const int i = threadIdx.x >> 4, last = static_cast<int>(p.few.rows) * blocks - 1;
        const Words<X> first = load_x<X>(p, i < last ? i : last, blocks);
        load(g[0], wave);
        load(g[1], wave + kStep);
        hold<X>(p, h, blocks, first);
        // only LDS has to be there: the loads above stay under way
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        run();
    } else if (blocks <= kStep) {   // one group of each wave holds all of the contraction
        load(g[0], wave);
        multiply(g[0], wave);
    } else {
        load(g[0], wave);
        load(g[1], wave + kStep);
        run();
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) *reinterpret_cast<v4f*>(sums[wave][n][m][lane]) = acc[n][m];
    __syncthreads();
    // element e of lane l: row 4 (l / 16) + e of the larger operand's tile, row l % 16 of the few's
    for (int i = threadIdx.x; i < NT * MT * 256; i += kThreads) {
        const int e = i & 3, l = i >> 2 & 63, m = (i >> 8) % MT, n = (i >> 8) / MT;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += sums[w][n][m][l][e];
        const int64_t row = r0 + n * 16 + (l >> 4) * 4 + e, col = m0 + m * 16 + (l & 15);
        if (row >= p.big.rows || col >= p.few.rows) continue;
        const int64_t at = row * p.stride_big + col * p.stride_few;
        if (p.c_dtype == DTYPE_F32) {
            float* c = static_cast<float*>(p.c) + blockIdx.z * p.part + at;
            *c = p.accumulate ? *c + s : s;
        } else if (p.c_dtype == DTYPE_BF16) {
            bf16* c = static_cast<bf16*>(p.c) + at;
            *c = from_float<bf16>(p.accumulate ? to_float(*c) + s : s);
        } else {
            f16* c = static_cast<f16*>(p.c) + at;
            *c = from_float<f16>(p.accumulate ? to_float(*c) + s : s);
        }
    }
#endif
}

// 32 rows a block where that still gives every CU one, else 16.
constexpr int64_t kRowsFor32 = 256 * 32;
template <typename X, bool FUSED, bool WIDE, int FBIG, int FFEW, int MT>
hipError_t launch_rows(const Few& p, hipStream_t s)
{
    const int64_t blocks = (p.few.k + kFp8Block - 1) / kFp8Block, held = blocks < p.steps ? blocks : p.steps;
    const size_t lds = FUSED ? held_bytes(p.few.rows, held * kFp8Block) : 0;
    const int stride = FUSED ? held_stride(held * kFp8Block) : 0;
    const unsigned splits = static_cast<unsigned>((blocks + p.steps - 1) / p.steps);
    const unsigned along = static_cast<unsigned>((p.few.rows + 16 * MT - 1) / (16 * MT));
    if (MT == 1 && p.big.rows >= kRowsFor32)
        product_few<X, FUSED, WIDE, FBIG, FFEW, MT, MT == 1 ? 2 : 1>
            <<<dim3(static_cast<unsigned>((p.big.rows + 31) / 32), along, splits), kThreads, lds, s>>>(p, stride);
    else
        product_few<X, FUSED, WIDE, FBIG, FFEW, MT, 1>
            <<<dim3(static_cast<unsigned>((p.big.rows + 15) / 16), along, splits), kThreads, lds, s>>>(p, stride);
    return hipGetLastError();
}

template <bool WIDE, int FBIG, int FFEW> hipError_t launch_few_rows(const Few& p, hipStream_t s)
{
    if (p.few.rows <= 16) return launch_rows<float, false, WIDE, FBIG, FFEW, 1>(p, s);
    return launch_rows<float, false, WIDE, FBIG, FFEW, 2>(p, s);
}

template <bool WIDE> hipError_t launch_formats(const Few& p, hipStream_t s)
{
    if (p.big.format == FP8_E4M3)
        return p.few.format == FP8_E4M3 ? launch_few_rows<WIDE, 0, 0>(p, s) : launch_few_rows<WIDE, 0, 1>(p, s);
    return p.few.format == FP8_E4M3 ? launch_few_rows<WIDE, 1, 0>(p, s) : launch_few_rows<WIDE, 1, 1>(p, s);
}

template <typename X, bool WIDE> hipError_t launch_fused(const Few& p, hipStream_t s)
{
    return p.big.format == FP8_E4M3 ? launch_rows<X, true, WIDE, 0, 0, 1>(p, s) : launch_rows<X, true, WIDE, 1, 0, 1>(p, s);
}

}  // namespace

// Beyond 16 rows, where these blocks of 16 x 32 outputs are estimated to take
// no more than 9.5 us, about what the tiles of fp8_product.hip take for so
// little: 3.2 us for each round of 512 blocks, and a block's reads of a block
// of 128 at 0.0034 us a row (500 x 500 x 500 5 against 7 to 10 us, 64 x 1,000
// x 3,000 8 against 10 to 12; but 1,000 x 784 x 128 12 against 7 to 9, 32 x
// 1,000 x 16,000 24 against 13 to 17).
bool fp8_few(int64_t m, int64_t n, int64_t k)
{
    const int64_t few = m < n ? m : n, big = m < n ? n : m;
    if (few <= 16) return true;
    const int64_t blocks = ((big + 15) / 16) * ((few + 31) / 32), rows = 16 + (few < 32 ? few : 32);
    const double per_cu = blocks > 256 ? static_cast<double>(blocks) / 256 : 1.0;
    return 3.2 * static_cast<double>((blocks + 511) / 512) +
               0.0034 * static_cast<double>(rows * ((k + kFp8Block - 1) / kFp8Block)) * per_cu <= 9.5;
}

// Each 32 blocks of x take a turn of a block's threads: beyond 4 turns a launch
// of their own costs less (16 x 2,048 x 16,384: 12 against 16 us, 12 x 2,000 x
// 8,192: 8.4 against 9.9).
bool fp8_linear_few(int64_t m, int64_t k) { return m <= 16 && m * ((k + kFp8Block - 1) / kFp8Block) <= 128; }

// Splits of the contraction of a product of up to 16 rows, whose blocks alone
// may leave most of the CUs idle: by the estimate above and that of the join,
// 4 us and 0.15 for each part (unsplit and split, fp32 out: 10 x 1,000 x 65,536
// 52 and 19 us, 16 x 16 x 2^20 904 and 24, 10 x 1,000 x 8,192 9.3 and 7.0; one
// token through 256 x 16,384 bf16 12.9 and 7.4; 10 x 4,096 x 16,384 stays at
// 19, two parts take 23).
int fp8_few_splits(int64_t m, int64_t n, int64_t k)
{
    const int64_t few = m < n ? m : n, big = m < n ? n : m;
    if (few < 1 || few > 16) return 1;
    const int64_t rows = big >= kRowsFor32 ? 32 : 16, wide = (big + rows - 1) / rows, blocks = (k + kFp8Block - 1) / kFp8Block;
    int best = 1;
    double least = 0.0;
    for (int s = 1; s <= 64 && (s == 1 || wide * s <= 512); s *= 2) {
        const double per_cu = wide * s > 256 ? static_cast<double>(wide * s) / 256 : 1.0;
        const double t = 0.0034 * static_cast<double>((rows + 16) * ((blocks + s - 1) / s)) * per_cu + (s > 1 ? 4.0 + 0.15 * s : 0.0);
        if (s == 1 || t < least) {
            least = t;
            best = s;
        }
    }
    const int64_t steps = (blocks + best - 1) / best;       // so that no split is empty
    return static_cast<int>((blocks + steps - 1) / steps);
}

namespace {

// The product as the kernel takes it, big the larger operand.  Splits leave
// their fp32 products in q's workspace.
Few few_of(const Fp8Product& q, const Fp8View& big, const Fp8View& few, bool big_is_a, int splits)
{
    const int64_t blocks = (q.a.k + kFp8Block - 1) / kFp8Block;
    Few p;
    memset(&p, 0, sizeof p);
    p.big = big;
    p.few = few;
    const int64_t ldc = splits > 1 ? q.b.rows : q.ldc;
    p.c = splits > 1 ? q.partial : q.c;
    p.stride_big = big_is_a ? ldc : 1;
    p.stride_few = big_is_a ? 1 : ldc;
    p.c_dtype = splits > 1 ? static_cast<int32_t>(DTYPE_F32) : q.c_dtype;
    p.accumulate = splits > 1 ? 0 : q.accumulate;
    p.steps = static_cast<int32_t>((blocks + splits - 1) / splits);
    p.part = splits > 1 ? q.a.rows * q.b.rows : 0;
    return p;
}

}  // namespace

hipError_t launch_fp8_few(const Fp8Product& q, hipStream_t s)
{
    const int splits = fp8_few_splits(q.a.rows, q.b.rows, q.a.k);
    const bool b_few = q.b.rows <= q.a.rows;
    const Few p = b_few ? few_of(q, q.a, q.b, true, splits) : few_of(q, q.b, q.a, false, splits);
    const hipError_t e = q.short_sums ? launch_formats<false>(p, s) : launch_formats<true>(p, s);
    return e == hipSuccess && splits > 1 ? launch_fp8_join(q, splits, s) : e;
}

hipError_t launch_fp8_linear_few(const void* x, int64_t ldx, const Fp8Product& q, hipStream_t s)
{
    const int splits = fp8_few_splits(q.a.rows, q.b.rows, q.a.k);
    Few p = few_of(q, q.b, q.a, false, splits);
    p.x = x;
    p.ldx = ldx;
    hipError_t e;
    if (q.c_dtype == DTYPE_F32) e = launch_fused<float, true>(p, s);
    else if (q.c_dtype == DTYPE_BF16) e = q.short_sums ? launch_fused<bf16, false>(p, s) : launch_fused<bf16, true>(p, s);
    else e = q.short_sums ? launch_fused<f16, false>(p, s) : launch_fused<f16, true>(p, s);
    return e == hipSuccess && splits > 1 ? launch_fp8_join(q, splits, s) : e;
}

}  // namespace fasgd
