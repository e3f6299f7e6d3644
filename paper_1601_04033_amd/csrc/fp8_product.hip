// client_fp8_matmul: C = A B^T of two 8-bit operands with a power-of-two scale
// per row and block of 128 along the contraction.
//
//   c[m][n] = sum_kb 2^(ea[kb][m] + eb[kb][n]) sum_{k in kb} qa[m][k] qb[n][k]
//
// Two arithmetics, by the type of c:
//   16-bit c: the scaled 8-bit matrix instruction
//     (v_mfma_scale_f32_32x32x64_f8f6f4), which takes one exponent byte per
//     row and 32 values of each operand, so scales cost no arithmetic.  It
//     sums each 8 consecutive products to 2^-13 of the largest of them (what
//     lies below is cut off) and everything beyond that in fp32: with
//     random operands an error of about 3e-5 of c's size, a hundredth of
//     c's rounding to bf16 and a seventh of fp16's.
//   fp32 c: 8-bit values times their scales are exact in bf16, whose
//     instruction (v_mfma_f32_32x32x16_bf16) sums in fp32 throughout: half the
//     rate, and as accurate as c can hold.
#include "client_kernels.hpp"

namespace fasgd {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;       // 4 waves, 2 x 2 of them
constexpr int kBytes = kFp8Block;   // contraction per stage: one scale each way
constexpr int kMaxSplits = 16;

// A wave owns W x W outputs as (W/32)^2 matrix tiles.  Row r of tile i is the
// wave's row (W/32) r + i, so a lane's scales for its tiles are neighbouring
// bytes (one load; the instruction picks the byte) and its outputs are
// neighbouring columns.
template <int W> struct Geometry {
    static constexpr int kTiles = W / 32;
    static constexpr int kSide = 2 * W;                         // block tile
    static constexpr int kStage = kSide * kBytes;               // LDS bytes of one operand's stage
    static constexpr int kLoads = kStage / (kThreads * 16);     // 16-byte loads per thread and operand
};

// The 16-byte chunk of a row that lies in slot s of its 128 LDS bytes.  Rows
// that one read touches together (kTiles apart) get their chunks in
// different banks.
template <int W> __device__ __forceinline__ int swizzle(int row) { return (row / Geometry<W>::kTiles) & 7; }

typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

// One operand's stage, global memory straight to LDS.
template <int W>
__device__ __forceinline__ void load_stage(const uint8_t* base, const uint32_t (&offset)[Geometry<W>::kLoads],
                                           uint8_t* stage, int wave)
{
#pragma unroll
    for (int p = 0; p < Geometry<W>::kLoads; ++p)
        __builtin_amdgcn_global_load_lds((global_ptr)(base + offset[p]),
                                         (lds_ptr)(stage + (p * 4 + wave) * 1024), 16, 0, 0);
}

// The fragments of one half stage (64 of the contraction): lane l holds row
// l % 32 of each tile, two chunks of it.
template <int W>
__device__ __forceinline__ void read_fragments(const uint8_t* stage, int row, int lane, int half,
                                               v8i (&f)[Geometry<W>::kTiles])
{
#pragma unroll
    for (int i = 0; i < Geometry<W>::kTiles; ++i) {
        const int r = row + i;
        const uint8_t* p = stage + r * kBytes;
        const int c = half * 4 + (lane >> 5) * 2;
        const v4i lo = *reinterpret_cast<const v4i*>(p + ((c ^ swizzle<W>(r)) * 16));
        const v4i hi = *reinterpret_cast<const v4i*>(p + (((c + 1) ^ swizzle<W>(r)) * 16));
        f[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

template <int FA, int FB, int I, int J, int N>
__device__ __forceinline__ void multiply_tile(v16f (&acc)[N][N], const v8i (&a)[N], const v8i (&b)[N], int sa, int sb)
{
    acc[I][J] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[I], b[J], acc[I][J], FA, FB, I, sa, J, sb);
    if constexpr (J + 1 < N) multiply_tile<FA, FB, I, J + 1, N>(acc, a, b, sa, sb);
    else if constexpr (I + 1 < N) multiply_tile<FA, FB, I + 1, 0, N>(acc, a, b, sa, sb);
}

// 8 of a fragment's values (dwords 2 T and 2 T + 1) times 2^(scale - 127), as bf16: exact.
template <int FORMAT, int T> __device__ __forceinline__ v8bf widen(const v8i& f, float scale)
{
    v2bf x[4];
    if constexpr (FORMAT == FP8_E4M3) {
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * T], scale, false);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * T], scale, true);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * T + 1], scale, false);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * T + 1], scale, true);
    } else {
        x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(f[2 * T], scale, false);
        x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(f[2 * T], scale, true);
        x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(f[2 * T + 1], scale, false);
        x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(f[2 * T + 1], scale, true);
    }
    return v8bf{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

// byte I of packed scales as the power of two it stands for
template <int I> __device__ __forceinline__ float scale_value(int scales)
{
    return __uint_as_float((static_cast<uint32_t>(scales) >> (8 * I) & 0xffu) << 23);
}

// The same half stage with both operands widened to bf16, 8 values of each
// lane at a time.
template <int FA, int FB, int T, int N>
__device__ __forceinline__ void multiply_wide(v16f (&acc)[N][N], const v8i (&a)[N], const v8i (&b)[N],
                                              const float (&sa)[N], const float (&sb)[N])
{
    v8bf wa[N], wb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        wa[i] = widen<FA, T>(a[i], sa[i]);
        wb[i] = widen<FB, T>(b[i], sb[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa[i], wb[j], acc[i][j], 0, 0, 0);
    if constexpr (T + 1 < 4) multiply_wide<FA, FB, T + 1, N>(acc, a, b, sa, sb);
}

template <int N> __device__ __forceinline__ void scale_values(int scales, float (&s)[N])
{
    s[0] = scale_value<0>(scales);
    s[1] = scale_value<1>(scales);
    if constexpr (N == 4) {
        s[2] = scale_value<2>(scales);
        s[3] = scale_value<3>(scales);
    }
}

template <int N> __device__ __forceinline__ int load_scales(const uint8_t* p)
{
    if constexpr (N == 4) return *reinterpret_cast<const int*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
}

template <typename T, int N>
__device__ __forceinline__ void store_row(T* c, int64_t n, int64_t cols, const float (&v)[N], bool add)
{
    if (n + N <= cols) {
        Pack<T, N> p;
        if (add) p = load_pack<T, N>(c + n);
#pragma unroll
        for (int j = 0; j < N; ++j) p.v[j] = from_float<T>(add ? to_float(p.v[j]) + v[j] : v[j]);
        store_pack(c + n, p);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (n + j < cols) c[n + j] = from_float<T>(add ? to_float(c[n + j]) + v[j] : v[j]);
}

struct Grid {
    int32_t tiles_m, tiles_n, splits, steps;    // steps: stages per split
};

template <int W, int FA, int FB, bool WIDE>
__global__ __launch_bounds__(kThreads, 1) void product(Fp8Product p, Grid g)
{
    using G = Geometry<W>;
    constexpr int N = G::kTiles;
    __shared__ __attribute__((aligned(16))) uint8_t a0[G::kStage], b0[G::kStage], a1[G::kStage], b1[G::kStage];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Consecutive blocks go to the 8 XCDs in turn: give each XCD a run of
    // tiles, 8 rows of tiles deep, so that its L2 serves their operands.
    const int tiles = g.tiles_m * g.tiles_n;
    int id = blockIdx.x % tiles;
    const int split = blockIdx.x / tiles;
    {
        const int xcd = id & 7, each = tiles >> 3, extra = tiles & 7;
        id = xcd * each + (xcd < extra ? xcd : extra) + (id >> 3);
        const int deep = 8 * g.tiles_n, group = id / deep, first = group * 8;
        const int rows = g.tiles_m - first < 8 ? g.tiles_m - first : 8;
        const int in = id - group * deep;
        id = (first + in % rows) * g.tiles_n + in / rows;
    }
    const int64_t m0 = static_cast<int64_t>(id / g.tiles_n) * G::kSide, n0 = static_cast<int64_t>(id % g.tiles_n) * G::kSide;
    const int64_t blocks = (p.a.k + kBytes - 1) / kBytes;
    const int64_t kb0 = static_cast<int64_t>(split) * g.steps;
    const int steps = static_cast<int>(blocks - kb0 < g.steps ? blocks - kb0 : g.steps);

    // A row past the operand's end is read as its last row: its outputs are
    // not stored.
    uint32_t off_a[G::kLoads], off_b[G::kLoads];
#pragma unroll
    for (int q = 0; q < G::kLoads; ++q) {
        const int row = (q * 4 + wave) * 8 + (lane >> 3);
        const uint32_t chunk = ((lane & 7) ^ swizzle<W>(row)) * 16;
        const int64_t ra = p.a.rows - m0 - 1 < row ? p.a.rows - m0 - 1 : row;
        const int64_t rb = p.b.rows - n0 - 1 < row ? p.b.rows - n0 - 1 : row;
        off_a[q] = static_cast<uint32_t>(ra * p.a.ld) + chunk;
        off_b[q] = static_cast<uint32_t>(rb * p.b.ld) + chunk;
    }
    const uint8_t* ga = p.a.data + m0 * p.a.ld + kb0 * kBytes;
    const uint8_t* gb = p.b.data + n0 * p.b.ld + kb0 * kBytes;
    const int row_a = (wave >> 1) * W + (lane & 31) * N, row_b = (wave & 1) * W + (lane & 31) * N;
    const int64_t sra = m0 + row_a < p.a.lds - N ? m0 + row_a : p.a.lds - N;
    const int64_t srb = n0 + row_b < p.b.lds - N ? n0 + row_b : p.b.lds - N;
    const uint8_t* sa = p.a.scales + kb0 * p.a.lds + sra;
    const uint8_t* sb = p.b.scales + kb0 * p.b.lds + srb;

    v16f acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    auto stage = [&](int k, uint8_t* a, uint8_t* b) {
        load_stage<W>(ga + static_cast<int64_t>(k) * kBytes, off_a, a, wave);
        load_stage<W>(gb + static_cast<int64_t>(k) * kBytes, off_b, b, wave);
    };
    auto compute = [&](const uint8_t* a, const uint8_t* b, int xa, int xb) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            v8i fa[N], fb[N];
            read_fragments<W>(a, row_a, lane, half, fa);
            read_fragments<W>(b, row_b, lane, half, fb);
            if constexpr (WIDE) {
                float wa[N], wb[N];
                scale_values<N>(xa, wa);
                scale_values<N>(xb, wb);
                multiply_wide<FA, FB, 0, N>(acc, fa, fb, wa, wb);
            } else {
                multiply_tile<FA, FB, 0, 0, N>(acc, fa, fb, xa, xb);
            }
        }
    };
    stage(0, a0, b0);
    for (int k = 0; k < steps; k += 2) {
        int xa = load_scales<N>(sa + k * p.a.lds), xb = load_scales<N>(sb + k * p.b.lds);
        __syncthreads();
        if (k + 1 < steps) stage(k + 1, a1, b1);
        compute(a0, b0, xa, xb);
        if (k + 1 >= steps) break;
        xa = load_scales<N>(sa + (k + 1) * p.a.lds);
        xb = load_scales<N>(sb + (k + 1) * p.b.lds);
        __syncthreads();
        if (k + 2 < steps) stage(k + 2, a0, b0);
        compute(a1, b1, xa, xb);
    }

    const int64_t n = n0 + row_b;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t m = m0 + (wave >> 1) * W + (8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * N + i;
            if (m >= p.a.rows || n >= p.b.rows) continue;
            float v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = acc[i][j][r];
            if (g.splits > 1) {
                store_row<float, N>(p.partial + (split * p.a.rows + m) * p.b.rows, n, p.b.rows, v, false);
            } else if (p.c_dtype == DTYPE_F32) {
                store_row<float, N>(static_cast<float*>(p.c) + m * p.ldc, n, p.b.rows, v, p.accumulate);
            } else if (p.c_dtype == DTYPE_BF16) {
                store_row<bf16, N>(static_cast<bf16*>(p.c) + m * p.ldc, n, p.b.rows, v, p.accumulate);
            } else {
                store_row<f16, N>(static_cast<f16*>(p.c) + m * p.ldc, n, p.b.rows, v, p.accumulate);
            }
        }
}

// The splits' partial products joined in order (splits = 0: an empty
// contraction).
template <typename T> __global__ __launch_bounds__(256) void join(Fp8Product p, int splits)
{
    const int64_t n = p.b.rows, total = p.a.rows * n;
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    for (int e = 0; e < 4; ++e) {
        if (i + e >= total) return;
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += p.partial[k * total + i + e];
        T* c = static_cast<T*>(p.c) + (i + e) / n * p.ldc + (i + e) % n;
        *c = from_float<T>(p.accumulate ? to_float(*c) + s : s);
    }
}

hipError_t launch_join(const Fp8Product& p, int splits, hipStream_t s)
{
    const int64_t quads = (p.a.rows * p.b.rows + 3) / 4;
    const unsigned blocks = static_cast<unsigned>((quads + 255) / 256);
    if (p.c_dtype == DTYPE_F32) join<float><<<blocks, 256, 0, s>>>(p, splits);
    else if (p.c_dtype == DTYPE_BF16) join<bf16><<<blocks, 256, 0, s>>>(p, splits);
    else join<f16><<<blocks, 256, 0, s>>>(p, splits);
    return hipGetLastError();
}

// 256 x 256 tiles where they fill the chip, else 128 x 128 ones, their
// contraction split until 256 blocks are there (at least 4 stages each).
struct Plan {
    bool large;
    Grid g;
};
Plan plan_of(int64_t m, int64_t n, int64_t k)
{
    Plan p;
    const int64_t large = ((m + 255) / 256) * ((n + 255) / 256);
    p.large = large >= 192;
    const int64_t side = p.large ? 256 : 128;
    p.g.tiles_m = static_cast<int32_t>((m + side - 1) / side);
    p.g.tiles_n = static_cast<int32_t>((n + side - 1) / side);
    const int64_t tiles = static_cast<int64_t>(p.g.tiles_m) * p.g.tiles_n, blocks = (k + kBytes - 1) / kBytes;
    int64_t splits = 1;
    if (!p.large && tiles < 256) {
        splits = (256 + tiles - 1) / tiles;
        if (splits > blocks / 4) splits = blocks / 4;
        if (splits > kMaxSplits) splits = kMaxSplits;
        if (splits < 1) splits = 1;
    }
    p.g.steps = static_cast<int32_t>((blocks + splits - 1) / splits);
    p.g.splits = static_cast<int32_t>((blocks + p.g.steps - 1) / p.g.steps);
    return p;
}

template <int FA, int FB> hipError_t launch_formats(const Fp8Product& p, const Plan& plan, hipStream_t s)
{
    const unsigned blocks = static_cast<unsigned>(plan.g.tiles_m) * plan.g.tiles_n * plan.g.splits;
    if (p.c_dtype == DTYPE_F32) {
        if (plan.large) product<128, FA, FB, true><<<blocks, kThreads, 0, s>>>(p, plan.g);
        else product<64, FA, FB, true><<<blocks, kThreads, 0, s>>>(p, plan.g);
    } else {
        if (plan.large) product<128, FA, FB, false><<<blocks, kThreads, 0, s>>>(p, plan.g);
        else product<64, FA, FB, false><<<blocks, kThreads, 0, s>>>(p, plan.g);
    }
    return hipGetLastError();
}

}  // namespace

size_t fp8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m < 1 || n < 1 || k < 1) return 0;
    const Plan p = plan_of(m, n, k);
    return p.g.splits > 1 ? sizeof(float) * static_cast<size_t>(p.g.splits) * static_cast<size_t>(m) * static_cast<size_t>(n) : 0;
}

hipError_t launch_fp8_product(const Fp8Product& p, hipStream_t s)
{
    if (p.a.k == 0) return launch_join(p, 0, s);
    const Plan plan = plan_of(p.a.rows, p.b.rows, p.a.k);
    hipError_t e;
    if (p.a.format == FP8_E4M3)
        e = p.b.format == FP8_E4M3 ? launch_formats<0, 0>(p, plan, s) : launch_formats<0, 1>(p, plan, s);
    else
        e = p.b.format == FP8_E4M3 ? launch_formats<1, 0>(p, plan, s) : launch_formats<1, 1>(p, plan, s);
    if (e == hipSuccess && plan.g.splits > 1) e = launch_join(p, plan.g.splits, s);
    return e;
}

}  // namespace fasgd
