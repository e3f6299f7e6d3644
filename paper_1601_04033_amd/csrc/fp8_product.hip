// client_fp8_matmul: C = A B^T of two 8-bit operands with a power-of-two scale
// per row and block of 128 along the contraction.
//
//   c[m][n] = sum_kb 2^(ea[kb][m] + eb[kb][n]) sum_{k in kb} qa[m][k] qb[n][k]
//
// Two arithmetics:
//   full sums (all products but those of the next kind): 8-bit values times
//     their scales are exact in bf16 (from 2^-133 on), whose instruction
//     (v_mfma_f32_32x32x16_bf16) sums in fp32 throughout.
//   short sums, where the caller asks for them and c has 16 bits: the scaled
//     8-bit instruction (v_mfma_scale_f32_32x32x64_f8f6f4), which takes one
//     exponent byte per row and 32 values of each operand, so scales cost no
//     arithmetic, at twice the rate.  It sums each 8 consecutive products to
//     2^-13 of the largest of them (what lies below is cut off) and
//     everything beyond that in fp32: where large products of a group cancel,
//     its small ones are lost.  With random operands that is an error of
//     about 3e-5 of c's size, a hundredth of c's rounding to bf16 and a
//     seventh of fp16's.
//
// Bound by the matrix instructions where tiles fill the chip: 8,192^3 with
// bf16 outputs in 746 us (full sums, 1,470 TFLOP/s; the library's bf16 product
// 1,450) and 377 us (short sums, 2,920; the library's 8-bit product 2,970); fp32
// outputs 780 us.  Below, by whole rounds of tiles and about 8 us of launch, first
// loads and last stores.
#include "fp8_math.hpp"

namespace fasgd {
namespace {

constexpr int kThreads = 256;       // 4 waves
constexpr int kBytes = kFp8Block;   // contraction per stage: one scale each way
constexpr int kMaxSplits = 16;

// A wave owns W x W outputs as (W/32)^2 matrix tiles, and WM of the block's 4
// waves stand along a's rows.  Row r of tile i is the wave's row
// (W/32) r + i, so a lane's scales for its tiles are neighbouring bytes (one
// load; the instruction picks the byte) and its outputs are neighbouring
// columns.
template <int W, int WM> struct Geometry {
    static constexpr int kTiles = W / 32;
    static constexpr int kWavesN = 4 / WM;
    static constexpr int kRowsA = W * WM, kRowsB = W * kWavesN;             // block tile
    static constexpr int kStageA = kRowsA * kBytes, kStageB = kRowsB * kBytes;  // LDS bytes of a stage
    static constexpr int kLoadsA = kStageA / (kThreads * 16);               // 16-byte loads per thread
    static constexpr int kLoadsB = kStageB / (kThreads * 16);
};

#if defined(__HIP_DEVICE_COMPILE__)     // the host pass does not know buffer resources

// A stage in LDS: the rows that one read touches together, row r of tile i
// for r = 0 .. 31, are neighbours, and the 16-byte chunk c of a row's 128
// bytes lies in slot c ^ (r / 2 mod 8), so that 16 lanes meet in no bank.
__device__ __forceinline__ int slot(int c, int r) { return c ^ (r >> 1 & 7); }

typedef __attribute__((address_space(3))) void* lds_ptr;

// A stage is worked through in sub-steps of 1,024 matrix cycles per wave (at
// W = 128): 64 of the contraction with short sums, 32 with full ones.  A
// sub-step's fragments (lane l: row l % 32 of a tile, the 16-byte chunks of
// its half of the sub-step) are read while the one before is multiplied.
template <bool WIDE> struct Sub {
    static constexpr int kCount = WIDE ? 4 : 2;     // per stage
    static constexpr int kChunks = WIDE ? 1 : 2;    // 16-byte chunks per lane and row
};
template <bool WIDE, int N> struct Fragments {
    v4i a[N][Sub<WIDE>::kChunks], b[N][Sub<WIDE>::kChunks];
};

// Where a lane finds its chunks: the first tile's row, and the swizzled place
// of each of its four chunks in a row's 128 bytes.  Which of the contraction's
// values a lane holds does not matter as long as both operands agree.
struct Places {
    int row_a, row_b;
    int chunk[4];
};
// Read q of the 2 N kChunks reads of a sub-step's fragments.
template <bool WIDE, int N>
__device__ __forceinline__ void read_one(Fragments<WIDE, N>& f, const uint8_t* a, const uint8_t* b, const Places& at,
                                         int s, int q)
{
    constexpr int C = Sub<WIDE>::kChunks;
    const int i = q / (2 * C), rest = q % (2 * C), c = rest % C;
    const uint8_t* p = rest < C ? a + at.row_a : b + at.row_b;
    const v4i x = *reinterpret_cast<const v4i*>(p + at.chunk[s * C + c] + i * 32 * kBytes);
    if (rest < C) f.a[i][c] = x;
    else f.b[i][c] = x;
}

// byte i of packed scales as the power of two it stands for
__device__ __forceinline__ float scale_value(int scales, int i)
{
    return __uint_as_float((static_cast<uint32_t>(scales) >> (8 * i) & 0xffu) << 23);
}

template <int N> struct Wide {
    v8bf a[N], b[N];
};
// Half t of a sub-step's fragments, widened.
template <int FA, int FB, int N>
__device__ __forceinline__ void widen_half(Wide<N>& w, const Fragments<true, N>& f, int t, int sa, int sb)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        w.a[i] = widen<FA>(f.a[i][0][2 * t], f.a[i][0][2 * t + 1], scale_value(sa, i));
        w.b[i] = widen<FB>(f.b[i][0][2 * t], f.b[i][0][2 * t + 1], scale_value(sb, i));
    }
}

template <int FA, int FB, int I, int J, int N>
__device__ __forceinline__ void multiply_scaled(v16f (&acc)[N][N], const Fragments<false, N>& f, int sa, int sb)
{
    acc[I][J] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join_chunks(f.a[I][0], f.a[I][1]),
                                                                join_chunks(f.b[J][0], f.b[J][1]), acc[I][J], FA, FB,
                                                                I, sa, J, sb);
    if constexpr (J + 1 < N) multiply_scaled<FA, FB, I, J + 1, N>(acc, f, sa, sb);
    else if constexpr (I + 1 < N) multiply_scaled<FA, FB, I + 1, 0, N>(acc, f, sa, sb);
}
template <int N> __device__ __forceinline__ void multiply_wide(v16f (&acc)[N][N], const Wide<N>& w)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.a[i], w.b[j], acc[i][j], 0, 0, 0);
}

// Orders of the instructions of a sub-step for the compiler's scheduler:
// between two matrix instructions go one LDS read, the loads of the stage
// after next, and the conversions of what is multiplied next.
template <int MFMA, int READS, int LOADS, int VALU, int I = 0> __device__ __forceinline__ void interleave()
{
    constexpr int kMfma = 0x8, kDsRead = 0x100, kVmem = 0x20, kValu = 0x2;
    constexpr int kReads = (I + 1) * READS / MFMA - I * READS / MFMA, kLoads = (I + 1) * LOADS / MFMA - I * LOADS / MFMA;
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(kDsRead, kReads, 0);
    if constexpr (kLoads > 0) __builtin_amdgcn_sched_group_barrier(kVmem, kLoads, 0);
    if constexpr (VALU > 0) __builtin_amdgcn_sched_group_barrier(kValu, VALU / MFMA, 0);
    if constexpr (I + 1 < MFMA) interleave<MFMA, READS, LOADS, VALU, I + 1>();
}

// A lane's N neighbouring scales, the first in byte 0.  p: as many bytes on,
// but no further than 4 before the scales' end (N = 3: then `shift` bits before them).
template <int N> __device__ __forceinline__ int load_scales(const uint8_t* p, int shift)
{
    if constexpr (N == 4) return *reinterpret_cast<const int*>(p);
    if constexpr (N == 2) return *reinterpret_cast<const uint16_t*>(p);
    uint32_t x;
    __builtin_memcpy(&x, p, sizeof x);
    return static_cast<int>(x >> shift);
}

// One row of tiles in vector registers.  Accumulators stay in the accumulation
// registers until here: without this the compiler wants all of them where
// the conversions below can read them, and has no room.
template <int N> __device__ __forceinline__ void take_row(const v16f (&acc)[N], v16f (&t)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        t[j] = acc[j];
        asm volatile("" : "+v"(t[j]));
    }
}

// A wave's outputs to rows m on and columns n on of c ([rows][cols], row
// stride ld): each lane N neighbouring columns at once, at any alignment.
// WHOLE: all of them lie in c, and c is not added to.  Otherwise a lane that
// c's last column cuts through stores its columns one by one.  (The checks
// cost 2 us of a 4,096 x 4,096 x 1,024 product's 22 with short sums.)
template <typename T, int W, int N, bool WHOLE>
__device__ __forceinline__ void write_tiles(const v16f (&acc)[N][N], T* c, int64_t ld, int64_t rows, int64_t cols,
                                              int64_t m, int64_t n, bool add, int lane)
{
    const int rows_left = static_cast<int>(rows - m < W ? rows - m : W) - 4 * N * (lane >> 5);
    const int cols_left = static_cast<int>(cols - n < W ? cols - n : W) - N * (lane & 31);
    T* base = c + (m + 4 * N * (lane >> 5)) * ld + n + N * (lane & 31);
    const bool cut = __ballot(cols_left > 0 && cols_left < N) != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v16f t[N];
        take_row<N>(acc[i], t);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = (8 * (r >> 2) + (r & 3)) * N + i;
            T* out = base + row * ld;
            if (WHOLE || (row < rows_left && cols_left >= N)) {
                Pack<T, N> x;
                if (!WHOLE && add) x = load_pack<T, N>(out);
#pragma unroll
                for (int j = 0; j < N; ++j) x.v[j] = from_float<T>(!WHOLE && add ? to_float(x.v[j]) + t[j][r] : t[j][r]);
                store_pack(out, x);
            }
            if (!WHOLE && cut && row < rows_left) {
#pragma unroll
                for (int j = 0; j + 1 < N; ++j)
                    if (j < cols_left && cols_left < N) out[j] = from_float<T>(add ? to_float(out[j]) + t[j][r] : t[j][r]);
            }
        }
    }
}

template <typename T, int W, int N>
__device__ __forceinline__ void write_outputs(const v16f (&acc)[N][N], T* c, int64_t ld, int64_t rows, int64_t cols,
                                              int64_t m, int64_t n, bool add, int lane)
{
    if (!add && m + W <= rows && n + W <= cols) write_tiles<T, W, N, true>(acc, c, ld, rows, cols, m, n, add, lane);
    else write_tiles<T, W, N, false>(acc, c, ld, rows, cols, m, n, add, lane);
}

#endif

struct Grid {
    int32_t tiles_m, tiles_n, splits, steps;    // steps: stages per split
};

template <int W, int WM, int FA, int FB, bool WIDE>
__global__ __launch_bounds__(kThreads, W >= 96 ? 1 : 2) void product(Fp8Product p, Grid g)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = Geometry<W, WM>;
    constexpr int N = G::kTiles;
    __shared__ __attribute__((aligned(16))) uint8_t a0[G::kStageA], b0[G::kStageB], a1[G::kStageA], b1[G::kStageB];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / G::kWavesN, wave_n = wave % G::kWavesN;

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
    const int64_t m0 = static_cast<int64_t>(id / g.tiles_n) * G::kRowsA, n0 = static_cast<int64_t>(id % g.tiles_n) * G::kRowsB;
    const int64_t blocks = (p.a.k + kBytes - 1) / kBytes;
    const int64_t kb0 = static_cast<int64_t>(split) * g.steps;
    const int steps = static_cast<int>(blocks - kb0 < g.steps ? blocks - kb0 : g.steps);

    // A row past the operand's end is read as its last row: its outputs are
    // not stored.
    uint32_t off_a[G::kLoadsA], off_b[G::kLoadsB];
    const int last_a = static_cast<int>(p.a.rows - m0 < G::kRowsA ? p.a.rows - m0 : G::kRowsA) - 1;
    const int last_b = static_cast<int>(p.b.rows - n0 < G::kRowsB ? p.b.rows - n0 : G::kRowsB) - 1;
    auto offset = [&](int q, int last, int64_t ld) {
        const int place = (q * 4 + wave) * 8 + (lane >> 3), r = place % 32;
        const int row = place / W * W + r * N + place % W / 32;
        return static_cast<uint32_t>(row < last ? row : last) * static_cast<uint32_t>(ld) + slot(lane & 7, r) * 16u;
    };
#pragma unroll
    for (int q = 0; q < G::kLoadsA; ++q) off_a[q] = offset(q, last_a, p.a.ld);
#pragma unroll
    for (int q = 0; q < G::kLoadsB; ++q) off_b[q] = offset(q, last_b, p.b.ld);
    const auto ga = buffer(p.a.data + m0 * p.a.ld + kb0 * kBytes,
                                             (p.a.rows - m0) * p.a.ld - kb0 * kBytes);
    const auto gb = buffer(p.b.data + n0 * p.b.ld + kb0 * kBytes,
                                             (p.b.rows - n0) * p.b.ld - kb0 * kBytes);
    const int row_a = wave_m * W + (lane & 31) * N, row_b = wave_n * W + (lane & 31) * N;
    constexpr int kSpan = N == 3 ? 4 : N;   // bytes that a lane's scales are read from
    auto scale_place = [&](int64_t row, int64_t lds, int& shift) {
        const int64_t at = row < lds - kSpan ? row : lds - kSpan;
        shift = row - at < 3 ? static_cast<int>(row - at) * 8 : 24;
        return at;
    };
    int shift_a, shift_b;
    const int64_t sra = scale_place(m0 + row_a, p.a.lds, shift_a), srb = scale_place(n0 + row_b, p.b.lds, shift_b);
    const uint8_t* sa = p.a.scales + kb0 * p.a.lds + sra;
    const uint8_t* sb = p.b.scales + kb0 * p.b.lds + srb;

    Places places;
    places.row_a = (wave_m * W + (lane & 31)) * kBytes;
    places.row_b = (wave_n * W + (lane & 31)) * kBytes;
#pragma unroll
    for (int c = 0; c < 4; ++c) places.chunk[c] = slot(c * 2 + (lane >> 5), lane & 31) * 16;

    v16f acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // A stage goes from global memory straight to LDS.  Stages go in pairs, and every step loads the stage after next, so that
    // the loop has one body and one exit.  A stage past the last is the last
    // one again, with scales of 2^-127 each way: products of 0 in fp32.
    auto load = [&](int k, uint8_t* a, uint8_t* b) {
        const int at = (k < steps ? k : steps - 1) * kBytes;
#pragma unroll
        for (int q = 0; q < G::kLoadsA; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ga, (lds_ptr)(a + (q * 4 + wave) * 1024), 16, off_a[q], at, 0, 0);
#pragma unroll
        for (int q = 0; q < G::kLoadsB; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(gb, (lds_ptr)(b + (q * 4 + wave) * 1024), 16, off_b[q], at, 0, 0);
    };
    Fragments<WIDE, N> frag[2];
    Wide<N> wide[2];
    constexpr int kReads = 2 * N * Sub<WIDE>::kChunks, kMfma = WIDE ? 2 * N * N : N * N;
    auto read = [&](Fragments<WIDE, N>& f, const uint8_t* a, const uint8_t* b, int s) {
#pragma unroll
        for (int q = 0; q < kReads; ++q) read_one<WIDE, N>(f, a, b, places, s, q);
    };
    // multiplies f; next: the fragments multiplied after it (with scales na, nb)
    auto multiply = [&](const Fragments<WIDE, N>& f, int xa, int xb, const Fragments<WIDE, N>& next, int na, int nb) {
        if constexpr (WIDE) {
            widen_half<FA, FB, N>(wide[1], f, 1, xa, xb);
            multiply_wide<N>(acc, wide[0]);
            widen_half<FA, FB, N>(wide[0], next, 0, na, nb);
            multiply_wide<N>(acc, wide[1]);
        } else {
            multiply_scaled<FA, FB, 0, 0, N>(acc, f, xa, xb);
        }
    };
    int xa[2], xb[2];
    auto scales = [&](int k, int s) {
        const int64_t at = k < steps ? k : steps - 1;
        const int in = k < steps ? -1 : 0;
        xa[s] = load_scales<N>(sa + at * p.a.lds, shift_a) & in;
        xb[s] = load_scales<N>(sb + at * p.b.lds, shift_b) & in;
    };
    // Stage k lies in (a, b), stage k + 1 in (an, bn) or on its way there, and
    // frag[0] holds stage k's first sub-step.
    auto step = [&](int k, int s, uint8_t* a, uint8_t* b, uint8_t* an, uint8_t* bn) {
#pragma unroll
        for (int u = 0; u + 1 < Sub<WIDE>::kCount; ++u) {
            read(frag[(u + 1) & 1], a, b, u + 1);
            multiply(frag[u & 1], xa[s], xb[s], frag[(u + 1) & 1], xa[s], xb[s]);
            interleave<kMfma, kReads, 0, WIDE ? kMfma * 2 : 0>();
            __builtin_amdgcn_sched_barrier(0);
        }
        // Stage k + 1 has arrived and every wave holds the rest of stage k in
        // registers: its LDS is free for stage k + 2.
        __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read(frag[0], an, bn, 0);
        load(k + 2, a, b);
        multiply(frag[1], xa[s], xb[s], frag[0], xa[s ^ 1], xb[s ^ 1]);
        interleave<kMfma, kReads, G::kLoadsA + G::kLoadsB, WIDE ? kMfma * 2 : 0>();
        __builtin_amdgcn_sched_barrier(0);
        scales(k + 2, s);
    };
    load(0, a0, b0);
    scales(0, 0);
    load(1, a1, b1);
    scales(1, 1);
    // every wave's part of the first stage has arrived
    __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0)
    __syncthreads();
    read(frag[0], a0, b0, 0);
    if constexpr (WIDE) widen_half<FA, FB, N>(wide[0], frag[0], 0, xa[0], xb[0]);
    int k = 0;
    do {
        step(k, 0, a0, b0, a1, b1);
        step(k + 1, 1, a1, b1, a0, b0);
        k += 2;
    } while (k < steps);

    // the last loads land in LDS before this block gives it up
    __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
    const int64_t m = m0 + wave_m * W, n = n0 + wave_n * W, rows = p.a.rows, cols = p.b.rows;
    const bool add = p.accumulate != 0;
    if (g.splits > 1)
        write_outputs<float, W, N>(acc, p.partial + split * rows * cols, cols, rows, cols, m, n, false, lane);
    else if (WIDE && p.c_dtype == DTYPE_F32)    // short sums are of 16-bit outputs
        write_outputs<float, W, N>(acc, static_cast<float*>(p.c), p.ldc, rows, cols, m, n, add, lane);
    else if (p.c_dtype == DTYPE_BF16)
        write_outputs<bf16, W, N>(acc, static_cast<bf16*>(p.c), p.ldc, rows, cols, m, n, add, lane);
    else
        write_outputs<f16, W, N>(acc, static_cast<f16*>(p.c), p.ldc, rows, cols, m, n, add, lane);
#endif
}

// The splits' partial products joined in order (splits = 0: an empty
// contraction), 4 outputs a thread.
template <typename T> __global__ __launch_bounds__(256) void join(Fp8Product p, int splits)
{
    const int64_t n = p.b.rows, total = p.a.rows * n;
    for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < total;
         i += static_cast<int64_t>(gridDim.x) * 1024) {
        const int count = total - i < 4 ? static_cast<int>(total - i) : 4;
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (count == 4) {
#pragma unroll 4
            for (int k = 0; k < splits; ++k) {
                const Pack<float, 4> x = load_pack<float, 4>(p.partial + k * total + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += x.v[e];
            }
        } else {
            for (int k = 0; k < splits; ++k)
                for (int e = 0; e < count; ++e) s[e] += p.partial[k * total + i + e];
        }
        int64_t row = i / n, col = i - row * n;
        for (int e = 0; e < count; ++e) {
            T* c = static_cast<T*>(p.c) + row * p.ldc + col;
            *c = from_float<T>(p.accumulate ? to_float(*c) + s[e] : s[e]);
            if (++col == n) {
                col = 0;
                ++row;
            }
        }
    }
}

enum Shape { k256, k192, k128, k64Rows, k64Cols };  // block tiles 256 x 256, 192 x 192, 128 x 128, 64 x 256, 256 x 64
struct Plan {
    Shape shape;
    Grid g;
};

// Microseconds of a square tile's blocks: of a stage with as many blocks on a
// CU as fit (of 128 x 128 two, of the others one), of a stage of a 128 x 128
// tile alone on its CU, and of what a tile costs besides its stages.  The
// choice goes by their ratios: 8,192 x 8,192 x 4,096 takes a sixth less than
// they say with all three.  The larger tile has the higher rate (there 205, 322
// and 247 us with 256, 192 and 128, short sums; 390, 524 and 440 with full
// ones), the smaller ones waste less of a product's edges and of the last round
// (4,099 x 2,002 x 5,003: 65, 55 and 70, full 116, 88 and 110; 2,500 x 2,500 x
// 2,500: 38, 33 and 23, full 51, 49 and 36).
struct Rate {
    Shape shape;
    int side;
    double stage, alone, besides;
};
constexpr Rate kRates[2][3] = {
    {{k256, 256, 1.65, 1.65, 8.0}, {k192, 192, 1.30, 1.30, 6.0}, {k128, 128, 1.00, 0.68, 4.0}},
    {{k256, 256, 3.20, 3.20, 8.0}, {k192, 192, 2.10, 2.10, 6.0}, {k128, 128, 1.80, 1.15, 4.0}}};  // full sums

int64_t count(int64_t x, int64_t side) { return (x + side - 1) / side; }

double time_of(const Rate& r, int64_t tiles, int64_t stages)
{
    const int64_t slots = r.side == 128 ? 512 : 256, full = tiles / slots, rest = tiles % slots;
    const double last = rest == 0 ? 0.0 : (rest <= 256 ? r.alone : r.stage) * static_cast<double>(stages) + r.besides;
    return static_cast<double>(full) * (r.stage * static_cast<double>(stages) + r.besides) + last;
}

// The square tile that takes the least time, or tiles of 64 rows where one
// side has no more.  Where tiles leave half of the chip or more idle, the
// contraction is split, at least 4 stages each.
Plan plan_of(int64_t m, int64_t n, int64_t k, bool wide)
{
    const int64_t blocks = count(k, kBytes);
    const auto splits_of = [&](int64_t tiles) {
        int64_t s = 256 / tiles;
        if (s > blocks / 4) s = blocks / 4;
        if (s > kMaxSplits) s = kMaxSplits;
        return s < 1 ? 1 : s;
    };
    Plan p;
    int64_t side_m = 64, side_n = 256;
    if (m <= kFewRows) {
        p.shape = k64Rows;
    } else if (n <= kFewRows) {
        p.shape = k64Cols;
        side_m = 256;
        side_n = 64;
    } else {
        double best = 0.0;
        for (const Rate& r : kRates[wide]) {
            const int64_t tiles = count(m, r.side) * count(n, r.side), s = splits_of(tiles);
            double t = time_of(r, tiles * s, count(blocks, s));
            // the parts are written and read again, at about 4 TB/s, by one launch more
            if (s > 1) t += 3.0 + 8.0 * static_cast<double>(s) * static_cast<double>(m) * static_cast<double>(n) / 4e6;
            if (best == 0.0 || t < best) {
                best = t;
                p.shape = r.shape;
                side_m = side_n = r.side;
            }
        }
    }
    const int64_t splits = splits_of(count(m, side_m) * count(n, side_n));
    p.g.tiles_m = static_cast<int32_t>(count(m, side_m));
    p.g.tiles_n = static_cast<int32_t>(count(n, side_n));
    p.g.steps = static_cast<int32_t>(count(blocks, splits));
    if (splits > 1) p.g.steps += p.g.steps & 1;     // the kernel takes stages in pairs
    p.g.splits = static_cast<int32_t>(count(blocks, p.g.steps));
    return p;
}

template <int FA, int FB, bool WIDE> hipError_t launch_arithmetic(const Fp8Product& p, const Plan& plan, hipStream_t s)
{
    const unsigned blocks = static_cast<unsigned>(plan.g.tiles_m) * plan.g.tiles_n * plan.g.splits;
    switch (plan.shape) {
    case k256: product<128, 2, FA, FB, WIDE><<<blocks, kThreads, 0, s>>>(p, plan.g); break;
    case k192: product<96, 2, FA, FB, WIDE><<<blocks, kThreads, 0, s>>>(p, plan.g); break;
    case k128: product<64, 2, FA, FB, WIDE><<<blocks, kThreads, 0, s>>>(p, plan.g); break;
    case k64Rows: product<64, 1, FA, FB, WIDE><<<blocks, kThreads, 0, s>>>(p, plan.g); break;
    case k64Cols: product<64, 4, FA, FB, WIDE><<<blocks, kThreads, 0, s>>>(p, plan.g); break;
    }
    return hipGetLastError();
}

template <int FA, int FB> hipError_t launch_formats(const Fp8Product& p, const Plan& plan, hipStream_t s)
{
    return p.short_sums ? launch_arithmetic<FA, FB, false>(p, plan, s) : launch_arithmetic<FA, FB, true>(p, plan, s);
}

}  // namespace

hipError_t launch_fp8_join(const Fp8Product& p, int splits, hipStream_t s)
{
    const int64_t quads = (p.a.rows * p.b.rows + 3) / 4;
    const unsigned blocks = static_cast<unsigned>((quads + 255) / 256 < kLaunchBlocks ? (quads + 255) / 256 : kLaunchBlocks);
    if (p.c_dtype == DTYPE_F32) join<float><<<blocks, 256, 0, s>>>(p, splits);
    else if (p.c_dtype == DTYPE_BF16) join<bf16><<<blocks, 256, 0, s>>>(p, splits);
    else join<f16><<<blocks, 256, 0, s>>>(p, splits);
    return hipGetLastError();
}

size_t fp8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m < 1 || n < 1 || k < 1) return 0;
    int splits = 1;
    if (fp8_few(m, n, k)) {
        splits = fp8_few_splits(m, n, k);
    } else {
        for (const bool wide : {false, true}) {
            const int planned = plan_of(m, n, k, wide).g.splits;
            if (planned > splits) splits = planned;
        }
    }
    return splits > 1 ? sizeof(float) * static_cast<size_t>(splits) * static_cast<size_t>(m) * static_cast<size_t>(n) : 0;
}

hipError_t launch_fp8_product(const Fp8Product& p, hipStream_t s)
{
    if (p.a.k == 0) return launch_fp8_join(p, 0, s);
    if (fp8_few(p.a.rows, p.b.rows, p.a.k)) return launch_fp8_few(p, s);
    const Plan plan = plan_of(p.a.rows, p.b.rows, p.a.k, !p.short_sums);
    hipError_t e;
    if (p.a.format == FP8_E4M3)
        e = p.b.format == FP8_E4M3 ? launch_formats<0, 0>(p, plan, s) : launch_formats<0, 1>(p, plan, s);
    else
        e = p.b.format == FP8_E4M3 ? launch_formats<1, 0>(p, plan, s) : launch_formats<1, 1>(p, plan, s);
    if (e == hipSuccess && plan.g.splits > 1) e = launch_fp8_join(p, plan.g.splits, s);
    return e;
}

}  // namespace fasgd
