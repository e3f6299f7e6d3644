// Tiles of the matrix products that go through LDS: what a wave owns, how a
// stage lies in LDS, the order of a sub-step's instructions and the way
// outputs are stored.
#pragma once

#include "fp8_math.hpp"

namespace fasgd {
namespace {

constexpr int kThreads = 256;       // 4 waves
constexpr int kBytes = 128;         // of each operand's row per stage

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

// The tile of a block among tiles_m x tiles_n, as row tiles_n + column.
// Consecutive blocks go to the 8 XCDs in turn: give each XCD a run of tiles, 8
// rows of tiles deep, so that its L2 serves their operands.
__device__ __forceinline__ int tile_of(int id, int tiles_m, int tiles_n)
{
    const int tiles = tiles_m * tiles_n, xcd = id & 7, each = tiles >> 3, extra = tiles & 7;
    id = xcd * each + (xcd < extra ? xcd : extra) + (id >> 3);
    const int deep = 8 * tiles_n, group = id / deep, first = group * 8;
    const int rows = tiles_m - first < 8 ? tiles_m - first : 8;
    const int in = id - group * deep;
    return (first + in % rows) * tiles_n + in / rows;
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

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// 16 x 16 sums of 32 products of bf16's or fp16's: lane l holds 8 values of row
// l % 16 of each operand (chunk l / 16 of the row's 64 bytes), and of the sums
// column l % 16 and rows 4 (l / 16) to 4 (l / 16) + 3.  At the chip's power limit
// it does an eighth more than 32 x 32 x 16 (random values in registers 2,070
// against 1,810 TFLOP/s).
template <typename T> __device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& c);
template <> __device__ __forceinline__ v4f mfma<bf16>(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ v4f mfma<f16>(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// A tile in vector registers.  Accumulators stay in the accumulation
// registers until here: without this the compiler wants all of them where
// the conversions after it can read them, and has no room.
__device__ __forceinline__ v16f take(const v16f& acc)
{
    v16f t = acc;
    asm volatile("" : "+v"(t));
    return t;
}
__device__ __forceinline__ v4f take(const v4f& acc)
{
    v4f t = acc;
    asm volatile("" : "+v"(t));
    return t;
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
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = take(acc[i][j]);
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

}  // namespace
}  // namespace fasgd
