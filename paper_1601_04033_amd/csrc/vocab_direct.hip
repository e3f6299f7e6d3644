// The losses over a large vocabulary for few rows and for small problems: x, W
// and the gradients as they lie, without gathering, laying out or 16-bit terms.
//
// A few rows against a large vocabulary are bound by reading W (twice forward
// and backward, and once more for dx) and writing dW; a small problem by its
// chain of launches.  So there are one or two forward and two to five backward,
// the matrix instruction
// takes operands from global memory straight into registers (16 x 16 tiles:
// 16-bit types as they are, fp32 by the fp32 instruction), and the gradient of
// the logits is held in fp32.
//
// Measured (bf16, 4,096 columns, 131,072 classes): logits of 1 row 190 us, 5.6 TB/s
// of W; of 16 rows 223 to 238, 4.6; dx of 16 rows 236, 4.5; dW 399, 5.4 TB/s of
// stores.  More rows than 16 read W again for each 16, from L2 or the last-level
// cache: 1,024 x 1,024 x 1,024 fp32 45 us forward, 48 TFLOP/s.
#include <float.h>

#include "fp8_math.hpp"
#include "vocab_rows.hpp"

namespace fasgd {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ---- logits: 16 rows by 16 classes at a time

// A block's 8 waves each take a part of the contraction and keep the rows' part
// of x in registers; W goes by, 16 classes a group.  The parts' sums meet in LDS,
// where a wave each joins a group's, in order.
constexpr int kLogitThreads = 512, kLogitWaves = 8;

struct Direct {
    int64_t groups_each;    // groups of 16 classes a block
    int64_t padded;         // rows to a multiple of 16
    float2* partial;        // [gridDim.x][padded]
    float* partial_sum;
    float *dz, *dzt;        // fp32 [rows][vocab], [vocab][padded]
    int32_t* used;          // [padded]
};

// 16 bytes of a lane: what it holds of an operand's row per step of 64 bytes a row.
template <typename T> struct Chunk {
    static constexpr int kValues = 16 / sizeof(T);      // per lane
    static constexpr int kStep = 4 * kValues;           // per row
};

#if defined(__HIP_DEVICE_COMPILE__)

__device__ __forceinline__ v4f tile(const bf16*, const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f tile(const f16*, const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}
__device__ __forceinline__ v4f tile(const float*, const v4i& a, const v4i& b, v4f c)
{
    const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
    return c;
}

// 16 bytes from value k on of a row of `cols`; zeros past its end.
template <typename T> __device__ __forceinline__ v4i load_chunk(const T* row, int k, int cols)
{
    Pack<T, Chunk<T>::kValues> p;
    if (k + Chunk<T>::kValues <= cols) {
        p = load_pack<T, Chunk<T>::kValues>(row + k);
    } else {
#pragma unroll
        for (int e = 0; e < Chunk<T>::kValues; ++e) p.v[e] = k + e < cols ? row[k + e] : from_float<T>(0.0f);
    }
    return __builtin_bit_cast(v4i, p);
}

#endif

// NK: steps of a wave at most; 0: any number, with x read beside W, from L2, since
// the registers do not hold it.  GRADIENT: dz of the rows, else their statistics
// and the picked logits.
template <typename T, int NK, bool GRADIENT>
__global__ __launch_bounds__(kLogitThreads) void logits(VocabArgs a, Direct d)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kBatch = 8;       // groups between two meetings of the waves
    constexpr bool kWide = NK == 0;
    constexpr int kHold = kWide ? 1 : NK;
    constexpr int kLoads = kWide || NK > 8 ? 8 : NK, kParts = kHold / kLoads;       // of a group: loads in flight, times
    constexpr int kSequence = kParts == 1 ? 2 : kParts;                 // loads with a buffer each of two
    __shared__ v4f part[kLogitWaves][kBatch][64];
    __shared__ float table[16][kBatch * 16 + 4];
    __shared__ float2 stat[kLogitWaves][16];
    __shared__ float stat_sum[kLogitWaves][16];
    __shared__ VocabRow coefficient[16];
    __shared__ Teacher teachers[16];
    __shared__ int used[16];
    constexpr int kHeld = 2048;
    __shared__ int32_t cls[kHeld];
    __shared__ float weights[GRADIENT ? kHeld : 1], total[GRADIENT ? kHeld : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * 16;
    const int cols = static_cast<int>(a.cols);
    const int rows = a.rows - r0 < 16 ? static_cast<int>(a.rows - r0) : 16;

    const int steps = (cols + Chunk<T>::kStep - 1) / Chunk<T>::kStep, each = (steps + kLogitWaves - 1) / kLogitWaves;
    const int first = wave * each;
    const int own = steps - first < each ? (steps - first < 0 ? 0 : steps - first) : each;     // <= NK
    const int k0 = first * Chunk<T>::kStep + (lane >> 4) * Chunk<T>::kValues;
    // the steps whose 64 bytes all lie within the rows
    const int whole = cols / Chunk<T>::kStep - first;

    v4i x[kHold];
    const T* x_row = static_cast<const T*>(a.x) + (r0 + ((lane & 15) < rows ? lane & 15 : 0)) * a.ldx;
    if constexpr (!kWide) {
        const T* row = x_row;
#pragma unroll
        for (int s = 0; s < NK; ++s) {
            if (s < whole && s < own) x[s] = __builtin_bit_cast(v4i, load_pack<T, Chunk<T>::kValues>(row + k0 + s * Chunk<T>::kStep));
            else if (s < own) x[s] = load_chunk<T>(row, k0 + s * Chunk<T>::kStep, cols);
            else x[s] = v4i{0, 0, 0, 0};
        }
    }

    // The entries: their classes (-1: left out) and, backward, their weights, in
    // LDS where they fit; which rows take part, and their coefficients, two rows
    // a wave.
    const int entries = rows * a.entries;
    const bool held = entries <= kHeld;
    if (held)
        for (int at = threadIdx.x; at < entries; at += kLogitThreads) {
            const int64_t here = r0 * a.entries + at;
            cls[at] = counts(a, here) ? static_cast<int32_t>(a.index[here]) : -1;
        }
    for (int i = wave * 2; i < wave * 2 + 2; ++i) {
        const int64_t r = r0 + i;
        bool any = false;
        if (i < rows)
            for (int k = lane; k < a.entries; k += 64) any |= counts(a, r * a.entries + k);
        any = __ballot(any) != 0;
        VocabRow c = {0.0f, 0.0f, 0.0f, 0.0f};
        Teacher t = {0.0f, 0.0f};
        if (GRADIENT && any) {
            t = teacher_of(a, r, lane);
            c = coefficients_of(a, r, t, lane);
        }
        if (GRADIENT && held && i < rows)
            for (int k = lane; k < a.entries; k += 64) weights[i * a.entries + k] = any ? weight(a, t, r * a.entries + k) : 0.0f;
        if (lane == 0) {
            used[i] = any;
            coefficient[i] = c;
            teachers[i] = t;
            if (GRADIENT && blockIdx.x == 0) d.used[r] = any;
        }
    }
    __syncthreads();
    const bool live = used[lane & 15] != 0;
    if (!kWide && !live) {      // what a row that is left out holds reaches nothing
#pragma unroll
        for (int s = 0; s < NK; ++s) x[s] = v4i{0, 0, 0, 0};
    }
    if (GRADIENT && held && a.entries > 1) {    // weights of one class of a row add up at its first entry
        for (int at = threadIdx.x; at < entries; at += kLogitThreads) {
            const int base = at / a.entries * a.entries, mine = cls[at];
            float q = 0.0f;
            bool later = false;
            for (int j = base; j < base + a.entries; ++j) {
                const bool same = cls[j] == mine;
                q += same ? weights[j] : 0.0f;
                later |= same && j < at;
            }
            total[at] = later ? -1.0f : q;
        }
        __syncthreads();
        for (int at = threadIdx.x; at < entries; at += kLogitThreads) {
            weights[at] = total[at];
            if (total[at] < 0.0f) cls[at] = -1;
        }
        __syncthreads();
    }
    const int64_t groups = (a.vocab + 15) / 16, g0 = static_cast<int64_t>(blockIdx.x) * d.groups_each;
    const int64_t g1 = g0 + d.groups_each < groups ? g0 + d.groups_each : groups;

    v4i w[2][kLoads], beside[2][kWide ? kLoads : 1];
    auto load_x = [&](int buffer, int at) {
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            const int step = at * kLoads + s;
            v4i v = {0, 0, 0, 0};
            if (step < whole && step < own) v = __builtin_bit_cast(v4i, load_pack<T, Chunk<T>::kValues>(x_row + k0 + step * Chunk<T>::kStep));
            else if (step < own) v = load_chunk<T>(x_row, k0 + step * Chunk<T>::kStep, cols);
            beside[buffer][s] = live ? v : v4i{0, 0, 0, 0};
        }
    };
    auto load = [&](int buffer, int64_t group, int at) {
        const int64_t c = group * 16 + (lane & 15);
        const T* row = static_cast<const T*>(a.w) + (c < a.vocab ? c : a.vocab - 1) * a.ldw;
#pragma unroll
        for (int s = 0; s < kLoads; ++s) {
            const int step = at * kLoads + s;
            if (step < whole && step < own) w[buffer][s] = __builtin_bit_cast(v4i, load_pack<T, Chunk<T>::kValues>(row + k0 + step * Chunk<T>::kStep));
            else if (step < own) w[buffer][s] = load_chunk<T>(row, k0 + step * Chunk<T>::kStep, cols);
            else w[buffer][s] = v4i{0, 0, 0, 0};
        }
    };
    const float c = a.scale * kLog2e;
    float top = -FLT_MAX, sum = 0.0f, all = 0.0f;      // of this lane's row and the classes it sees
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!kWide && g0 < g1) load(0, g0, 0);
    for (int64_t b0 = g0; b0 < g1; b0 += kBatch) {
        const int batch = static_cast<int>(g1 - b0 < kBatch ? g1 - b0 : kBatch);
        if constexpr (kWide) {
            const int parts = (each + kLoads - 1) / kLoads, times = batch * parts;
            load(0, b0, 0);
            load_x(0, 0);
            int here = 0, at = 0;
            for (int q = 0; q < times; q += 2) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (q + s >= times) break;
                    const bool last = at + 1 == parts;
                    if (q + s + 1 < times) {
                        load(s ^ 1, b0 + here + (last ? 1 : 0), last ? 0 : at + 1);
                        load_x(s ^ 1, last ? 0 : at + 1);
                    }
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) acc = tile(static_cast<const T*>(nullptr), w[s][i], beside[s][i], acc);
                    if (last) {
                        part[wave][here][lane] = acc;
                        acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                    }
                    here += last;
                    at = last ? 0 : at + 1;
                }
            }
        }
        for (int g = 0; !kWide && g < batch; g += kParts == 1 ? 2 : 1) {
#pragma unroll
            for (int s = 0; s < kSequence; ++s) {
                const int here = kParts == 1 ? g + s : g, at = kParts == 1 ? 0 : s;
                // the next loads: of this group's rest, or of the next group
                const bool last = kParts == 1 || s + 1 == kParts;
                const int64_t next = b0 + here + (last ? 1 : 0);
                if (next < g1) load((s + 1) & 1, next, last ? 0 : s + 1);
                if (here < batch) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) acc = tile(static_cast<const T*>(nullptr), w[s & 1][i], x[kWide ? 0 : at * kLoads + i], acc);
                    if (last) {
                        part[wave][here][lane] = acc;
                        acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                    }
                }
            }
        }
        __syncthreads();
        if (wave < batch) {     // a group each: lane l has row l % 16 and classes 4 (l / 16) on
            v4f z = part[0][wave][lane];
#pragma unroll
            for (int i = 1; i < kLogitWaves; ++i) z += part[i][wave][lane];
            const int64_t first_class = (b0 + wave) * 16 + 4 * (lane >> 4);
            const int left = a.vocab - first_class < 4 ? static_cast<int>(a.vocab - first_class) : 4;
            if (GRADIENT) {
                const VocabRow row = coefficient[lane & 15];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    table[lane & 15][wave * 16 + 4 * (lane >> 4) + e] =
                        used[lane & 15] ? __builtin_fmaf(row.f, power(__builtin_fmaf(z[e], c, -row.l)), -row.b) : 0.0f;
            } else {
                float most = -FLT_MAX;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    table[lane & 15][wave * 16 + 4 * (lane >> 4) + e] = z[e];
                    all += e < left ? z[e] : 0.0f;
                    most = e < left ? fmaxf(most, z[e] * c) : most;
                }
                const float next = fmaxf(top, most);
                sum *= power(top - next);
                top = next;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += e < left ? power(__builtin_fmaf(z[e], c, -top)) : 0.0f;
            }
        }
        __syncthreads();
        // The entries among the batch's classes.
        for (int at = threadIdx.x; at < entries; at += kLogitThreads) {
            if (held && cls[at] < 0) continue;
            const int64_t here = r0 * a.entries + at, c0 = (held ? cls[at] : a.index[here]) - b0 * 16;
            if (c0 < 0 || c0 >= batch * 16 || (!held && !counts(a, here))) continue;
            const int i = at / a.entries;
            if (!GRADIENT) {
                a.picked[here] = table[i][c0] * a.scale;
            } else if (held) {
                table[i][c0] = entry_value(coefficient[i], a.picked[here], weights[at]);
            } else {
                float z;
                if (entry_gradient(a, coefficient[i], teachers[i], r0 + i, at - i * a.entries, &z)) table[i][c0] = z;
            }
        }
        if (GRADIENT) {
            __syncthreads();
            const int64_t c0 = b0 * 16;
            const int n = a.vocab - c0 < batch * 16 ? static_cast<int>(a.vocab - c0) : batch * 16;
            if (d.dz)
                for (int at = threadIdx.x; at < rows * kBatch * 16; at += kLogitThreads) {
                    const int i = at / (kBatch * 16), k = at % (kBatch * 16);
                    if (k < n) d.dz[(r0 + i) * a.vocab + c0 + k] = table[i][k];
                }
            if (d.dzt)
                for (int at = threadIdx.x; at < n * 16; at += kLogitThreads) d.dzt[(c0 + at / 16) * d.padded + r0 + at % 16] = table[at % 16][at / 16];
        }
        __syncthreads();
    }
    if (GRADIENT) return;
    // statistics: the lanes of a row, then the waves, in order
    const float most = larger_of(top, 16), m2 = larger_of(most, 32);
    sum *= power(top - m2);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    all += __shfl_xor(all, 16);
    all += __shfl_xor(all, 32);
    if (lane < 16) {
        stat[wave][lane] = make_float2(m2, sum);
        stat_sum[wave][lane] = all;
    }
    __syncthreads();
    if (threadIdx.x < 16) {
        float m = -FLT_MAX, s = 0.0f, t = 0.0f;
        for (int i = 0; i < kLogitWaves; ++i) m = fmaxf(m, stat[i][threadIdx.x].x);
        for (int i = 0; i < kLogitWaves; ++i) {
            s += stat[i][threadIdx.x].y * power(stat[i][threadIdx.x].x - m);
            t += stat_sum[i][threadIdx.x];
        }
        if (gridDim.x == 1) {   // all classes were here
            stat[0][threadIdx.x] = make_float2(__builtin_fmaf(m, kLn2, logf(s)), t * a.scale / static_cast<float>(a.vocab));
        } else {
            d.partial[blockIdx.x * d.padded + r0 + threadIdx.x] = make_float2(m, s);
            if (d.partial_sum) d.partial_sum[blockIdx.x * d.padded + r0 + threadIdx.x] = t;
        }
    }
    if (gridDim.x > 1) return;
    __syncthreads();
    for (int i = wave; i < rows; i += kLogitWaves) finish_row(a, r0 + i, stat[0][i].x, stat[0][i].y, false, lane);
#endif
}

// ---- dx and dW: c[r][n] = sum_k a[k][r] b[k][n], both along k

// A wave owns 16 rows and 128 columns: lane l holds 8 columns of b at row l / 16
// of each 4 of k, and so the same columns of 4 rows of c.
struct Thin {
    const float* a;         // [k][lda]
    int64_t lda, ldb, rows, cols, k, k_each;        // k_each: of a split, a multiple of 4
    const void* b;
    const int32_t* used_k;  // b's rows that take part (NULL: all)
    void* c;                // one split: the output; else fp32 [split][rows padded to 16][cols padded to 128]
    int64_t ldc;
    const int32_t* used_r;  // rows of c that take part, zeros for the others (NULL: all)
    float by;
    int32_t add, splits, row_tiles;     // row_tiles: that a wave goes through (short_product)
    int32_t column_blocks, row_blocks;
    int32_t brief;          // k of at most 16 times this, by short_product; 0: by long_product
    int64_t blocks;         // in all; 0: not wanted
};

#if defined(__HIP_DEVICE_COMPILE__)
// N values of a row from column n on; zeros past its end.
template <typename T, int N> __device__ __forceinline__ Pack<T, N> load_values(const T* row, int64_t n, int64_t cols)
{
    if (n + N <= cols) return load_pack<T, N>(row + n);
    Pack<T, N> p;
#pragma unroll
    for (int e = 0; e < N; ++e) p.v[e] = n + e < cols ? row[n + e] : from_float<T>(0.0f);
    return p;
}

// N values to row `row` of c, from column n on.
template <typename OUT, int N> __device__ __forceinline__ void store_values(const Thin& p, int64_t row, int64_t n, const float (&v)[N])
{
    if (row >= p.rows) return;
    const bool in = !p.used_r || p.used_r[row];
    OUT* out = static_cast<OUT*>(p.c) + row * p.ldc + n;
    Pack<OUT, N> o;
    if (n + N <= p.cols) {
        if (p.add) o = load_pack<OUT, N>(out);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = in ? v[e] * p.by : 0.0f;
            o.v[e] = from_float<OUT>(p.add ? to_float(o.v[e]) + x : x);
        }
        store_pack(out, o);
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (n + e < p.cols) {
            const float x = in ? v[e] * p.by : 0.0f;
            out[e] = from_float<OUT>(p.add ? to_float(out[e]) + x : x);
        }
}
#endif

#if defined(__HIP_DEVICE_COMPILE__)

// k of at most 16 KB: b's values stay in registers, the row tiles go by.  Bound by
// the stores of c, so a lane's columns are 4 neighbours in each half of the
// wave's 128: 16 lanes store 256 bytes.
template <typename T, typename OUT, int KB> __device__ __forceinline__ void thin_short(const Thin& p, int column_block, int64_t row_block)
{
    const int lane = threadIdx.x & 63;
    const int64_t n0 = (static_cast<int64_t>(column_block) * 4 + (threadIdx.x >> 6)) * 128, n = n0 + 4 * (lane & 15);
    if (n0 >= p.cols) return;
    constexpr int kSteps = 4 * KB;
    float held[kSteps][8];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int64_t k = 4 * s + (lane >> 4);
        const bool in = k < p.k && (!p.used_k || p.used_k[k]);
        Pack<T, 4> v[2];
        if (in) {
            v[0] = load_values<T, 4>(static_cast<const T*>(p.b) + k * p.ldb, n, p.cols);
            v[1] = load_values<T, 4>(static_cast<const T*>(p.b) + k * p.ldb, n + 64, p.cols);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) held[s][e] = in ? to_float(v[e >> 2].v[e & 3]) : 0.0f;
    }
    const int64_t t0 = row_block * p.row_tiles;
    const float* at = p.a + (lane >> 4) * p.lda + (lane & 15);
    auto take_a = [&](int64_t r0, float (&x)[kSteps]) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            x[s] = 4 * s + (lane >> 4) < p.k && r0 + (lane & 15) < p.rows ? at[4 * s * p.lda + r0] : 0.0f;
    };
    float x[kSteps];
    take_a(t0 * 16, x);
    const bool plain = n0 + 128 <= p.cols && !p.used_r && !p.add;     // nothing to look at per store
    OUT* out = static_cast<OUT*>(p.c) + (t0 * 16 + 4 * (lane >> 4)) * p.ldc + n;
    for (int t = 0; t < p.row_tiles; ++t, out += 16 * p.ldc) {
        const int64_t r0 = (t0 + t) * 16;
        if (r0 >= p.rows) return;
        float next[kSteps];
        take_a(r0 + 16, next);
        v4f acc[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[s], held[s][e], acc[e], 0, 0, 0);
        if (plain && r0 + 16 <= p.rows) {
            OUT* at_row = out;
#pragma unroll
            for (int i = 0; i < 4; ++i, at_row += p.ldc)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Pack<OUT, 4> o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o.v[e] = from_float<OUT>(acc[4 * h + e][i] * p.by);
                    store_pack(at_row + 64 * h, o);
                }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[4 * h + e][i];
                    store_values<OUT, 4>(p, r0 + 4 * (lane >> 4) + i, n + 64 * h, v);
                }
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) x[s] = next[s];
    }
}

// Any k: a block's 4 waves take 16 of it in turn and join their sums in order.
// A lane has 8 neighbouring columns.
// MASK: used_k is there.
template <typename T, typename OUT, bool MASK>
__device__ __forceinline__ void thin_long(const Thin& p, v4f (&part)[4][8][64], int column_block, int64_t row_block, int split)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = static_cast<int64_t>(column_block) * 128, n = n0 + 8 * (lane & 15);
    const int64_t r0 = row_block * 16, r = r0 + (lane & 15);
    const int64_t k0 = split * p.k_each, k1 = k0 + p.k_each < p.k ? k0 + p.k_each : p.k;
    constexpr int kFlight = 8;      // loads on their way at once, of 4 of k each
    constexpr int64_t kStep = 4 * kFlight;
    v4f acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const float* a = p.a + (r < p.rows ? r : r0);
    struct Loads {
        float x[kFlight];
        Pack<T, 8> v[kFlight];
        int in[kFlight];
    };
    auto multiply = [&](const Loads& l) {
#pragma unroll
        for (int s = 0; s < kFlight; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(l.x[s], l.in[s] ? to_float(l.v[s].v[e]) : 0.0f, acc[e], 0, 0, 0);
    };
    int64_t kb = k0 + wave * kStep;
    if (n0 + 128 <= p.cols) {       // whole steps, the next on its way while one is multiplied
        const T* b = static_cast<const T*>(p.b) + n;
        auto load = [&](Loads& l) {
            const int64_t k = kb + (lane >> 4);
#pragma unroll
            for (int s = 0; s < kFlight; ++s) {
                l.x[s] = a[(k + 4 * s) * p.lda];
                l.v[s] = load_pack<T, 8>(b + (k + 4 * s) * p.ldb);
                l.in[s] = MASK ? p.used_k[k + 4 * s] : 1;
            }
            kb += 4 * kStep;
        };
        Loads l0, l1;
        if (kb + kStep <= k1) {
            load(l0);
            while (true) {
                if (kb + kStep > k1) {
                    multiply(l0);
                    break;
                }
                load(l1);
                multiply(l0);
                if (kb + kStep > k1) {
                    multiply(l1);
                    break;
                }
                load(l0);
                multiply(l1);
            }
        }
    }
    for (; kb < k1; kb += 4 * kStep) {      // what is cut by the end of k or of the columns
        Loads l;
#pragma unroll
        for (int s = 0; s < kFlight; ++s) {
            const int64_t k = kb + 4 * s + (lane >> 4);
            l.in[s] = k < k1 && (!MASK || p.used_k[k]);
            l.x[s] = 0.0f;
            if (l.in[s]) {
                l.x[s] = a[k * p.lda];
                l.v[s] = load_values<T, 8>(static_cast<const T*>(p.b) + k * p.ldb, n, p.cols);
            }
        }
        multiply(l);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][e][lane] = acc[e];
    __syncthreads();
    // a wave each: rows 4 (lane / 16) + wave
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = part[0][e][lane][wave] + part[1][e][lane][wave] + part[2][e][lane][wave] + part[3][e][lane][wave];
    const int64_t row = r0 + 4 * (lane >> 4) + wave;
    if (p.splits > 1) {
        Pack<float, 8> o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = v[e];
        store_pack(static_cast<float*>(p.c) + (split * ((p.rows + 15) / 16 * 16) + row) * p.ldc + n, o);
    } else {
        store_values<OUT, 8>(p, row, n, v);
    }
}

// A block of a product of long k among all of its blocks.
template <typename T, typename OUT, bool MASK>
__device__ __forceinline__ void long_block(const Thin& p, v4f (&part)[4][8][64], int id)
{
    const int rest = id / p.column_blocks;
    thin_long<T, OUT, MASK>(p, part, id % p.column_blocks, rest % p.row_blocks, rest / p.row_blocks);
}

// Consecutive blocks go to the 8 XCDs in turn: give each XCD a run of them, so
// that its L2 sees whole rows.  (A column block of each row alone lies in a few
// of its channels.)
__device__ __forceinline__ int64_t in_runs(int64_t all)
{
    const int64_t each = all >> 3, extra = all & 7, xcd = blockIdx.x & 7;
    return xcd * each + (xcd < extra ? xcd : extra) + (blockIdx.x >> 3);
}

#endif

// dW of a few rows; dx of a few classes.
template <typename T, typename OUT, int KB> __global__ __launch_bounds__(256, KB < 4 ? 3 : 2) void short_product(Thin p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const int64_t id = in_runs(p.blocks);
    thin_short<T, OUT, KB>(p, static_cast<int>(id % p.column_blocks), id / p.column_blocks);
#endif
}

template <typename T, typename OUT, bool MASK> __global__ __launch_bounds__(256, 2) void long_product(Thin p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ v4f part[4][8][64];
    long_block<T, OUT, MASK>(p, part, static_cast<int>(in_runs(p.blocks)));
#endif
}

// Both of a small problem in one launch, dx's blocks first.
template <typename T, typename OUT> __global__ __launch_bounds__(256, 2) void long_products(Thin dx, Thin dw)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ v4f part[4][8][64];
    const int id = blockIdx.x;
    if (id < dx.blocks) long_block<T, T, false>(dx, part, id);
    else long_block<T, OUT, true>(dw, part, id - static_cast<int>(dx.blocks));
#endif
}

// An output from the splits' parts, in order: 4 columns a thread.  used: rows
// that take part (NULL: all).
template <typename T> __global__ __launch_bounds__(256) void join(Thin p, T* out, int64_t ld, const int32_t* used, int add)
{
    const int64_t r = blockIdx.y, n = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (n >= p.cols) return;
    const float* c = static_cast<const float*>(p.c) + r * p.ldc + n;
    const int64_t apart = (p.rows + 15) / 16 * 16 * p.ldc;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int k = 0; k < p.splits; ++k) {
        const Pack<float, 4> x = load_pack<float, 4>(c + k * apart);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += x.v[e];
    }
    const bool in = !used || used[r] != 0;
    out += r * ld + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < p.cols) out[e] = from_float<T>((in ? s[e] * p.by : 0.0f) + (add ? to_float(out[e]) : 0.0f));
}

int64_t count(int64_t x, int64_t side) { return (x + side - 1) / side; }

// ---- the host's side

struct Layout {
    int64_t padded, cols_padded, groups_each, blocks;
    int splits, dw_splits;
    int64_t k_each, dw_each;
    int64_t used, dz, dzt, sums, dw_sums, partial, partial_sum, bytes;
};

Layout layout_of(int64_t rows, int64_t cols, int64_t vocab, bool backward)
{
    Layout l = {};
    l.padded = count(rows, 16) * 16;
    l.cols_padded = count(cols, 128) * 128;
    // a block a CU
    const int64_t groups = count(vocab, 16), row_tiles = l.padded / 16;
    l.groups_each = count(groups, row_tiles < 256 ? 256 / row_tiles : 1);
    l.blocks = count(groups, l.groups_each);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = (at + bytes + 255) / 256 * 256;
        return here;
    };
    l.used = take(4 * l.padded);
    if (backward) {
        // dx: blocks for 16 rows x 128 columns, the classes split to make about 512 of them
        const int64_t blocks = row_tiles * l.cols_padded / 128;
        int64_t s = 512 / blocks;
        if (s > count(vocab, 256)) s = count(vocab, 256);
        if (s < 1) s = 1;
        l.k_each = count(count(vocab, s), 4) * 4;
        l.splits = static_cast<int>(count(vocab, l.k_each));
        l.dz = take(4 * rows * vocab);
        l.dzt = take(4 * l.padded * vocab);
        l.sums = take(l.splits > 1 ? 4 * l.splits * l.padded * l.cols_padded : 0);
        // dW alike, of few classes: the rows split (6,575 x 350 x 25 fp32: 460 us in one part, 78 so, with the forward pass)
        s = 512 / (groups * l.cols_padded / 128);
        if (s > count(rows, 256)) s = count(rows, 256);
        if (s < 1) s = 1;
        l.dw_each = count(count(rows, s), 4) * 4;
        l.dw_splits = static_cast<int>(count(rows, l.dw_each));
        l.dw_sums = take(l.dw_splits > 1 ? 4 * l.dw_splits * groups * 16 * l.cols_padded : 0);
    } else {
        l.partial = take(8 * l.blocks * l.padded);
        l.partial_sum = take(4 * l.blocks * l.padded);
    }
    l.bytes = at;
    return l;
}

template <typename T, bool GRADIENT> hipError_t launch_logits(const VocabArgs& a, const Direct& d, int64_t blocks, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(d.padded / 16));
    const int64_t each = count(count(a.cols, 64 / static_cast<int64_t>(sizeof(T))), kLogitWaves);
    if (each <= 2) logits<T, 2, GRADIENT><<<grid, kLogitThreads, 0, s>>>(a, d);
    else if (each <= 8) logits<T, 8, GRADIENT><<<grid, kLogitThreads, 0, s>>>(a, d);
    else if (each <= 16) logits<T, 16, GRADIENT><<<grid, kLogitThreads, 0, s>>>(a, d);
    else if (each <= 32) logits<T, 32, GRADIENT><<<grid, kLogitThreads, 0, s>>>(a, d);
    else logits<T, 0, GRADIENT><<<grid, kLogitThreads, 0, s>>>(a, d);
    return hipGetLastError();
}

template <bool GRADIENT> hipError_t launch_logits_of(const VocabArgs& a, const Direct& d, int64_t blocks, hipStream_t s)
{
    if (a.dtype == DTYPE_F32) return launch_logits<float, GRADIENT>(a, d, blocks, s);
    if (a.dtype == DTYPE_BF16) return launch_logits<bf16, GRADIENT>(a, d, blocks, s);
    return launch_logits<f16, GRADIENT>(a, d, blocks, s);
}

void set_blocks(Thin& p, bool brief)
{
    p.brief = !brief ? 0 : (p.k <= 16 ? 1 : (p.k <= 32 ? 2 : 4));
    p.column_blocks = static_cast<int32_t>(count(p.cols, brief ? 512 : 128));
    p.row_blocks = static_cast<int32_t>(count(count(p.rows, 16), p.row_tiles));
    p.blocks = static_cast<int64_t>(p.column_blocks) * p.row_blocks * p.splits;
}

template <typename T, typename OUT> hipError_t launch_products(const Thin& dx, const Thin& dw, hipStream_t s)
{
    const unsigned n = static_cast<unsigned>(dx.blocks), m = static_cast<unsigned>(dw.blocks);
    if (n && m && !dx.brief && !dw.brief) {
        long_products<T, OUT><<<n + m, 256, 0, s>>>(dx, dw);
        return hipGetLastError();
    }
    if (n && dx.brief) short_product<T, T, 1><<<n, 256, 0, s>>>(dx);
    else if (n) long_product<T, T, false><<<n, 256, 0, s>>>(dx);
    VOCAB_TRY(hipGetLastError());
    if (m && dw.brief == 1) short_product<T, OUT, 1><<<m, 256, 0, s>>>(dw);
    else if (m && dw.brief == 2) short_product<T, OUT, 2><<<m, 256, 0, s>>>(dw);
    else if (m && dw.brief) short_product<T, OUT, 4><<<m, 256, 0, s>>>(dw);
    else if (m) long_product<T, OUT, true><<<m, 256, 0, s>>>(dw);
    return hipGetLastError();
}

template <typename T> hipError_t backward(const VocabArgs& a, const Layout& l, uint8_t* base, hipStream_t s)
{
    const int32_t* used = reinterpret_cast<int32_t*>(base + l.used);
    Thin dx = {}, dw = {};
    if (a.dx) {
        dx.a = reinterpret_cast<float*>(base + l.dzt);
        dx.lda = l.padded;
        dx.b = a.w;
        dx.ldb = a.ldw;
        dx.rows = a.rows;
        dx.cols = a.cols;
        dx.k = a.vocab;
        dx.k_each = l.k_each;
        dx.splits = l.splits;
        dx.row_tiles = 1;
        dx.by = a.scale;
        dx.c = l.splits > 1 ? base + l.sums : static_cast<uint8_t*>(a.dx);
        dx.ldc = l.splits > 1 ? l.cols_padded : a.lddx;
        dx.used_r = used;
        // with dW in one launch where that is long, as long as a launch stays well below 2^32 threads
        const bool together = a.dw && a.rows > 16 && count(a.rows, 16) * count(a.cols, 128) <= (int64_t(1) << 23);
        set_blocks(dx, a.vocab <= 16 && !together);
    }
    if (a.dw) {
        dw.a = reinterpret_cast<float*>(base + l.dz);
        dw.lda = a.vocab;
        dw.b = a.x;
        dw.ldb = a.ldx;
        dw.rows = a.vocab;
        dw.cols = a.cols;
        dw.k = a.rows;
        dw.k_each = l.dw_each;
        dw.splits = l.dw_splits;
        dw.used_k = used;
        dw.by = a.scale;
        dw.add = l.dw_splits > 1 ? 0 : a.accumulate;
        dw.c = l.dw_splits > 1 ? base + l.dw_sums : static_cast<uint8_t*>(a.dw);
        dw.ldc = l.dw_splits > 1 ? l.cols_padded : a.lddw;
        // by short_product: so many row tiles a wave that about 8,192 waves are left
        const int64_t waves = count(a.vocab, 16) * count(a.cols, 128);
        const bool brief = a.rows <= 16 || (a.rows <= 64 && waves >= 2048);
        const int64_t each = brief ? waves / 8192 : 1;
        dw.row_tiles = static_cast<int32_t>(each < 1 ? 1 : each);
        set_blocks(dw, brief);
    }
    if (a.dw_dtype == DTYPE_F32) VOCAB_TRY((launch_products<T, float>(dx, dw, s)));
    else VOCAB_TRY((launch_products<T, T>(dx, dw, s)));
    if (a.dx && l.splits > 1) {
        const dim3 grid(static_cast<unsigned>(count(a.cols, 1024)), static_cast<unsigned>(a.rows));
        join<T><<<grid, 256, 0, s>>>(dx, static_cast<T*>(a.dx), a.lddx, used, 0);
        VOCAB_TRY(hipGetLastError());
    }
    if (a.dw && l.dw_splits > 1) {
        const dim3 grid(static_cast<unsigned>(count(a.cols, 1024)), static_cast<unsigned>(a.vocab));
        if (a.dw_dtype == DTYPE_F32) join<float><<<grid, 256, 0, s>>>(dw, static_cast<float*>(a.dw), a.lddw, nullptr, a.accumulate);
        else join<T><<<grid, 256, 0, s>>>(dw, static_cast<T*>(a.dw), a.lddw, nullptr, a.accumulate);
        VOCAB_TRY(hipGetLastError());
    }
    return hipSuccess;
}

}  // namespace

// A few rows, or less time by what this way and the other took of m x d x V,
// forward and backward (the other lays operands out, which costs the weights
// several times over, and goes through six products of fp32, in long sums where
// there are few tiles).  This way and the other, us, bf16: 17 x 4,096 x 32,768 389 and
// 655; 32 x 8,192 x 65,536 1,458 and 2,436; 40 x 2,000 x 30,000 403 and 326; 64 x 4,096 x
// 4,096 146 and 168; 1,024 x 1,024 x 1,024 103 and 107; 128 x 8,192 x 4,096 369 and 279;
// 512 x 1,024 x 4,096 183 and 108; 3,063 x 3,371 x 139 348 and 242.  fp32: 17 x 4,096 x
// 32,768 627 and 2,603; 64 x 512 x 65,536 361 and 694; 128 x 8,192 x 4,096 714 and 1,331;
// 1,024 x 1,024 x 1,024 146 and 233; 1,024 x 2,048 x 2,048 505 and 364.
bool vocab_direct(int64_t rows, int64_t cols, int64_t vocab, int dtype)
{
    const bool single = dtype == DTYPE_F32;
    if (rows <= (single ? 64 : 32) && rows * vocab <= (int64_t(1) << 26)) return true;
    if (rows > (1 << 19) || rows * vocab > (int64_t(1) << (single ? 24 : 21))) return false;
    const double w = static_cast<double>(vocab) * static_cast<double>(cols), all = w * static_cast<double>(count(rows, 16) * 16);
    return single ? 100e-9 * all <= 100.0 + 0.12 * static_cast<double>(cols) + 6.5e-6 * w
                  : 75e-9 * all <= 60.0 + 0.02 * static_cast<double>(cols);
}

size_t vocab_direct_bytes(int64_t rows, int64_t cols, int64_t vocab, bool backward)
{
    return static_cast<size_t>(layout_of(rows, cols, vocab, backward).bytes);
}

hipError_t launch_vocab_direct_forward(const VocabArgs& a, hipStream_t s)
{
    const Layout l = layout_of(a.rows, a.cols, a.vocab, false);
    uint8_t* base = static_cast<uint8_t*>(a.workspace);
    Direct d = {};
    d.groups_each = l.groups_each;
    d.padded = l.padded;
    d.partial = reinterpret_cast<float2*>(base + l.partial);
    d.partial_sum = a.smoothing != 0.0f ? reinterpret_cast<float*>(base + l.partial_sum) : nullptr;
    VOCAB_TRY(launch_logits_of<false>(a, d, l.blocks, s));
    if (l.blocks > 1) finish<<<static_cast<unsigned>(count(a.rows, 8)), kBlock, 0, s>>>(a, nullptr, nullptr, d.partial, d.partial_sum, l.blocks, l.padded);
    return hipGetLastError();
}

hipError_t launch_vocab_direct_backward(const VocabArgs& a, hipStream_t s)
{
    const Layout l = layout_of(a.rows, a.cols, a.vocab, true);
    uint8_t* base = static_cast<uint8_t*>(a.workspace);
    Direct d = {};
    d.groups_each = l.groups_each;
    d.padded = l.padded;
    d.used = reinterpret_cast<int32_t*>(base + l.used);
    d.dz = a.dw ? reinterpret_cast<float*>(base + l.dz) : nullptr;
    d.dzt = a.dx ? reinterpret_cast<float*>(base + l.dzt) : nullptr;
    VOCAB_TRY(launch_logits_of<true>(a, d, l.blocks, s));
    if (a.dtype == DTYPE_F32) return backward<float>(a, l, base, s);
    if (a.dtype == DTYPE_BF16) return backward<bf16>(a, l, base, s);
    return backward<f16>(a, l, base, s);
}

}  // namespace fasgd
