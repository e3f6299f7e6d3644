// The matrix products of the losses over a large vocabulary, with what becomes
// of them: statistics of the logits, the logits' gradient, or outputs.
//
//   c[m][n] = sum over pairs of terms (s, t) of sum_k a_s[m][k] b_t[n][k]
//
// Operands are 16-bit terms (client activations of 16 bits are one, fp32 is
// the sum of three in bf16: 24 bits).  Their products are exact in fp32 and
// summed there by v_mfma_f32_16x16x32.  For the logits a holds the classes and
// b the rows, so that what a lane has of a wave's tile is a run of classes of
// each of a few neighbouring rows: maxima and sums over classes stay within a
// lane but for two exchanges, and the gradient is laid out along the rows (for
// dW) and along the classes (for dx) straight from registers.
//
// Bound by the matrix instructions, and by the power that they draw: without
// loads, 16 x 16 x 32 instructions alone reach 2,070 TFLOP/s on random operands
// (2,450 on zeros), 32 x 32 x 16 ones 1,810.  Measured, bf16, 8,192 rows, pieces of
// 16,384 classes, 4,096 columns: statistics 850 us (1,295 TFLOP/s), gradient with
// one term along the rows and three along the classes 980 (1,120; with two 920), dx
// 770 (1,425), dW from three terms 2,330 (1,415; from two 1,550); the vendor's
// library 690 to 800 for one such product with nothing before or after.
#include <float.h>
#include <type_traits>

#include "tiles.hpp"
#include "vocab_kernels.hpp"

namespace fasgd {
namespace {

#if defined(__HIP_DEVICE_COMPILE__)

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// A wave's tile of W x W is N x N tiles of 16 x 16.  Row r of tile i is a's row
// N r + i, so a lane, which has rows 4 (l / 16) on of each tile, has the 4 N
// classes from 4 N (l / 16) on.  Column c of tile j is b's row b_row(j, c): runs of
// 4 neighbours a lane, and 16 lanes store whole lines.
__device__ __forceinline__ int b_row(int j, int c) { return j / 4 * 64 + c * 4 + j % 4; }

// Statistics of a wave's classes for each of its rows (include/fasgd_client.h):
// the largest exponent in powers of two, the sum of powers relative to it and,
// where asked for, the sum of the logits.  One pass over the accumulators, 16
// values at a time with the running maximum, since each is read out of the
// accumulation registers.
template <int W, int N>
__device__ __forceinline__ void statistics(const v4f (&acc)[N][N], const VocabProduct& p, int64_t m, int64_t n, int left,
                                           int lane)
{
    const float c = p.scale_log2e;
    const bool cut = left < W;
    const int64_t at = (p.first + m) / W * p.padded + n + 4 * (lane & 15);
    Pack<float2, 4> result[N / 4];
    Pack<float, 4> total[N / 4];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float top = -FLT_MAX, part[4] = {0.0f, 0.0f, 0.0f, 0.0f}, all = 0.0f;      // four sums: short chains
#pragma unroll
        for (int i0 = 0; i0 < N; i0 += 4) {
            float t[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v4f x = take(acc[i0 + i][j]);
#pragma unroll
                for (int r = 0; r < 4; ++r) t[i][r] = x[r];
            }
            if (cut) {      // classes past the last take no part
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const bool in = N * (4 * (lane >> 4) + r) + i0 + i < left;
                        all += in ? t[i][r] : 0.0f;
                        t[i][r] = in ? t[i][r] : -INFINITY;
                    }
            } else if (p.partial_sum) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) all += t[i][r];
            }
            float most[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) most[r] = fmaxf(fmaxf(t[0][r], t[1][r]), fmaxf(t[2][r], t[3][r]));
            const float next = fmaxf(top, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * c);
            const float down = power(top - next);
            top = next;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                part[r] *= down;
#pragma unroll
                for (int i = 0; i < 4; ++i) part[r] += power(__builtin_fmaf(t[i][r], c, -top));
            }
        }
        const float sum = (part[0] + part[1]) + (part[2] + part[3]);
        Pair x = across<16>(top);
        x = across<32>(fmaxf(x.x, x.y));
        const float both = fmaxf(x.x, x.y);
        Pair s = across<16>(sum * power(top - both));
        s = across<32>(s.x + s.y);
        result[j / 4].v[j % 4] = make_float2(both, s.x + s.y);
        s = across<16>(all);
        s = across<32>(s.x + s.y);
        total[j / 4].v[j % 4] = s.x + s.y;
    }
    if (lane < 16) {
#pragma unroll
        for (int h = 0; h < N / 4; ++h) {
            store_pack(p.partial + at + 64 * h, result[h]);
            if (p.partial_sum) store_pack(p.partial_sum + at + 64 * h, total[h]);
        }
    }
}

// The logits at the targets that lie among a wave's classes.  Each row's lies in
// one tile of all, so most of a wave's runs of rows have none.
template <int W, int N>
__device__ __forceinline__ void pick_targets(const v4f (&acc)[N][N], const VocabProduct& p, int64_t m, int64_t n, int left,
                                             int active, int lane)
{
    const int first = 4 * N * (lane >> 4);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int64_t at = n + b_row(j, lane & 15);
        const int row = at < active ? p.list[at] : -1;
        const int64_t off = row < 0 ? -1 : p.target[row] - (p.first + m);
        const bool here = off >= first && off < first + 4 * N && off < left;
        if (__builtin_amdgcn_ballot_w64(here) == 0) continue;
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const v4f x = take(acc[i][j]);
#pragma unroll
            for (int r = 0; r < 4; ++r) z = off == first + N * r + i ? x[r] : z;
        }
        if (here) p.picked[row] = z * p.by;
    }
}

typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// Two terms in a word, and the values they stand for.
template <typename T> __device__ __forceinline__ uint32_t two_terms(float x, float y);
template <> __device__ __forceinline__ uint32_t two_terms<bf16>(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{x, y}), v2bf));
}
template <> __device__ __forceinline__ uint32_t two_terms<f16>(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{x, y}), v2h));
}
template <typename T> __device__ __forceinline__ float low_term(uint32_t u);
template <> __device__ __forceinline__ float low_term<bf16>(uint32_t u) { return __uint_as_float(u << 16); }
template <> __device__ __forceinline__ float low_term<f16>(uint32_t u) { return static_cast<float>(__builtin_bit_cast(v2h, u)[0]); }
template <typename T> __device__ __forceinline__ float high_term(uint32_t u);
template <> __device__ __forceinline__ float high_term<bf16>(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
template <> __device__ __forceinline__ float high_term<f16>(uint32_t u) { return static_cast<float>(__builtin_bit_cast(v2h, u)[1]); }

// x[r] of the lanes of parts 0 to 3 (lane / 16), for r = 0 to 3, turned: x[s] of
// part g is then what part s had in x[g].
__device__ __forceinline__ void turn_parts(uint32_t (&x)[4])
{
    // halves: the upper one of the first is exchanged with the lower one of the second; rows of 16 lanes alike
    const auto a = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false), b = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
    const auto e = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), f = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    x[0] = e[0];
    x[1] = e[1];
    x[2] = f[0];
    x[3] = f[1];
}

// The gradient of a wave's logits, in both layouts.  A lane holds N rows and 4 N
// neighbouring classes; 4 rows at a time.  Words of two rows go to dz^T as they
// are, words of two classes are put together from them and turned among the parts
// of the wave, so that 4 lanes store neighbouring classes.  (Each layout's stores
// as they come, 16 bytes a lane with gaps between, cost 20 % of the 8,192 x 16,384
// x 4,096 product.)  Where the scale of a row of fp16 is its own, dz takes a turn of
// the loop before those of dz^T, which is scaled for all rows alike.  (Always so,
// a training step of 4,427 x 70 x 58,000 took 1,405 instead of 1,304 us.)
template <typename T, int W, int N>
__device__ __forceinline__ void gradient(const v4f (&acc)[N][N], const VocabProduct& p, int64_t m, int64_t n, int left,
                                         int lane)
{
    const float c = p.scale_log2e;
    constexpr bool kScaled = __is_same(T, f16);
    const float up = term_scale<T>(*p.largest);
    const int terms = p.dz_terms > p.dzt_terms ? p.dz_terms : p.dzt_terms, first = 4 * N * (lane >> 4);
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += 4) {
        const int64_t row0 = n + 16 * j0 + 4 * (lane & 15);
        float l[4], f[4], b[4], down[4];        // down: from dz's scale to that of dz^T
        bool differ = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const VocabRow row = p.row[row0 + j];
            const float own = row_scale<T>(row, up);
            l[j] = row.l;
            f[j] = row.f * own;
            b[j] = row.b * own;
            down[j] = up / own;
            differ |= own != up;
        }
        const bool apart = kScaled && __builtin_amdgcn_ballot_w64(differ) != 0;
        float v[4][N][4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float z = acc[i][j0 + j][r];
                    asm volatile("" : "+v"(z));     // read out of the accumulation registers here
                    v[r][i][j] = __builtin_fmaf(f[j], power(__builtin_fmaf(z, c, -l[j])), -b[j]);
                    if (left < W) v[r][i][j] = first + N * r + i < left ? v[r][i][j] : 0.0f;     // nothing of classes past the last
                }
        // Term t in both layouts; `alone`, dz's one term, and the values to the scale of dz^T.
        auto take_term = [&](auto alone, int t) {
            constexpr bool kAlone = decltype(alone)::value;
            uint16_t* dzt = p.dzt + (m + first) * p.ld_dzt + t * p.padded + row0;
            uint32_t own[4][N / 2][4];     // of row j: word of classes, part's run r
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t w[N][2];
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
                        const uint32_t u = two_terms<T>(v[r][i][j], v[r][i][j + 1]);
                        w[i][j / 2] = u;
                        v[r][i][j] = kAlone ? v[r][i][j] * down[j] : v[r][i][j] - low_term<T>(u);
                        v[r][i][j + 1] = kAlone ? v[r][i][j + 1] * down[j + 1] : v[r][i][j + 1] - high_term<T>(u);
                    }
                if (!kAlone && t < p.dzt_terms) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        Pack<uint32_t, 2> x;
                        x.v[0] = w[i][0];
                        x.v[1] = w[i][1];
                        store_pack(reinterpret_cast<uint32_t*>(dzt + (N * r + i) * p.ld_dzt), x);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < N; i += 2)
                        own[j][i / 2][r] = __builtin_amdgcn_perm(w[i + 1][j / 2], w[i][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
            }
            if (t >= p.dz_terms || (!kAlone && apart)) return;
            uint16_t* dz = p.dz + row0 * p.ld_dz + t * p.classes + m + N * (lane >> 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) turn_parts(own[j][i]);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    Pack<uint32_t, N / 2> x;
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) x.v[i] = own[j][i][s];
                    store_pack(reinterpret_cast<uint32_t*>(dz + j * p.ld_dz + 4 * N * s), x);
                }
            }
        };
        if constexpr (kScaled) {
            if (apart) take_term(std::true_type{}, 0);
        }
        for (int t = 0; t < terms; ++t) take_term(std::false_type{}, t);
    }
}

// A wave's outputs times `by` to rows m on and columns n on of c ([rows][cols],
// row stride ld), 4 neighbouring columns of a lane at once, at any alignment.
// WHOLE: all of them lie in c, and c is not added to.
template <typename OUT, int W, int N, bool WHOLE>
__device__ __forceinline__ void write_sums(const v4f (&acc)[N][N], OUT* c, int64_t ld, int64_t rows, int64_t cols, int64_t m,
                                           int64_t n, bool add, int lane, float by)
{
    const int first = 4 * N * (lane >> 4);
    const int rows_left = static_cast<int>(rows - m < W ? rows - m : W) - first;
    const int cols_left = static_cast<int>(cols - n < W ? cols - n : W) - 4 * (lane & 15);
    OUT* base = c + (m + first) * ld + n + 4 * (lane & 15);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int h = 0; h < N / 4; ++h) {
            v4f t[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = take(acc[i][4 * h + e]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                OUT* out = base + (N * r + i) * ld + 64 * h;
                Pack<OUT, 4> x;
                if (WHOLE) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[e] = from_float<OUT>(t[e][r] * by);
                    store_pack(out, x);
                } else if (N * r + i < rows_left) {
                    const int here = cols_left - 64 * h;
                    if (here >= 4) {
                        if (add) x = load_pack<OUT, 4>(out);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x.v[e] = from_float<OUT>(add ? to_float(x.v[e]) + t[e][r] * by : t[e][r] * by);
                        store_pack(out, x);
                    } else {
#pragma unroll
                        for (int e = 0; e < 3; ++e)
                            if (e < here) out[e] = from_float<OUT>(add ? to_float(out[e]) + t[e][r] * by : t[e][r] * by);
                    }
                }
            }
        }
}

template <typename OUT, int W, int N>
__device__ __forceinline__ void write_product(const v4f (&acc)[N][N], OUT* c, int64_t ld, int64_t rows, int64_t cols, int64_t m,
                                              int64_t n, bool add, int lane, float by)
{
    if (!add && m + W <= rows && n + W <= cols) write_sums<OUT, W, N, true>(acc, c, ld, rows, cols, m, n, add, lane, by);
    else write_sums<OUT, W, N, false>(acc, c, ld, rows, cols, m, n, add, lane, by);
}

// c += a b in c's own accumulation registers.  A wave's 128 x 128 sums fill all
// 256 of them, and the compiler, which may give the instruction another place for
// its result, moves a quarter of the sums about in each round of the loop for it.
// What reads c next as anything but a sum waits for it (sums_done).
template <typename T> __device__ __forceinline__ void multiply_into(v4f& c, const v4i& a, const v4i& b);
template <> __device__ __forceinline__ void multiply_into<bf16>(v4f& c, const v4i& a, const v4i& b)
{
    asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
template <> __device__ __forceinline__ void multiply_into<f16>(v4f& c, const v4i& a, const v4i& b)
{
    asm("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
template <int N> __device__ __forceinline__ void sums_done(v4f (&c)[N][N])
{
    // the sums pass through on both sides: the last instruction is before the
    // wait, which is longer than its passes, and every read of them after it
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) asm volatile("" : "+a"(c[i][j]));
    asm volatile("s_nop 15" ::: "memory");
    asm volatile("s_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) asm volatile("" : "+a"(c[i][j]));
}

// What is the same in all lanes, said so: where the compiler does not see it, it
// loops over the lanes' buffers at each load of a stage (the gradient's product
// at 8,192 x 16,384 x 4,096 1,130 against 960 us).
__device__ __forceinline__ const uint8_t* same_pointer(const uint8_t* p)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint32_t low = __builtin_amdgcn_readfirstlane(static_cast<int>(at)), high = __builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32));
    return reinterpret_cast<const uint8_t*>(static_cast<uint64_t>(high) << 32 | low);
}
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Where an operand's next stage is loaded from.
struct Place {
    const uint8_t* base;    // of the tile's rows
    uint32_t bytes;         // of the buffer; 0 behind the last stage: zeros are read
    uint32_t which;         // of the terms, 2 bits a pair
    int plane, at, pair;
};

#endif

// The block's tile goes through LDS, 64 of the contraction a stage, each
// operand's row 128 bytes of it, loaded straight to LDS.  (Rows of 64 bytes, with
// stages half as long and twice as many on their way, took 8 % longer: L2 gives
// whole lines.)  A stage is two sub-steps of 32, whose fragments are read while
// the one before is multiplied.  Parts of stages (a's or b's rows) go round five
// slots: a's part of stage k + 2 into the fifth while stage k's first sub-step is
// multiplied, b's into a's slot as soon as every wave has read it.  Five stages are
// a round; those behind the last are zeros, so a contraction of 16 pays for 20.
// (Two whole stages in four slots, stage k + 2 into stage k's place: as fast over
// 64 stages, slower over long contractions, with 32 x 32 x 16 instructions dW
// 1,650 against 1,580 us.)
// CUT: a's rows end before the contraction's last block.
template <typename T, int W, int WM, int WHAT, bool CUT>
__global__ __launch_bounds__(kThreads, W >= 96 ? 1 : 2) void vocab_product(VocabProduct p, int tiles_m, int tiles_n, int per_split)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = Geometry<W, WM>;
    static_assert(G::kStageA == G::kStageB, "a slot takes either operand");
    constexpr int N = W / 16, kSlot = G::kStageA, kLoads = G::kLoadsA;
    __shared__ __attribute__((aligned(16))) uint8_t s0[kSlot], s1[kSlot], s2[kSlot], s3[kSlot], s4[kSlot];
    const int active = same(*p.active);
    const int tiles = tiles_m * tiles_n;
    // (quotients come from the vector unit; all that follows from them is the same in all lanes)
    const int split = same(static_cast<int>(blockIdx.x) / tiles);
    const int id = same(tile_of(static_cast<int>(blockIdx.x) - split * tiles, tiles_m, tiles_n)), row = same(id / tiles_n);
    const int64_t m0 = static_cast<int64_t>(row) * G::kRowsA, n0 = static_cast<int64_t>(id - row * tiles_n) * G::kRowsB;
    const int rows_a = p.rows_a_active ? active : p.a.rows, rows_b = p.rows_b_active ? active : p.b.rows;
    // rows of a gradient that a contraction reads are whole blocks of 128
    const int pad_b = p.rows_b_active ? (rows_b + 127) / 128 * 128 : rows_b;
    if (m0 >= rows_a || n0 >= pad_b) return;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / G::kWavesN, wave_n = wave % G::kWavesN;

    const int blocks = p.k_active ? (active + 127) / 128 * 2 : p.blocks;
    const int kb0 = split * per_split;
    const int own_blocks = blocks - kb0 < per_split ? blocks - kb0 : per_split;
    const int terms = same(p.terms), along = same(own_blocks * kBytes), steps = own_blocks > 0 ? own_blocks * terms : 0;

    // Rows past a's last are read as its last; b's are padded to 128,
    // and what lies behind that is read as the last of it.  Load q of a wave
    // fills 8 rows of a slot, 128 bytes each, the 16-byte chunk c of row r of a
    // tile in place slot(c, r).
    uint32_t off_a[kLoads], off_b[kLoads];
    const int last_a = static_cast<int>(rows_a - m0 < G::kRowsA ? rows_a - m0 : G::kRowsA) - 1;
    const int last_b = static_cast<int>(pad_b - n0 < G::kRowsB ? pad_b - n0 : G::kRowsB) - 1;
    const int chunk_at = slot(lane & 7, (wave * 8 + (lane >> 3)) % 16) * 16;     // of the lane's loads
#pragma unroll
    for (int q = 0; q < kLoads; ++q) {
        const int place = (q * 4 + wave) * 8 + (lane >> 3), i = place % W / 16, r = place % 16;
        const int row_a = place / W * W + N * r + i, row_b = place / W * W + b_row(i, r);
        off_a[q] = static_cast<uint32_t>(row_a < last_a ? row_a : last_a) * static_cast<uint32_t>(p.a.ld) + chunk_at;
        off_b[q] = static_cast<uint32_t>(row_b < last_b ? row_b : last_b) * static_cast<uint32_t>(p.b.ld) + chunk_at;
    }
    // the bytes are those of the tile's rows: what lies 2^31 on is past the end
    const int64_t skip = static_cast<int64_t>(kb0) * kBytes;
    Place pa = {same_pointer(p.a.data + m0 * p.a.ld + skip), static_cast<uint32_t>(same(static_cast<int>((last_a + 1) * p.a.ld - skip))),
                static_cast<uint32_t>(same(p.terms_a)), same(p.a.plane), 0, 0};
    Place pb = {same_pointer(p.b.data + n0 * p.b.ld + skip), static_cast<uint32_t>(same(static_cast<int>((last_b + 1) * p.b.ld - skip))),
                static_cast<uint32_t>(same(p.terms_b)), same(p.b.plane), 0, 0};

    const int place_a = (wave_m * W + (lane & 15)) * kBytes, place_b = (wave_n * W + (lane & 15)) * kBytes;
    const int chunk[2] = {slot(lane >> 4, lane & 15) * 16, slot(4 + (lane >> 4), lane & 15) * 16};

    v4f acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // Loads go on from stage to stage, a pair of terms over the contraction and
    // then the next pair, then zeros.  The pairs come with the smallest first: the
    // matrix instruction aligns its products with the sum and cuts off what lies
    // 3 bits below the sum's last, so the large sums are to be met as few times
    // as there are blocks (fp32, 1,024 rows: dx off by 3.3e-6 with a block's
    // pairs together, 1.4e-6 so).
    auto next = [&](Place& l) {     // without branches, which would part the stage's instructions
        const int more = (l.at + kBytes - along) >> 31, turn = ~more & (l.pair + 1 - terms) >> 31;     // all ones: yes
        l.at = (l.at + (kBytes & more)) & ~turn;
        l.pair -= turn;
        l.bytes &= static_cast<uint32_t>(more | turn);
    };
    auto load_a = [&](uint8_t* to, int from, int until) {
        const int at = same(pa.at + static_cast<int>(pa.which >> (2 * pa.pair) & 3u) * pa.plane), rest = CUT ? p.a_bytes - pa.at : 0;
        const auto from_a = buffer(pa.base, static_cast<uint32_t>(same(static_cast<int>(pa.bytes))));
#pragma unroll
        for (int q = from; q < until; ++q)      // past a buffer's end zeros are read
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_a, (lds_ptr)(to + (q * 4 + wave) * 1024), 16,
                                                     CUT && chunk_at >= rest ? 0x80000000u : off_a[q], at, 0, 0);
        if (until == kLoads) next(pa);
    };
    auto load_b = [&](uint8_t* to, int from, int until) {
        const int at = same(pb.at + static_cast<int>(pb.which >> (2 * pb.pair) & 3u) * pb.plane);
        const auto from_b = buffer(pb.base, static_cast<uint32_t>(same(static_cast<int>(pb.bytes))));
#pragma unroll
        for (int q = from; q < until; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from_b, (lds_ptr)(to + (q * 4 + wave) * 1024), 16, off_b[q], at, 0, 0);
        if (until == kLoads) next(pb);
    };
    v4i fa[2][N], fb[2][N];
    auto read = [&](int f, int q, const uint8_t* a, const uint8_t* b, int u) {     // fragment q of 2 N: b's, then a's
        if (q < N) fb[f][q] = *reinterpret_cast<const v4i*>(b + place_b + chunk[u] + q * 16 * kBytes);
        else fa[f][q - N] = *reinterpret_cast<const v4i*>(a + place_a + chunk[u] + (q - N) * 16 * kBytes);
    };
    // Multiplies fragments f.  Between the matrix instructions, in this order, go
    // the reads of the next fragments, in the first half, so that they have arrived
    // at its end, and kLoads loads, spread evenly.
    auto multiply = [&](int f, const uint8_t* a, const uint8_t* b, int u, auto load) {
        constexpr int kPairs = N * N / 2, kReads = 2 * N / (kPairs / 2), kApart = kPairs / kLoads;
#pragma unroll
        for (int s = 0; s < kPairs; ++s) {
            if (s < kPairs / 2) {
#pragma unroll
                for (int q = 0; q < kReads; ++q) read(f ^ 1, s * kReads + q, a, b, u);
            }
            if (s % kApart == kApart - 1) load(s / kApart);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = (2 * s + e) / N, j = (2 * s + e) % N;
                if constexpr (W == 128) multiply_into<T>(acc[i][j], fa[f][i], fb[f][j]);
                else acc[i][j] = mfma<T>(fa[f][i], fb[f][j], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Stage k lies in (a, b), the next in (an, bn) or on its way there, and the
    // first fragments hold stage k's first sub-step.
    auto step = [&](uint8_t* a, uint8_t* b, uint8_t* an, uint8_t* bn, uint8_t* fifth) {
        multiply(0, a, b, 1, [&](int q) { load_a(fifth, q, q + 1); });
        // The next stage has arrived (a's part of the one after it is on its way)
        // and every wave holds the rest of this one in registers.
        __builtin_amdgcn_s_waitcnt(0x0070 | kLoads);     // vmcnt(kLoads) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        multiply(1, an, bn, 0, [&](int q) { load_b(a, q, q + 1); });
    };
    if (steps > 0) {
        load_a(s0, 0, kLoads);
        load_b(s1, 0, kLoads);
        load_a(s2, 0, kLoads);
        load_b(s3, 0, kLoads);
        __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 2 * N; ++q) read(0, q, s0, s1, 0);
        __builtin_amdgcn_sched_barrier(0);
        int k = 0;
        do {
            step(s0, s1, s2, s3, s4);
            step(s2, s3, s4, s0, s1);
            step(s4, s0, s1, s2, s3);
            step(s1, s2, s3, s4, s0);
            step(s3, s4, s0, s1, s2);
            k += 5;
        } while (k < steps);
        // the last loads land in LDS before this block gives it up
        __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
        if constexpr (W == 128) sums_done<N>(acc);
    }

    const int64_t m = m0 + wave_m * W, n = n0 + wave_n * W;
    if constexpr (WHAT == VOCAB_STATISTICS) {
        const int here = static_cast<int>(rows_a - m < W ? rows_a - m : W);
        if (m < rows_a) statistics<W, N>(acc, p, m, n, here, lane);
        if (m < rows_a && p.target) pick_targets<W, N>(acc, p, m, n, here, active, lane);
    } else if constexpr (WHAT == VOCAB_GRADIENT) {
        const int64_t left = rows_a - m;
        const int here = static_cast<int>(left < W ? (left < 0 ? 0 : left) : W);
        gradient<T, W, N>(acc, p, m, n, here, lane);
    } else {
        const float by = p.by / (p.largest ? term_scale<T>(*p.largest) : 1.0f);
        const bool add = p.add != 0;
        if (m >= rows_a) return;
        if (p.c_dtype == DTYPE_F32)
            write_product<float, W, N>(acc, static_cast<float*>(p.c) + split * p.split_stride, p.ldc, rows_a, rows_b, m, n, add, lane, by);
        else
            write_product<T, W, N>(acc, static_cast<T*>(p.c), p.ldc, rows_a, rows_b, m, n, add, lane, by);
    }
#endif
}

int64_t count(int64_t x, int64_t side) { return (x + side - 1) / side; }

template <typename T, int W> hipError_t launch_what(int what, const VocabProduct& p, int64_t m, int64_t n, hipStream_t s)
{
    constexpr int kSide = 2 * W;
    const int tiles_m = static_cast<int>(count(m, kSide)), tiles_n = static_cast<int>(count(n, kSide));
    const unsigned blocks = static_cast<unsigned>(tiles_m) * tiles_n * p.splits;
    const int per_split = static_cast<int>(count(p.blocks, p.splits));
    switch (what) {
    case VOCAB_STATISTICS:
        if (p.a_bytes) vocab_product<T, W, 2, VOCAB_STATISTICS, true><<<blocks, kThreads, 0, s>>>(p, tiles_m, tiles_n, per_split);
        else vocab_product<T, W, 2, VOCAB_STATISTICS, false><<<blocks, kThreads, 0, s>>>(p, tiles_m, tiles_n, per_split);
        break;
    case VOCAB_GRADIENT:
        if (p.a_bytes) vocab_product<T, W, 2, VOCAB_GRADIENT, true><<<blocks, kThreads, 0, s>>>(p, tiles_m, tiles_n, per_split);
        else vocab_product<T, W, 2, VOCAB_GRADIENT, false><<<blocks, kThreads, 0, s>>>(p, tiles_m, tiles_n, per_split);
        break;
    default: vocab_product<T, W, 2, VOCAB_STORE, false><<<blocks, kThreads, 0, s>>>(p, tiles_m, tiles_n, per_split); break;
    }
    return hipGetLastError();
}

}  // namespace

// Microseconds of a tile's blocks: of a stage with as many blocks on a CU as
// fit (of 128 x 128 two, of 256 x 256 one), of a stage of a 128 x 128 tile
// alone on its CU, and of what a tile costs besides (256 tiles of 256 x 256 over
// 4,096 take 103 us, over 1,024 35, and 104 and 42 where sums are stored; of
// 128 x 128 39 and 14; 512 of those 62 and 22).  A split contraction's parts are
// read again, at about 4 TB/s.
VocabPlan vocab_plan(int64_t m, int64_t n, int64_t stages, int most_splits)
{
    VocabPlan best = {64, 1};
    double least = 0.0;
    for (const int wave : {128, 64}) {
        const int64_t tiles = count(m, 2 * wave) * count(n, 2 * wave);
        const double stage = wave == 128 ? 1.41 : 0.84, alone = wave == 128 ? 1.41 : 0.52, besides = wave == 128 ? 13.0 : 8.0;
        for (int s = 1; s <= most_splits && s <= stages; ++s) {
            const int64_t blocks = tiles * s, slots = wave == 128 ? 256 : 512, rest = blocks % slots;
            const double each = static_cast<double>(count(stages, s));
            double t = static_cast<double>(blocks / slots) * (stage * each + besides);
            if (rest > 0) t += (rest <= 256 ? alone : stage) * each + besides;
            if (s > 1) t += 4.0 * s * static_cast<double>(m) * static_cast<double>(n) / 4e6;
            if (least == 0.0 || t < least) {
                least = t;
                best = VocabPlan{wave, s};
            }
        }
    }
    return best;
}

hipError_t launch_vocab_product(int what, const VocabProduct& p, int64_t m, int64_t n, hipStream_t s)
{
    if (p.wave == 128)
        return p.f16 ? launch_what<f16, 128>(what, p, m, n, s) : launch_what<bf16, 128>(what, p, m, n, s);
    return p.f16 ? launch_what<f16, 64>(what, p, m, n, s) : launch_what<bf16, 64>(what, p, m, n, s);
}

}  // namespace fasgd
