// The matrix products of the losses over a large vocabulary, with what becomes
// of them: statistics of the logits, the logits' gradient, or outputs.
//
//   c[m][n] = sum over pairs of terms (s, t) of sum_k a_s[m][k] b_t[n][k]
//
// Operands are 16-bit terms (client activations of 16 bits are one, fp32 is
// the sum of three in bf16: 24 bits).  Their products are exact in fp32 and
// summed there by v_mfma_f32_32x32x16.  For the logits a holds the classes and
// b the rows, so that a lane's 16 outputs of a matrix tile are classes of one
// row: maxima and sums over classes stay within a lane but for one exchange,
// and the gradient is laid out along the rows (for dW) and along the classes
// (for dx) straight from registers.
//
// Bound by the matrix instructions.
#include <float.h>

#include "tiles.hpp"
#include "vocab_kernels.hpp"

namespace fasgd {
namespace {

#if defined(__HIP_DEVICE_COMPILE__)

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// x of this lane and the lane 32 away: the larger, the sum.
__device__ __forceinline__ float larger_half(float x)
{
    const Pair p = across<32>(x);
    return fmaxf(p.x, p.y);
}
__device__ __forceinline__ float sum_half(float x)
{
    const Pair p = across<32>(x);
    return p.x + p.y;
}

// Statistics of a wave's classes for each of its rows (include/fasgd_client.h):
// the largest exponent in powers of two, the sum of powers relative to it and,
// where asked for, the sum of the logits.  One pass over the accumulators, a
// matrix tile at a time with the running maximum, since each is read out of
// the accumulation registers.
template <int W, int N>
__device__ __forceinline__ void statistics(const v16f (&acc)[N][N], const VocabProduct& p, int64_t m, int64_t n, int left,
                                           int lane)
{
    const float c = p.scale_log2e;
    const bool cut = left < W;
    float2* out = p.partial + (p.first + m) / W * p.padded + n + N * (lane & 31);
    float* out_sum = p.partial_sum ? p.partial_sum + (p.first + m) / W * p.padded + n + N * (lane & 31) : nullptr;
    Pack<float2, N> result;
    Pack<float, N> total;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float top = -FLT_MAX, sum = 0.0f, all = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v16f t = take(acc[i][j]);
            if (cut) {      // classes past the last take no part
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = (8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * N + i;
                    all += row < left ? t[r] : 0.0f;
                    t[r] = row < left ? t[r] : -INFINITY;
                }
            } else if (out_sum) {
#pragma unroll
                for (int r = 0; r < 16; ++r) all += t[r];
            }
            float most = t[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) most = fmaxf(most, t[r]);
            const float next = fmaxf(top, most * c);
            sum *= power(top - next);
            top = next;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += power(__builtin_fmaf(t[r], c, -top));
        }
        const float both = larger_half(top);
        sum = sum_half(sum * power(top - both));
        result.v[j] = make_float2(both, sum);
        total.v[j] = sum_half(all);
    }
    if (lane < 32) {
        store_pack(out, result);
        if (out_sum) store_pack(out_sum, total);
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

// The gradient of a wave's logits, in both layouts.  A lane holds N rows and,
// at a time, 4 N neighbouring classes: words of two rows go to dz^T as they are,
// words of two classes are put together from them.
template <typename T, int W, int N>
__device__ __forceinline__ void gradient(const v16f (&acc)[N][N], const VocabProduct& p, int64_t m, int64_t n, int left,
                                         int lane)
{
    const float c = p.scale_log2e;
    float l[N], f[N], b[N];
    const float up = term_scale<T>(*p.largest);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const VocabRow row = p.row[n + N * (lane & 31) + j];
        l[j] = row.l;
        f[j] = row.f * up;
        b[j] = row.b * up;
    }
    const int terms = p.dz_terms > p.dzt_terms ? p.dz_terms : p.dzt_terms;
    uint16_t* dz = p.dz + (n + N * (lane & 31)) * p.ld_dz + m + 4 * N * (lane >> 5);
    uint16_t* dzt = p.dzt + (m + 4 * N * (lane >> 5)) * p.ld_dzt + n + N * (lane & 31);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float v[4 * N][N];
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float z = acc[i][j][4 * q + r];
                    asm volatile("" : "+v"(z));     // read out of the accumulation registers here
                    v[r * N + i][j] = __builtin_fmaf(f[j], power(__builtin_fmaf(z, c, -l[j])), -b[j]);
                }
        if (left < W) {     // nothing of classes past the last
#pragma unroll
            for (int k = 0; k < 4 * N; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) v[k][j] = 4 * N * (2 * q + (lane >> 5)) + k < left ? v[k][j] : 0.0f;
        }
        for (int t = 0; t < terms; ++t) {
            uint32_t w[4 * N][N / 2];
#pragma unroll
            for (int k = 0; k < 4 * N; ++k)
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const uint32_t u = two_terms<T>(v[k][j], v[k][j + 1]);
                    w[k][j / 2] = u;
                    v[k][j] -= low_term<T>(u);
                    v[k][j + 1] -= high_term<T>(u);
                }
            if (t < p.dzt_terms) {
                uint16_t* out = dzt + t * p.padded;
#pragma unroll
                for (int k = 0; k < 4 * N; ++k) {
                    Pack<uint32_t, N / 2> x;
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) x.v[j] = w[k][j];
                    store_pack(reinterpret_cast<uint32_t*>(out + (8 * N * q + k) * p.ld_dzt), x);
                }
            }
            if (t < p.dz_terms) {
                uint16_t* out = dz + t * p.classes + 8 * N * q;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    Pack<uint32_t, 2 * N> x;
#pragma unroll
                    for (int k = 0; k < 4 * N; k += 2)
                        x.v[k / 2] = __builtin_amdgcn_perm(w[k + 1][j / 2], w[k][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
                    store_pack(reinterpret_cast<uint32_t*>(out + j * p.ld_dz), x);
                }
            }
        }
    }
}

// A buffer that is the same in all lanes, said so: where the compiler does not
// see it, it loops over the lanes' values at each load of a stage (the gradient's
// product at 8,192 x 16,384 x 4,096 1,130 against @GB@ us).
__device__ __forceinline__ auto same_buffer(const uint8_t* p, int64_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    const uint32_t low = __builtin_amdgcn_readfirstlane(static_cast<int>(at)), high = __builtin_amdgcn_readfirstlane(static_cast<int>(at >> 32));
    const int64_t most = bytes < 0xffffffffll ? bytes : 0xffffffffll;
    const uint32_t n = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<uint32_t>(most)));
    return buffer(reinterpret_cast<const uint8_t*>(static_cast<uint64_t>(high) << 32 | low), n);
}

// Order of a sub-step's instructions for the compiler's scheduler: between
// matrix instructions go the LDS reads, in the first half, so that they have
// arrived at its end, and the loads.
template <int MFMA, int READS, int LOADS, int I = 0> __device__ __forceinline__ void order()
{
    constexpr int kMfma = 0x8, kDsRead = 0x100, kVmem = 0x20, kHalf = MFMA / 2;
    constexpr int kReads = I < kHalf ? (I + 1) * READS / kHalf - I * READS / kHalf : 0;
    constexpr int kLoads = (I + 1) * LOADS / MFMA - I * LOADS / MFMA;
    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
    if constexpr (kReads > 0) __builtin_amdgcn_sched_group_barrier(kDsRead, kReads, 0);
    if constexpr (kLoads > 0) __builtin_amdgcn_sched_group_barrier(kVmem, kLoads, 0);
    if constexpr (I + 1 < MFMA) order<MFMA, READS, LOADS, I + 1>();
}

#endif

// The block's tile goes through LDS as in the 8-bit product: two stages of 64
// along the contraction, each operand's row 128 bytes of it, loaded straight
// to LDS; a stage is four sub-steps of 16, whose fragments are read while the
// one before is multiplied.
// CUT: a's rows end before the contraction's last block.
template <typename T, int W, int WM, int WHAT, bool CUT>
__global__ __launch_bounds__(kThreads, W >= 96 ? 1 : 2) void vocab_product(VocabProduct p, int tiles_m, int tiles_n, int per_split)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = Geometry<W, WM>;
    constexpr int N = G::kTiles;
    __shared__ __attribute__((aligned(16))) uint8_t a0[G::kStageA], b0[G::kStageB], a1[G::kStageA], b1[G::kStageB];
    const int active = __builtin_amdgcn_readfirstlane(*p.active);
    const int tiles = tiles_m * tiles_n;
    const int id = tile_of(blockIdx.x % tiles, tiles_m, tiles_n);
    const int split = blockIdx.x / tiles;
    const int64_t m0 = static_cast<int64_t>(id / tiles_n) * G::kRowsA, n0 = static_cast<int64_t>(id % tiles_n) * G::kRowsB;
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
    const int steps = own_blocks > 0 ? own_blocks * p.terms : 0;

    // Rows past a's last are read as its last; b's padding to 128 rows of zeros
    // is there, and what lies behind it is read as its last.
    uint32_t off_a[G::kLoadsA], off_b[G::kLoadsB];
    const int last_a = static_cast<int>(rows_a - m0 < G::kRowsA ? rows_a - m0 : G::kRowsA) - 1;
    const int last_b = static_cast<int>(pad_b - n0 < G::kRowsB ? pad_b - n0 : G::kRowsB) - 1;
    auto offset = [&](int q, int last, int64_t ld) {
        const int place = (q * 4 + wave) * 8 + (lane >> 3), r = place % 32;
        const int row = place / W * W + r * N + place % W / 32;
        return static_cast<uint32_t>(row < last ? row : last) * static_cast<uint32_t>(ld) + slot(lane & 7, r) * 16u;
    };
#pragma unroll
    for (int q = 0; q < G::kLoadsA; ++q) off_a[q] = offset(q, last_a, p.a.ld);
#pragma unroll
    for (int q = 0; q < G::kLoadsB; ++q) off_b[q] = offset(q, last_b, p.b.ld);
    // no more than the tile's rows: what lies 2^31 bytes on is past the end
    const auto ga = same_buffer(p.a.data + m0 * p.a.ld + static_cast<int64_t>(kb0) * kBytes,
                                (last_a + 1) * p.a.ld - static_cast<int64_t>(kb0) * kBytes);
    const auto gb = same_buffer(p.b.data + n0 * p.b.ld + static_cast<int64_t>(kb0) * kBytes,
                                (last_b + 1) * p.b.ld - static_cast<int64_t>(kb0) * kBytes);

    const int place_a = (wave_m * W + (lane & 31)) * kBytes, place_b = (wave_n * W + (lane & 31)) * kBytes;
    int chunk[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) chunk[c] = slot(c * 2 + (lane >> 5), lane & 31) * 16;

    v16f acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // Loads go on from stage to stage, a pair of terms over the contraction and
    // then the next pair.  Past the last it is loaded again.  The pairs come
    // with the smallest first: the matrix instruction aligns its 16 products
    // with the sum and cuts off what lies 3 bits below the sum's last, so the
    // large sums are to be met as few times as there are blocks (fp32, 1,024
    // rows: dx off by 3.3e-6 with a block's pairs together, 1.4e-6 so).
    int at = 0, pair = 0;
    constexpr int kLoads = G::kLoadsA + G::kLoadsB;
    constexpr int kFirst = kLoads / 2;
    // (as same_buffer)
    const int terms = __builtin_amdgcn_readfirstlane(p.terms), along = __builtin_amdgcn_readfirstlane(own_blocks * kBytes);
    const uint32_t terms_a = __builtin_amdgcn_readfirstlane(p.terms_a), terms_b = __builtin_amdgcn_readfirstlane(p.terms_b);
    const int plane_a = __builtin_amdgcn_readfirstlane(p.a.plane), plane_b = __builtin_amdgcn_readfirstlane(p.b.plane);
    int at_a, at_b, rest = 0;
    auto own_chunk = [&](int q) { return slot(lane & 7, ((q * 4 + wave) * 8 + (lane >> 3)) % 32) * 16; };
    auto next = [&]() {
        if (CUT) rest = p.a_bytes - at;     // bytes of a row from here on
        at_a = at + static_cast<int>(terms_a >> (2 * pair) & 3u) * plane_a;
        at_b = at + static_cast<int>(terms_b >> (2 * pair) & 3u) * plane_b;
        if (at + kBytes < along) {
            at += kBytes;
        } else if (pair + 1 < terms) {
            ++pair;
            at = 0;
        }
    };
    auto load = [&](uint8_t* a, uint8_t* b, int from, int to) {
#pragma unroll
        for (int q = from; q < to; ++q) {
            if (q < G::kLoadsA)     // past a buffer's end zeros are read
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ga, (lds_ptr)(a + (q * 4 + wave) * 1024), 16,
                                                         CUT && own_chunk(q) >= rest ? 0x80000000u : off_a[q], at_a, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(gb, (lds_ptr)(b + ((q - G::kLoadsA) * 4 + wave) * 1024), 16, off_b[q - G::kLoadsA], at_b, 0, 0);
        }
    };
    v4i fa[2][N], fb[2][N];
    auto read = [&](int f, const uint8_t* a, const uint8_t* b, int u) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            fa[f][i] = *reinterpret_cast<const v4i*>(a + place_a + chunk[u] + i * 32 * kBytes);
            fb[f][i] = *reinterpret_cast<const v4i*>(b + place_b + chunk[u] + i * 32 * kBytes);
        }
    };
    auto multiply = [&](int f) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[i][j] = mfma<T>(fa[f][i], fb[f][j], acc[i][j]);
    };
    // Stage k lies in (a, b), the next in (an, bn) or on its way there, and the
    // first fragments hold stage k's first sub-step.
    auto step = [&](uint8_t* a, uint8_t* b, uint8_t* an, uint8_t* bn) {
#pragma unroll
        for (int u = 0; u < 3; ++u) {
            read((u + 1) & 1, a, b, u + 1);
            if (u == 0) load(an, bn, kFirst, kLoads);
            multiply(u & 1);
            if (u == 0) order<N * N, 2 * N, kLoads - kFirst>();
            else order<N * N, 2 * N, 0>();
            __builtin_amdgcn_sched_barrier(0);
        }
        // The next stage has arrived and every wave holds the rest of this one
        // in registers: its LDS is free for the stage after next.  Its loads go
        // over two sub-steps: at once they are more than the CU takes in while
        // one is multiplied (8,192 x 16,384 x 4,096 906 against 850 us).
        __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        next();
        read(0, an, bn, 0);
        load(a, b, 0, kFirst);
        multiply(1);
        order<N * N, 2 * N, kFirst>();
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
        next();
        load(a0, b0, 0, kLoads);
        next();
        load(a1, b1, 0, kFirst);
        __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0)
        __syncthreads();
        read(0, a0, b0, 0);
        int k = 0;
        do {        // an even number of stages
            step(a0, b0, a1, b1);
            step(a1, b1, a0, b0);
            k += 2;
        } while (k < steps);
        // the last loads land in LDS before this block gives it up
        __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
    }

    const int64_t m = m0 + wave_m * W, n = n0 + wave_n * W;
    if constexpr (WHAT == VOCAB_STATISTICS) {
        if (m < rows_a) statistics<W, N>(acc, p, m, n, static_cast<int>(rows_a - m < W ? rows_a - m : W), lane);
    } else if constexpr (WHAT == VOCAB_GRADIENT) {
        const int64_t left = rows_a - m;
        gradient<T, W, N>(acc, p, m, n, static_cast<int>(left < W ? (left < 0 ? 0 : left) : W), lane);
    } else {
        const float by = p.by / (p.largest ? term_scale<T>(*p.largest) : 1.0f);
        const bool add = p.add != 0;
        if (m >= rows_a) return;
        if (p.c_dtype == DTYPE_F32)
            write_outputs<float, W, N>(acc, static_cast<float*>(p.c) + split * p.split_stride, p.ldc, rows_a, rows_b, m, n, add, lane, by);
        else
            write_outputs<T, W, N>(acc, static_cast<T*>(p.c), p.ldc, rows_a, rows_b, m, n, add, lane, by);
    }
#endif
}

int64_t count(int64_t x, int64_t side) { return (x + side - 1) / side; }

template <typename T, int W> hipError_t launch_what(int what, const VocabProduct& p, int64_t m, int64_t n, hipStream_t s)
{
    constexpr int kSide = 2 * W;
    const int tiles_m = static_cast<int>(count(m, kSide)), tiles_n = static_cast<int>(count(n, kSide));
    const unsigned blocks = static_cast<unsigned>(tiles_m) * tiles_n * p.splits;
    int per_split = static_cast<int>(count(p.blocks, p.splits));
    per_split += per_split & 1;     // the kernel takes stages in pairs
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
// 4,096 take 104 us, over 1,024 32; of 128 x 128 47 and 13; 512 of those 62 and
// 18; stores add 4 to 8).  A split contraction's parts are read again, at
// about 4 TB/s.
VocabPlan vocab_plan(int64_t m, int64_t n, int64_t stages, int most_splits)
{
    VocabPlan best = {64, 1};
    double least = 0.0;
    for (const int wave : {128, 64}) {
        const int64_t tiles = count(m, 2 * wave) * count(n, 2 * wave);
        const double stage = wave == 128 ? 1.5 : 0.9, alone = wave == 128 ? 1.5 : 0.72, besides = wave == 128 ? 12.0 : 6.0;
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
