// The losses over a large vocabulary: softmax cross entropy and the divergence
// from a teacher's top logits, forward and backward (include/fasgd_client.h).
//
// Rows that take part are gathered first, so that the others cost nothing and
// whatever they hold reaches no result.  Forward, the logits' product keeps
// statistics of its tiles alone (vocab_product.hip), which are joined here in
// order.  Backward, a piece of the vocabulary at a time: its logits again, their
// gradient dz as 16-bit terms in the workspace, then dz W, added up over the
// pieces, and dz^T x, whole for the piece's classes.
//
// The entries that a row is held to (its target, a teacher's classes) are the
// largest of dz, with p - q cancelling.  They are computed here from the
// picked logits, put into dz^T in place of what the tile wrote, and left out
// of dz: dx takes them in fp32, times the rows of W, at the end.
#include "tiles.hpp"
#include "vocab_rows.hpp"

namespace fasgd {
namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Pairs of three terms each, those above 2^-24, the smallest first.
constexpr uint32_t kPairsA = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;
constexpr uint32_t kPairsB = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10;

// ---- rows that take part

// used[r], a wave each; what a forward call says of rows that take no part.
__global__ __launch_bounds__(kBlock) void mark_rows(VocabArgs a, int32_t* used)
{
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (r >= a.rows) return;
    bool any = false;
    for (int k = lane; k < a.entries; k += 64) any |= counts(a, r * a.entries + k);
    any = __ballot(any) != 0;
    if (lane == 0) used[r] = any;
    if (any || !a.loss) return;
    if (lane == 0) a.loss[r] = a.lse[r] = 0.0f;
    for (int k = lane; k < a.entries; k += 64) a.picked[r * a.entries + k] = 0.0f;
}

// list: the rows that take part, in order; place: where in it a row is, or -1.
// used: NULL for targets, which are looked at here.
__global__ __launch_bounds__(1024) void gather_rows(VocabArgs a, const int32_t* used, int32_t* list, int32_t* place, int32_t* active,
                                                    uint32_t* largest)
{
    __shared__ int waves[16];
    __shared__ int base;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) {
        base = 0;
        *largest = 0;
    }
    for (int64_t at = 0; at < a.rows; at += 1024) {
        const int64_t r = at + threadIdx.x;
        const bool in = r < a.rows && (used ? used[r] != 0 : counts(a, r));
        if (!used && r < a.rows && !in && a.loss) a.loss[r] = a.lse[r] = a.picked[r] = 0.0f;
        const unsigned long long votes = __ballot(in);
        if (lane == 0) waves[wave] = __popcll(votes);
        __syncthreads();
        int before = base, all = base;
        for (int w = 0; w < 16; ++w) {
            before += w < wave ? waves[w] : 0;
            all += waves[w];
        }
        const int here = before + __popcll(votes & ((1ull << lane) - 1));
        if (in) list[here] = static_cast<int32_t>(r);
        if (r < a.rows) place[r] = in ? here : -1;
        __syncthreads();
        if (threadIdx.x == 0) base = all;
    }
    __syncthreads();
    if (threadIdx.x == 0) *active = base;
}

// ---- operands

// A matrix as the products read it: by_rows, rows of [terms][cols_padded], and /
// or by_cols, columns of [terms][rows_padded], zeros in the padding.  list: its
// rows are these of src (as many as `active` says), and what fills up the last
// tile are copies of the last of them.  With coefficients of 0 those weigh nothing
// in dW, and their logits are NaN only where that row's are; an infinite weight
// makes a row of zeros NaN, and with it dW of the class that it masks.
struct LayOut {
    const void* src;
    int64_t ld, rows, cols;
    const int32_t *list, *active;
    uint16_t *by_rows, *by_cols;
    int64_t cols_padded, ld_rows, rows_padded, ld_cols;
};

// fp32 in three bf16 terms: the first two cut off, so that none exceeds the
// value, the last rounded.  An infinite value is an infinite first term and finite
// ones of its sign.  A weight's meets all terms of an activation, of which none
// may be 0 then (`FILL`): a term has at least 2^-26 of 2^-100, or of the value
// where that is less, which adds no more than 2^-26 of a finite product.
template <int TERM, bool FILL> __device__ __forceinline__ uint16_t term_of(float x)
{
    if constexpr (TERM == 0) return static_cast<uint16_t>(__float_as_uint(__builtin_canonicalizef(x)) >> 16);   // NaN without its lower bits
    constexpr uint32_t kUpper = 0xffff0000u;
    const float finite = __builtin_amdgcn_fmed3f(x, -FLT_MAX, FLT_MAX);
    const float rest = finite - __uint_as_float(__float_as_uint(finite) & kUpper);
    const float second = __uint_as_float(__float_as_uint(rest) & kUpper);
    uint32_t term = TERM == 1 ? __float_as_uint(second) >> 16 : from_float<bf16>(rest - second).bits;
    if constexpr (FILL) {
        const float least = fminf(fabsf(x), 0x1p-100f) * 0x1p-26f, size = __uint_as_float((term & 0x7fffu) << 16);
        term = __float_as_uint(fmaxf(size, least)) >> 16 | (__float_as_uint(x) >> 16 & 0x8000u);
    }
    return static_cast<uint16_t>(term);
}

template <bool FILL> __device__ __forceinline__ uint16_t term_at(float x, int term)
{
    return term == 0 ? term_of<0, FILL>(x) : (term == 1 ? term_of<1, FILL>(x) : term_of<2, FILL>(x));
}

// 64 x 64 elements a wave, 8 x 8 a lane, turned in registers: each load and each
// store of a wave is whole lines of 8 rows or columns.  (131,072 x 4,096 bf16
// turned in pieces: 4.2 TB/s; through LDS 3.7.)
template <typename T, int TERMS, bool FILL> __global__ __launch_bounds__(kBlock, 2) void lay_out(LayOut a)
{
    const int64_t rows = a.active ? *a.active : a.rows;
    const int lane = threadIdx.x & 63;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * 64, c0 = (static_cast<int64_t>(blockIdx.y) * kWaves + (threadIdx.x >> 6)) * 64;
    if (r0 >= (rows + kVocabTile - 1) / kVocabTile * kVocabTile || c0 >= a.cols_padded) return;
    const int64_t r = r0 + (lane >> 3) * 8, c = c0 + (lane & 7) * 8;
    Pack<T, 8> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i].v[e] = from_float<T>(0.0f);
        if (rows > 0 && (a.list || r + i < rows)) {
            const T* src = static_cast<const T*>(a.src) + (a.list ? a.list[r + i < rows ? r + i : rows - 1] : r + i) * a.ld + c;
            if (c + 8 <= a.cols) {
                x[i] = load_pack<T, 8>(src);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < a.cols) x[i].v[e] = src[e];
            }
        }
    }
#pragma unroll
    for (int term = 0; term < TERMS; ++term) {
        uint32_t w[8][4];       // two columns a word
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (TERMS == 1) {
                __builtin_memcpy(w[i], &x[i], sizeof w[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    w[i][e / 2] = term_at<FILL>(x[i].v[e], term) | static_cast<uint32_t>(term_at<FILL>(x[i].v[e + 1], term)) << 16;
                }
            }
            if (a.by_rows) {
                Pack<uint32_t, 4> o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o.v[e] = w[i][e];
                store_pack(reinterpret_cast<uint32_t*>(a.by_rows + (r + i) * a.ld_rows + term * a.cols_padded + c), o);
            }
        }
        if (!a.by_cols) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            Pack<uint32_t, 4> o;
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                o.v[i / 2] = __builtin_amdgcn_perm(w[i + 1][e / 2], w[i][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            if (c + e < a.cols) store_pack(reinterpret_cast<uint32_t*>(a.by_cols + (c + e) * a.ld_cols + term * a.rows_padded + r), o);
        }
    }
}

// ---- forward

#if defined(__HIP_DEVICE_COMPILE__)
template <int TERM, int N> __device__ __forceinline__ void multiply_terms(const Pack<float, 8> (&v)[N], const v4i (&b)[N], v4f& acc)
{
#pragma unroll
    for (int s = 0; s < N; ++s) {
        Pack<uint16_t, 8> t;
#pragma unroll
        for (int e = 0; e < 8; ++e) t.v[e] = term_of<TERM, false>(v[s].v[e]);
        acc = mfma<bf16>(__builtin_bit_cast(v4i, t), b[s], acc);
    }
}
#endif

// The logits at a teacher's entries, 16 a wave: the diagonal of the product of their
// classes' rows and their rows of x, by the instruction and in the order of
// the tiles, so that they are bit for bit what the tiles put into the sums of
// powers.  (A row's largest logit is often its target: an error that the sum
// has and p's numerator has not, or another, is p (1 - p) of itself in dz, not p.
// 8,192 x 4,096 x 131,072 bf16, dW off by 3.9e-6 with a sum in another order.)
// Bound by W's rows and the chain of loads, 16 steps (of fp32 8) on their way (4,096
// rows of 64 entries, 4,096 columns bf16: 365 us, 5.9 TB/s; 1,531 rows of 50: 45 us).
template <typename T> __global__ __launch_bounds__(64, 2) void pick(VocabArgs a, const int32_t* list, const int32_t* active,
                                                                const uint16_t* x, int64_t ld_x, int64_t cols_padded)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool kTerms = sizeof(T) == 4;
    constexpr int kFlight = kTerms ? 8 : 16;        // steps of 32 on their way
    const int lane = threadIdx.x, part = lane >> 4;
    const int64_t all = static_cast<int64_t>(*active) * a.entries, blocks = (all + 15) / 16;
    for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        const int64_t pair = block * 16 + (lane & 15);
        const int64_t at = pair < all ? pair / a.entries : 0;
        const int64_t r = list[at], here = r * a.entries + (pair < all ? pair % a.entries : 0);
        const bool in = pair < all && counts(a, here);
        const T* w = static_cast<const T*>(a.w) + (in ? a.index[here] : 0) * a.ldw;
        const uint16_t* row = x + at * ld_x;
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < (kTerms ? 6 : 1); ++p) {
            const int ta = kTerms ? kPairsA >> (2 * p) & 3u : 0, tb = kTerms ? kPairsB >> (2 * p) & 3u : 0;
            const uint16_t* b = row + tb * cols_padded;
            for (int64_t k0 = 8 * part; k0 - 8 * part < a.cols; k0 += 32 * kFlight) {
                v4i fb[kFlight];
                Pack<T, 8> v[kFlight];
                if (k0 - 8 * part + 32 * kFlight <= a.cols) {
#pragma unroll
                    for (int s = 0; s < kFlight; ++s) {
                        v[s] = load_pack<T, 8>(w + k0 + 32 * s);
                        fb[s] = *reinterpret_cast<const v4i*>(b + k0 + 32 * s);
                    }
                } else {
#pragma unroll
                    for (int s = 0; s < kFlight; ++s) {
                        const int64_t k = k0 + 32 * s;
                        if (k + 8 <= a.cols) {
                            v[s] = load_pack<T, 8>(w + k);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[s].v[e] = k + e < a.cols ? w[k + e] : from_float<T>(0.0f);
                        }
                        fb[s] = k < cols_padded ? *reinterpret_cast<const v4i*>(b + k) : v4i{0, 0, 0, 0};
                    }
                }
                if constexpr (!kTerms) {
#pragma unroll
                    for (int s = 0; s < kFlight; ++s) acc = mfma<T>(__builtin_bit_cast(v4i, v[s]), fb[s], acc);
                } else if (ta == 0) {       // the same in all lanes
                    multiply_terms<0>(v, fb, acc);
                } else if (ta == 1) {
                    multiply_terms<1>(v, fb, acc);
                } else {
                    multiply_terms<2>(v, fb, acc);
                }
            }
        }
        // lane l: column l % 16, rows 4 (l / 16) + i
        float z = acc[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) z = (lane & 3) == i ? acc[i] : z;
        if ((lane & 15) >> 2 == part && pair < all) a.picked[here] = in ? z * a.scale : 0.0f;
    }
#endif
}

// ---- backward

// Coefficients of the rows that take part (a wave each, 16 a block), zeros beside
// the last one's log-sum-exp for the rows that fill up the last tile (copies of
// it); the largest coefficient, where asked for.
__global__ __launch_bounds__(1024) void coefficients(VocabArgs a, const int32_t* list, const int32_t* active, VocabRow* row,
                                                     float2* teacher, uint32_t* largest)
{
    __shared__ float most[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = *active;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 16 + wave;
    if (at - wave >= (n + kVocabTile - 1) / kVocabTile * kVocabTile) return;
    VocabRow c = {0.0f, 0.0f, 0.0f, 0.0f};
    Teacher t = {0.0f, 0.0f};
    if (at < n) {
        const int64_t r = list[at];
        t = teacher_of(a, r, lane);
        c = coefficients_of(a, r, t, lane);
    } else {
        c.l = a.lse[list[n - 1]] * kLog2e;
    }
    if (lane == 0) {
        row[at] = c;
        teacher[at] = make_float2(t.top, t.by);
        // A row that is not finite has no say in the others' scale.  (A sum of finite
        // parts may be infinity: term_scale takes it for a value below 2^130.)
        const float entry = fabsf(a.teacher ? c.f : c.g), f = fabsf(c.f), b = fabsf(c.b);
        most[wave] = entry <= FLT_MAX && f <= FLT_MAX && b <= FLT_MAX ? entry + f + b : 0.0f;
    }
    if (!largest) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        float x = most[0];
        for (int i = 1; i < 16; ++i) x = fmaxf(x, most[i]);
        atomicMax(largest, __float_as_uint(x));     // of values that are not negative: the same in any order
    }
}

struct Gradient {
    const VocabRow* row;
    const float2* teacher;
    const int32_t *list, *place, *active;
    const uint32_t* largest;
    uint16_t *dz, *dzt;
    int32_t dz_terms, dzt_terms;
    int64_t first, classes, padded, ld_dz, ld_dzt;
    int64_t count;          // classes of the piece
    const float* sums;      // [splits][padded][cols_padded]: dz W without the entries
    int32_t splits;
    int64_t cols_padded;
};

// The entries of a piece's classes: into dz^T, and out of dz.  A wave a row.  Bound
// by stores of 2 bytes, a line each (4,096 rows of 64 entries: 43 us a piece).
template <typename T> __global__ __launch_bounds__(kBlock) void place_entries(VocabArgs a, Gradient g)
{
    const int lane = threadIdx.x & 63;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (at >= *g.active) return;
    const int64_t r = g.list[at];
    const VocabRow row = g.row[at];
    const Teacher t = {g.teacher[at].x, g.teacher[at].y};
    const float up = term_scale<T>(*g.largest);
    for (int k = lane; k < a.entries; k += 64) {
        const int64_t i = a.index[r * a.entries + k] - g.first;
        float x;
        if (i < 0 || i >= g.count || !entry_gradient(a, row, t, r, k, &x)) continue;
        x *= up;
        for (int j = 0; j < g.dz_terms; ++j) g.dz[at * g.ld_dz + j * g.classes + i] = 0;
        for (int j = 0; j < g.dzt_terms; ++j) {
            const T term = from_float<T>(x);
            x -= to_float(term);
            g.dzt[i * g.ld_dzt + j * g.padded + at] = __builtin_bit_cast(uint16_t, term);
        }
    }
}

// dx of a row: the products' sums and the entries', times the logits' scale.  A
// block a row; bound by the entries' rows of W (4,096 rows of 64, 4,096 columns
// bf16: 2.1 GB in 430 us, 5 TB/s; 8,192 rows of one target 60 us).
template <typename T, typename TERM> __global__ __launch_bounds__(kBlock) void finish_dx(VocabArgs a, Gradient g)
{
    __shared__ float value[kMostEntries];
    __shared__ int64_t of[kMostEntries];
    __shared__ int entries;
    const int64_t r = blockIdx.x;
    const int32_t at = g.place[r];
    T* out = static_cast<T*>(a.dx) + r * a.lddx;
    if (at < 0) {
        for (int64_t c = threadIdx.x; c < a.cols; c += kBlock) out[c] = from_float<T>(0.0f);
        return;
    }
    if (threadIdx.x < 64) {     // the entries in order
        const int lane = threadIdx.x;
        const VocabRow row = g.row[at];
        const Teacher t = {g.teacher[at].x, g.teacher[at].y};
        int n = 0;
        for (int k0 = 0; k0 < a.entries; k0 += 64) {
            const int k = k0 + lane;
            float x = 0.0f;
            const bool in = k < a.entries && entry_gradient(a, row, t, r, k, &x);
            const unsigned long long votes = __ballot(in);
            if (in) {
                const int here = n + __popcll(votes & ((1ull << lane) - 1));
                value[here] = x;
                of[here] = a.index[r * a.entries + k] * a.ldw;
            }
            n += __popcll(votes);
        }
        if (lane == 0) entries = n;
    }
    __syncthreads();
    const int n = entries;
    const float by = a.scale / row_scale<TERM>(g.row[at], term_scale<TERM>(*g.largest));
    const T* w = static_cast<const T*>(a.w);
    for (int64_t c = threadIdx.x * 4; c < a.cols; c += kBlock * 4) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f}, own[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < g.splits; ++s) {
            const Pack<float, 4> p = load_pack<float, 4>(g.sums + (s * g.padded + at) * g.cols_padded + c);
            for (int e = 0; e < 4; ++e) sum[e] += p.v[e];
        }
        if (c + 4 <= a.cols) {
#pragma unroll 4
            for (int k = 0; k < n; ++k) {
                const Pack<T, 4> p = load_pack<T, 4>(w + of[k] + c);
                for (int e = 0; e < 4; ++e) own[e] = __builtin_fmaf(value[k], to_float(p.v[e]), own[e]);
            }
        } else {
            for (int k = 0; k < n; ++k)
                for (int e = 0; e < 4 && c + e < a.cols; ++e) own[e] = __builtin_fmaf(value[k], to_float(w[of[k] + c + e]), own[e]);
        }
        for (int e = 0; e < 4 && c + e < a.cols; ++e) out[c + e] = from_float<T>(__builtin_fmaf(sum[e], by, own[e] * a.scale));
    }
}

// dW of no rows.
template <typename T> __global__ __launch_bounds__(kBlock) void clear(T* c, int64_t ld, int64_t rows, int64_t cols)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t i = threadIdx.x; i < cols; i += kBlock) c[r * ld + i] = from_float<T>(0.0f);
}

// ---- the host's side

// Where things lie in the workspace, in bytes.
struct Layout {
    int terms;
    int64_t padded, cols_padded, piece, pieces, slots;
    int64_t ld_cols, ld_rows, ld_piece;     // values between rows of terms along the columns, the rows, a piece's classes
    VocabPlan logits, dx, dw;
    int64_t used, list, place, scalars, row, teacher, x, xt, w, wt, dz, dzt, sums, partial, partial_sum, bytes;
};

// Bytes of a piece's gradient, and its part of W: pieces are large enough to
// fill the chip with tiles several times over, small beside the card's memory.
constexpr int64_t kPieceBytes = int64_t(1) << 30;

// Values between rows of n: an odd number of 512 bytes, so that the rows of a
// tile, which are read together, spread over L2's channels (8,192 x 4,096 x
// 16,384: rows 32 KB apart 855 us, 512 bytes more 822, 256 more 957).
int64_t apart(int64_t n) { return ((n + 255) / 256 | 1) * 256; }

// Terms of dz that dW is summed from.  For an fp32 one two of fp16 (22 bits) or
// three of bf16 (24): with two, 16 bits, dW is off by 1.7 to 2.7e-6 (relative, root
// mean square) where fp32 sums of 4,096 to 8,192 rows, of the values themselves, are
// off by 1.0 to 2.5e-6; with three by 0.5 to 1.2e-6.  (A training step of 8,192 x 4,096
// x 131,072 takes 38.9 ms with three and 33.0 with two, of 8,192 x 1,024 x 32,000 3.3 and
// 2.9, of 4,096 x 2,048 x 16,384 1.58 and 1.36.)  For a dw of 16 bits one: its rounding
// comes on top of dW's own, which is of the same size (fp16, 1,777 x 1,544 x 32,003:
// 3.2e-4 off, with two terms 2.5e-4, all of it dW's; bf16 2.3e-3 and 1.7e-3), and the
// training step takes 803 instead of 937 us.
int terms_for_dw(int dtype, int dw_dtype)
{
    if (dtype == DTYPE_F32) return 3;
    if (dw_dtype != DTYPE_F32) return 1;
    return dtype == DTYPE_BF16 ? 3 : 2;
}

Layout layout_of(int64_t rows, int64_t cols, int64_t vocab, int dtype, bool backward)
{
    Layout l = {};
    l.terms = vocab_terms(dtype);
    l.padded = round_up(rows, kVocabTile);
    l.cols_padded = round_up(cols, 128);
    const int dzt_terms = terms_for_dw(dtype, DTYPE_F32);
    // (bf16's third term comes on top: shorter pieces would leave more of the chip idle)
    const int64_t each = 2 * (l.padded * (l.terms == 3 ? 6 : 3) + 2 * l.cols_padded * l.terms);
    int64_t most = kPieceBytes / each / kVocabTile * kVocabTile;
    if (most < 2048) most = 2048;
    if (most > int64_t(1) << 20) most = int64_t(1) << 20;
    l.pieces = (vocab + most - 1) / most;
    l.piece = round_up((vocab + l.pieces - 1) / l.pieces, kVocabTile);
    l.pieces = (vocab + l.piece - 1) / l.piece;
    const int64_t pairs = l.terms == 3 ? 6 : 1;
    l.logits = vocab_plan(l.piece, rows, l.cols_padded / 64 * pairs, 1);
    l.dx = vocab_plan(rows, cols, l.piece / 64 * pairs, kVocabSplits);
    l.dw = vocab_plan(l.piece, cols, l.padded / 64 * (l.terms == 3 ? 6 : dzt_terms), 1);
    l.slots = (vocab + l.logits.wave - 1) / l.logits.wave;
    l.ld_cols = apart(l.terms * l.cols_padded);
    l.ld_rows = apart(l.terms * l.padded);
    l.ld_piece = apart(l.terms * l.piece);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = round_up(at + bytes, 256);
        return here;
    };
    l.used = take(4 * rows);
    l.list = take(4 * rows);
    l.place = take(4 * rows);
    l.scalars = take(256);      // rows that take part; the largest coefficient
    l.x = take(2 * l.padded * l.ld_cols);
    l.w = take(2 * l.piece * l.ld_cols);
    if (backward) {
        l.row = take(sizeof(VocabRow) * l.padded);
        l.teacher = take(sizeof(float2) * l.padded);
        l.xt = take(2 * cols * l.ld_rows);
        l.wt = take(2 * cols * l.ld_piece);
        l.dz = take(2 * l.padded * l.ld_piece);
        l.dzt = take(2 * l.piece * apart(dzt_terms * l.padded));
        l.sums = take(4 * l.dx.splits * l.padded * l.cols_padded);
    } else {
        l.partial = take(8 * l.slots * l.padded);
        l.partial_sum = take(4 * l.slots * l.padded);
    }
    l.bytes = at;
    return l;
}

// Whether the products can read W where it lies.
bool in_place(const VocabArgs& a)
{
    return a.dtype != DTYPE_F32 && a.cols % 8 == 0 && a.ldw % 8 == 0 && a.ldw <= (int64_t(1) << 21) &&
           (reinterpret_cast<uintptr_t>(a.w) & 15) == 0;
}

hipError_t launch_lay_out(const LayOut& l, int dtype, int64_t rows, int64_t cols, hipStream_t s)
{
    const dim3 grid(static_cast<unsigned>(round_up(rows, kVocabTile) / 64), static_cast<unsigned>(round_up(cols, 256) / 256));
    if (dtype == DTYPE_F32 && l.list) lay_out<float, 3, true><<<grid, kBlock, 0, s>>>(l);
    else if (dtype == DTYPE_F32) lay_out<float, 3, false><<<grid, kBlock, 0, s>>>(l);
    else lay_out<bf16, 1, false><<<grid, kBlock, 0, s>>>(l);       // bits of either 16-bit type
    return hipGetLastError();
}

struct Plan {
    Layout l;
    int32_t *used, *list, *place, *active;
    uint32_t* largest;
    uint8_t* base;
    bool w_in_place;
    template <typename T> T* at(int64_t offset) const { return reinterpret_cast<T*>(base + offset); }
};

// Rows that take part, and x as an operand (backward: transposed too).
hipError_t begin(const VocabArgs& a, bool backward, Plan& p, hipStream_t s)
{
    p.l = layout_of(a.rows, a.cols, a.vocab, a.dtype, backward);
    p.base = static_cast<uint8_t*>(a.workspace);
    p.used = p.at<int32_t>(p.l.used);
    p.list = p.at<int32_t>(p.l.list);
    p.place = p.at<int32_t>(p.l.place);
    p.active = p.at<int32_t>(p.l.scalars);
    p.largest = p.at<uint32_t>(p.l.scalars + 4);
    p.w_in_place = in_place(a);
    const bool entries = a.entries > 1;
    if (entries) {
        mark_rows<<<static_cast<unsigned>((a.rows + kWaves - 1) / kWaves), kBlock, 0, s>>>(a, p.used);
        VOCAB_TRY(hipGetLastError());
    }
    gather_rows<<<1, 1024, 0, s>>>(a, entries ? p.used : nullptr, p.list, p.place, p.active, p.largest);
    VOCAB_TRY(hipGetLastError());
    LayOut x = {};
    x.src = a.x;
    x.ld = a.ldx;
    x.rows = a.rows;
    x.cols = a.cols;
    x.list = p.list;
    x.active = p.active;
    x.by_rows = p.at<uint16_t>(p.l.x);
    x.by_cols = backward && a.dw ? p.at<uint16_t>(p.l.xt) : nullptr;
    x.cols_padded = p.l.cols_padded;
    x.ld_rows = p.l.ld_cols;
    x.rows_padded = p.l.padded;
    x.ld_cols = p.l.ld_rows;
    return launch_lay_out(x, a.dtype, a.rows, a.cols, s);
}

// The logits of classes first .. first + n - 1: W as an operand where it cannot
// be read in place (and transposed, for dx), and the product's two sides.
hipError_t piece_of(const VocabArgs& a, const Plan& p, int64_t first, int64_t n, bool transposed, VocabProduct& q, hipStream_t s)
{
    const Layout& l = p.l;
    const int64_t size = static_cast<int64_t>(dtype_size(a.dtype));
    const uint8_t* w = static_cast<const uint8_t*>(a.w) + first * a.ldw * size;
    if (!p.w_in_place || transposed) {
        LayOut o = {};
        o.src = w;
        o.ld = a.ldw;
        o.rows = n;
        o.cols = a.cols;
        o.by_rows = p.w_in_place ? nullptr : p.at<uint16_t>(l.w);
        o.by_cols = transposed ? p.at<uint16_t>(l.wt) : nullptr;
        o.cols_padded = l.cols_padded;
        o.ld_rows = l.ld_cols;
        o.rows_padded = l.piece;
        o.ld_cols = l.ld_piece;
        VOCAB_TRY(launch_lay_out(o, a.dtype, n, a.cols, s));
    }
    q = VocabProduct{};
    q.a.data = p.w_in_place ? w : p.at<uint8_t>(l.w);
    q.a.ld = p.w_in_place ? a.ldw * size : 2 * l.ld_cols;
    q.a.rows = static_cast<int32_t>(n);
    q.a_bytes = p.w_in_place && a.cols % 128 != 0 ? static_cast<int32_t>(a.cols * size) : 0;
    q.a.plane = q.b.plane = static_cast<int32_t>(2 * l.cols_padded);
    q.b.data = p.at<uint8_t>(l.x);
    q.b.ld = 2 * l.ld_cols;
    q.active = p.active;
    q.rows_b_active = 1;
    q.blocks = static_cast<int32_t>(l.cols_padded / 64);
    q.terms = l.terms == 3 ? 6 : 1;
    q.terms_a = l.terms == 3 ? kPairsA : 0;
    q.terms_b = l.terms == 3 ? kPairsB : 0;
    q.splits = 1;
    q.f16 = a.dtype == DTYPE_F16;
    q.scale_log2e = a.scale * kLog2e;
    q.first = first;
    q.padded = l.padded;
    return hipSuccess;
}

}  // namespace

size_t vocab_workspace_bytes(int64_t rows, int64_t cols, int64_t vocab, int dtype, bool backward)
{
    if (vocab_direct(rows, cols, vocab, dtype)) return vocab_direct_bytes(rows, cols, vocab, backward);
    return static_cast<size_t>(layout_of(rows, cols, vocab, dtype, backward).bytes);
}

hipError_t launch_vocab_forward(const VocabArgs& a, hipStream_t s)
{
    if (vocab_direct(a.rows, a.cols, a.vocab, a.dtype)) return launch_vocab_direct_forward(a, s);
    Plan p;
    VOCAB_TRY(begin(a, false, p, s));
    const Layout& l = p.l;
    for (int64_t first = 0; first < a.vocab; first += l.piece) {
        const int64_t n = a.vocab - first < l.piece ? a.vocab - first : l.piece;
        VocabProduct q;
        VOCAB_TRY(piece_of(a, p, first, n, false, q, s));
        q.wave = l.logits.wave;
        q.partial = p.at<float2>(l.partial);
        q.partial_sum = a.smoothing != 0.0f ? p.at<float>(l.partial_sum) : nullptr;
        if (!a.teacher) {
            q.list = p.list;
            q.target = a.index;
            q.picked = a.picked;
            q.by = a.scale;
        }
        VOCAB_TRY(launch_vocab_product(VOCAB_STATISTICS, q, n, a.rows, s));
    }
    if (a.teacher) {
        const int64_t blocks = (a.rows * a.entries + 15) / 16;
        const unsigned picks = static_cast<unsigned>(blocks < (1 << 20) ? blocks : 1 << 20);
        const uint16_t* x = p.at<uint16_t>(l.x);
        if (a.dtype == DTYPE_F32) pick<float><<<picks, 64, 0, s>>>(a, p.list, p.active, x, l.ld_cols, l.cols_padded);
        else if (a.dtype == DTYPE_BF16) pick<bf16><<<picks, 64, 0, s>>>(a, p.list, p.active, x, l.ld_cols, l.cols_padded);
        else pick<f16><<<picks, 64, 0, s>>>(a, p.list, p.active, x, l.ld_cols, l.cols_padded);
        VOCAB_TRY(hipGetLastError());
    }
    finish<<<static_cast<unsigned>((a.rows + 7) / 8), kBlock, 0, s>>>(a, p.list, p.active, p.at<float2>(l.partial),
                                                                      a.smoothing != 0.0f ? p.at<float>(l.partial_sum) : nullptr,
                                                                      l.slots, l.padded);
    return hipGetLastError();
}

hipError_t launch_vocab_backward(const VocabArgs& a, hipStream_t s)
{
    if (a.rows == 0) {
        if (!a.dw || a.accumulate) return hipSuccess;
        const unsigned blocks = static_cast<unsigned>(a.vocab < (1 << 16) ? a.vocab : 1 << 16);
        if (a.dw_dtype == DTYPE_F32) clear<float><<<blocks, kBlock, 0, s>>>(static_cast<float*>(a.dw), a.lddw, a.vocab, a.cols);
        else clear<bf16><<<blocks, kBlock, 0, s>>>(static_cast<bf16*>(a.dw), a.lddw, a.vocab, a.cols);
        return hipGetLastError();
    }
    if (vocab_direct(a.rows, a.cols, a.vocab, a.dtype)) return launch_vocab_direct_backward(a, s);
    Plan p;
    VOCAB_TRY(begin(a, true, p, s));
    const Layout& l = p.l;
    Gradient g = {};
    g.row = p.at<VocabRow>(l.row);
    g.teacher = p.at<float2>(l.teacher);
    g.list = p.list;
    g.place = p.place;
    g.active = p.active;
    g.largest = p.largest;
    g.dz = p.at<uint16_t>(l.dz);
    g.dzt = p.at<uint16_t>(l.dzt);
    g.dz_terms = a.dx ? l.terms : 0;
    g.dzt_terms = a.dw ? terms_for_dw(a.dtype, a.dw_dtype) : 0;
    g.classes = l.piece;
    g.padded = l.padded;
    g.ld_dz = l.ld_piece;
    g.ld_dzt = apart(g.dzt_terms * l.padded);
    g.sums = p.at<float>(l.sums);
    g.splits = l.dx.splits;
    g.cols_padded = l.cols_padded;
    const unsigned row_waves = static_cast<unsigned>((l.padded + kWaves - 1) / kWaves);
    coefficients<<<static_cast<unsigned>(l.padded / 16), 1024, 0, s>>>(a, p.list, p.active, p.at<VocabRow>(l.row), p.at<float2>(l.teacher),
                                                                      a.dtype == DTYPE_F16 ? p.largest : nullptr);
    VOCAB_TRY(hipGetLastError());
    for (int64_t first = 0; first < a.vocab; first += l.piece) {
        const int64_t n = a.vocab - first < l.piece ? a.vocab - first : l.piece;
        VocabProduct q;
        VOCAB_TRY(piece_of(a, p, first, n, a.dx != nullptr, q, s));
        q.wave = l.logits.wave;
        q.row = g.row;
        q.largest = p.largest;
        q.dz = g.dz;
        q.dzt = g.dzt;
        q.dz_terms = g.dz_terms;
        q.dzt_terms = g.dzt_terms;
        q.classes = g.classes;
        q.ld_dz = g.ld_dz;
        q.ld_dzt = g.ld_dzt;
        VOCAB_TRY(launch_vocab_product(VOCAB_GRADIENT, q, n, a.rows, s));
        g.first = first;
        g.count = n;
        if (a.dtype == DTYPE_F16) place_entries<f16><<<row_waves, kBlock, 0, s>>>(a, g);
        else place_entries<bf16><<<row_waves, kBlock, 0, s>>>(a, g);
        VOCAB_TRY(hipGetLastError());
        VocabProduct c = {};
        c.active = p.active;
        c.f16 = q.f16;
        c.largest = p.largest;
        if (a.dx) {
            c.a = VocabOperand{p.at<uint8_t>(l.dz), 2 * l.ld_piece, 0, static_cast<int32_t>(2 * l.piece)};
            c.b = VocabOperand{p.at<uint8_t>(l.wt), 2 * l.ld_piece, static_cast<int32_t>(a.cols), static_cast<int32_t>(2 * l.piece)};
            c.rows_a_active = 1;
            c.blocks = static_cast<int32_t>(round_up(n, 128) / 64);
            c.terms = q.terms;
            c.terms_a = q.terms_a;
            c.terms_b = q.terms_b;
            c.wave = l.dx.wave;
            c.splits = l.dx.splits;
            c.c = p.at<float>(l.sums);
            c.ldc = l.cols_padded;
            c.split_stride = l.padded * l.cols_padded;
            c.c_dtype = DTYPE_F32;
            c.add = first > 0;
            c.by = 1.0f;
            c.largest = nullptr;
            VOCAB_TRY(launch_vocab_product(VOCAB_STORE, c, a.rows, a.cols, s));
        }
        if (a.dw) {
            c.a = VocabOperand{p.at<uint8_t>(l.dzt), 2 * g.ld_dzt, static_cast<int32_t>(n), static_cast<int32_t>(2 * l.padded)};
            c.b = VocabOperand{p.at<uint8_t>(l.xt), 2 * l.ld_rows, static_cast<int32_t>(a.cols), static_cast<int32_t>(2 * l.padded)};
            c.rows_a_active = 0;
            c.k_active = 1;
            c.blocks = static_cast<int32_t>(l.padded / 64);
            c.terms = l.terms == 3 ? 6 : g.dzt_terms;
            c.terms_a = l.terms == 3 ? kPairsA : (g.dzt_terms == 3 ? 6 : g.dzt_terms - 1);     // dz's smallest term first
            c.terms_b = l.terms == 3 ? kPairsB : 0;
            c.wave = l.dw.wave;
            c.splits = 1;
            c.c = static_cast<uint8_t*>(a.dw) + first * a.lddw * static_cast<int64_t>(dtype_size(a.dw_dtype));
            c.ldc = a.lddw;
            c.c_dtype = a.dw_dtype;
            c.add = a.accumulate;
            c.by = a.scale;
            c.largest = p.largest;
            VOCAB_TRY(launch_vocab_product(VOCAB_STORE, c, n, a.cols, s));
        }
    }
    if (a.dx) {
        const unsigned rows = static_cast<unsigned>(a.rows);
        if (a.dtype == DTYPE_F32) finish_dx<float, bf16><<<rows, kBlock, 0, s>>>(a, g);
        else if (a.dtype == DTYPE_BF16) finish_dx<bf16, bf16><<<rows, kBlock, 0, s>>>(a, g);
        else finish_dx<f16, f16><<<rows, kBlock, 0, s>>>(a, g);
        VOCAB_TRY(hipGetLastError());
    }
    return hipSuccess;
}

}  // namespace fasgd
