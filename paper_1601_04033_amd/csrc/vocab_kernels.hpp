// Launchers of the losses over a large vocabulary (include/fasgd_client.h),
// called by the C ABI after it has validated every argument.
#pragma once

#include <float.h>

#include "client_kernels.hpp"

namespace fasgd {

constexpr int kMostEntries = 1024;      // a row's entries of a teacher

// Matrices that products read, in 16-bit terms: a 16-bit type as it is, fp32
// as the sum of three bf16 terms (24 bits).
constexpr int vocab_terms(int dtype) { return dtype == DTYPE_F32 ? 3 : 1; }

struct VocabArgs {
    int64_t rows, cols, vocab;
    int32_t dtype;
    float scale;            // of the logits, > 0
    const void *x, *w;
    int64_t ldx, ldw;
    // what the rows are held to: targets (teacher NULL), or K entries with the teacher's logits
    const int64_t* index;   // [rows] or [rows][entries]
    const void* teacher;    // [rows][entries] of dtype
    const float* teacher_lse;
    int32_t entries;        // 1 for targets
    float teacher_scale;
    float smoothing, z_loss;
    float *loss, *lse, *picked;     // fp32 [rows], [rows], [rows][entries]; the last two are read by the backward pass
    // backward
    const float* dloss;     // fp32 [rows], NULL: ones
    float grad_scale;
    void *dx, *dw;          // NULL: not wanted
    int64_t lddx, lddw;
    int32_t dw_dtype;       // DTYPE_F32 or dtype
    int32_t accumulate;     // dw is added to
    void* workspace;
};

size_t vocab_workspace_bytes(int64_t rows, int64_t cols, int64_t vocab, int dtype, bool backward);
hipError_t launch_vocab_forward(const VocabArgs& a, hipStream_t s);
hipError_t launch_vocab_backward(const VocabArgs& a, hipStream_t s);

// Few rows, and small problems, without operands laid out (vocab_direct.hip).
bool vocab_direct(int64_t rows, int64_t cols, int64_t vocab, int dtype);
size_t vocab_direct_bytes(int64_t rows, int64_t cols, int64_t vocab, bool backward);
hipError_t launch_vocab_direct_forward(const VocabArgs& a, hipStream_t s);
hipError_t launch_vocab_direct_backward(const VocabArgs& a, hipStream_t s);

// ---- the products (vocab_product.hip)

// An operand: rows of 16-bit terms, each term's values along the contraction
// padded with zeros to a multiple of 128, terms `plane` bytes apart in a row.
struct VocabOperand {
    const uint8_t* data;    // 16-byte aligned
    int64_t ld;             // bytes between rows, a multiple of 16
    int32_t rows;           // a row past the last is read as the last
    int32_t plane;
};

// Per row of the backward pass: dz = f exp2(z scale log2(e) - l) - b, less g
// times the weight q of an entry there.
struct VocabRow {
    float l, f, b, g;
};

// What the host knows before the launch stands here; how many rows take part
// is known on the device (`active`), and blocks beyond that end at once.
enum : int { VOCAB_STATISTICS, VOCAB_GRADIENT, VOCAB_STORE };
struct VocabProduct {
    VocabOperand a, b;
    int32_t a_bytes;        // of a row of a that are to be read (a multiple of 16), zeros from there on; 0: all
    const int32_t* active;
    int32_t rows_a_active, rows_b_active;   // the operand's rows are the rows that take part
    int32_t k_active;       // the contraction is over the rows that take part
    int32_t blocks;         // of 64 along the contraction, an even number (k_active: at most)
    int32_t terms;          // products of terms: how many, and which (2 bits each, the first lowest)
    uint32_t terms_a, terms_b;
    int32_t splits;         // of the contraction (VOCAB_STORE)
    int32_t f16;            // terms are fp16's, else bf16's
    int32_t wave;           // side of a wave's tile, 128 or 64
    float scale_log2e;
    // VOCAB_STATISTICS, a: the vocabulary from class `first` on, b: rows.  For the classes of each
    // wave's tile (a slot): largest exponent and sum of powers; sum of logits; `by` times the logits
    // at the rows' targets (of row list[i] for b's row i).
    float2* partial;        // [slots][padded]
    float* partial_sum;     // [slots][padded], or NULL
    int64_t first, padded;
    const int32_t* list;
    const int64_t* target;  // NULL: not wanted
    float* picked;
    // VOCAB_GRADIENT, same operands
    const VocabRow* row;    // [padded]
    const uint32_t* largest;        // of the rows' coefficients, as bits (fp16 terms of dz^T are scaled by it)
    uint16_t *dz, *dzt;     // rows of [dz_terms][classes] and of [dzt_terms][padded], ld_dz and ld_dzt values apart
    int64_t ld_dz, ld_dzt;
    int32_t dz_terms, dzt_terms;    // 0: not wanted
    int64_t classes;        // padded to 256
    // VOCAB_STORE: c[split] (+)= by a b^T, by divided by the gradient's scale
    void* c;
    int64_t ldc, split_stride;
    int32_t c_dtype, add;
    float by;
};

constexpr int64_t kVocabTile = 256;     // classes and rows are padded to this
// How an m x n product over `stages` of 64 (times the pairs of terms) goes:
// side of a wave's tile (128: blocks of 256 x 256; or 64), parts of the contraction.
struct VocabPlan {
    int wave, splits;
};
constexpr int kVocabSplits = 16;
VocabPlan vocab_plan(int64_t m, int64_t n, int64_t stages, int most_splits);
hipError_t launch_vocab_product(int what, const VocabProduct& p, int64_t m, int64_t n, hipStream_t s);

// What a gradient's terms are multiplied by: 1 in bf16; in fp16, whose range
// is short, the power of two that takes the largest coefficient to 2^14 (infinity
// is a sum beyond fp32's range, below 2^130).  dW sums over the rows, so that
// is the largest of all rows.
template <typename T> __device__ __forceinline__ float term_scale(uint32_t largest);
template <> __device__ __forceinline__ float term_scale<bf16>(uint32_t) { return 1.0f; }
template <> __device__ __forceinline__ float term_scale<f16>(uint32_t largest)
{
    const int e = static_cast<int>(largest >> 23);
    if (e == 0) return 1.0f;
    const int up = 127 + 14 - (e - 127);
    return __uint_as_float(static_cast<uint32_t>(up < 1 ? 1 : (up > 254 ? 254 : up)) << 23);
}

// A row of dx is its own affair: where its coefficients are far below the largest,
// they are taken to 2^14 by themselves.  Rows of much the same size share `up`, the
// scale of all, and their terms with dz^T.
template <typename T> __device__ __forceinline__ float row_scale(const VocabRow& row, float up)
{
    const float own = term_scale<T>(__float_as_uint(fabsf(row.f) + fabsf(row.b)));
    return own <= 8.0f * up || fabsf(row.f) + fabsf(row.b) < FLT_MIN ? up : own;
}
template <> __device__ __forceinline__ float row_scale<bf16>(const VocabRow&, float) { return 1.0f; }

}  // namespace fasgd
