// Launchers of the client's kernels, called by the C ABI after it has
// validated every argument.  Each returns the HIP launch status.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "client_math.hpp"

namespace fasgd {

enum : int { DTYPE_F32 = 0, DTYPE_BF16 = 1, DTYPE_F16 = 2 };
constexpr size_t dtype_size(int dtype) { return dtype == DTYPE_F32 ? 4 : 2; }

struct DropoutArgs {
    const void* x;
    const void* residual;   // NULL: none
    void* y;
    int64_t ldx, ldr, ldy;
    int64_t rows, cols;
    int64_t first;          // element that a launch begins at
    DropKey key;
};
// A launch may have fewer than 2^32 threads: larger work goes in several.
constexpr int64_t kLaunchBlocks = int64_t(1) << 23;
hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s);

enum : int { GATE_NONE = 0, GATE_CHANNEL = 1, GATE_ROW = 2, GATE_FULL = 3 };
enum : int { ACT_IDENTITY = 0, ACT_SIGMOID = 1, ACT_TANH = 2 };

// The residual norm (include/fasgd_client.h), forward and backward.
struct NormArgs {
    int64_t rows;
    int32_t cols;
    float n_cols, inv_cols; // cols, 1 / cols
    int32_t layer;          // layer norm (mean subtracted), else rms
    int32_t gate_form, gate_act;
    int32_t drop;           // 0: no dropout
    float rho, eps;
    const float *w_post, *b_post, *w_pre, *b_pre;
    const void* gate;       // channel, row: fp32; full: activations
    const void *branch, *residual;
    void* sum;              // read in the backward pass
    void* normed;
    float* stats;           // [rows][4]: mean, rstd of the branch; mean, rstd of the sum
    int64_t ld_branch, ld_residual, ld_gate, ld_sum, ld_normed;
    DropKey key;
    // backward
    const void *dsum, *dnormed;
    void *dbranch, *dresidual;
    void* dgate;
    int64_t ld_dsum, ld_dnormed, ld_dbranch, ld_dresidual, ld_dgate;
    float *dw_post, *db_post, *dw_pre, *db_pre;
    float* partial;         // [4][blocks][cols]
};
hipError_t launch_norm_forward(const NormArgs& a, int dtype, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, int dtype, hipStream_t s);
// Workspace of the backward pass's column sums.
size_t norm_workspace_bytes(int64_t rows, int64_t cols);


// ---- 8-bit operands (include/fasgd_client.h)

constexpr int kFp8Block = 128;      // contraction length under one scale
enum : int { FP8_E4M3 = 0, FP8_E5M2 = 1 };

struct Fp8View {
    uint8_t* data;          // [rows][ld], ld a multiple of 128
    uint8_t* scales;        // [ceil(k / 128)][lds]
    int64_t rows, k, ld, lds;
    int32_t format;
};

// x quantized into `row` (x's rows, blocks along its columns) and / or `col`
// (x's columns, blocks along its rows); data NULL: not wanted.  whole: one
// scale per 128 x 128 tile.
struct QuantizeArgs {
    const void* x;
    int64_t ldx, rows, cols;
    Fp8View row, col;
    int64_t first;          // block that a launch begins at (rows alone)
    int32_t whole;
};
hipError_t launch_quantize(const QuantizeArgs& a, int dtype, hipStream_t s);

// c[m][n] (+)= sum_k a[m][k] b[n][k]
struct Fp8Product {
    Fp8View a, b;
    void* c;
    int64_t ldc;
    int32_t c_dtype;
    int32_t accumulate;
    int32_t short_sums;     // 16-bit c: each 8 products to 2^-13 of the largest
    float* partial;         // [splits][m][n], unused with one split
};
// Products that read their operands straight into registers: launch_fp8_few,
// where fp8_few says so.  launch_fp8_linear_few takes q.a's rows from x and
// quantizes them on the way, where fp8_linear_few says that they fit.
constexpr int64_t kFewRows = 64;
bool fp8_few(int64_t m, int64_t n, int64_t k);
bool fp8_linear_few(int64_t m, int64_t k);
int fp8_few_splits(int64_t m, int64_t n, int64_t k);     // of a product that fp8_few takes
hipError_t launch_fp8_few(const Fp8Product& p, hipStream_t s);
hipError_t launch_fp8_linear_few(const void* x, int64_t ldx, const Fp8Product& q, hipStream_t s);
size_t fp8_workspace_bytes(int64_t m, int64_t n, int64_t k);
hipError_t launch_fp8_product(const Fp8Product& p, hipStream_t s);
// c from the splits' products in the workspace, added in order.
hipError_t launch_fp8_join(const Fp8Product& p, int splits, hipStream_t s);

}  // namespace fasgd
