// C ABI of the client's operators (declared in include/fasgd_client.h):
// host-side argument checks and kernel dispatch.
#include <math.h>
#include <string.h>

#include "../../include/fasgd_client.h"
#include "client_kernels.hpp"
#include "status.hpp"

static_assert(CLIENT_F32 == fasgd::DTYPE_F32 && CLIENT_BF16 == fasgd::DTYPE_BF16 && CLIENT_F16 == fasgd::DTYPE_F16,
              "dtype mismatch");

namespace {

using fasgd::aligned;
using fasgd::fail;
using fasgd::hip_fail;
using fasgd::ok;

#define FASGD_TRY(call)                          \
    do {                                         \
        const fasgd_status try_status = (call);  \
        if (try_status != FASGD_OK) return try_status; \
    } while (0)

constexpr int64_t kMaxElements = int64_t(1) << 40;     // of one matrix: every launch and index stays in range

fasgd_status check_shape(int64_t rows, int64_t cols, int32_t dtype)
{
    if (dtype != CLIENT_F32 && dtype != CLIENT_BF16 && dtype != CLIENT_F16)
        return fail(FASGD_ERR_ARG, "dtype = %d is not a client_dtype value", dtype);
    if (rows < 0 || cols < 0) return fail(FASGD_ERR_ARG, "rows = %lld and cols = %lld must be >= 0", (long long)rows, (long long)cols);
    if (rows > kMaxElements || cols > kMaxElements || (cols > 0 && rows > kMaxElements / cols))
        return fail(FASGD_ERR_ARG, "rows x cols = %lld x %lld exceeds 2^40", (long long)rows, (long long)cols);
    return FASGD_OK;
}

// One matrix of a call: a pointer its type aligns, rows at least cols apart
// (the stride of a single row is not used).
fasgd_status check_matrix(const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype)
{
    if (!p) return fail(FASGD_ERR_NULL, "%s is NULL", name);
    if (!aligned(p, fasgd::dtype_size(dtype)))
        return fail(FASGD_ERR_ALIGN, "%s is not %zu-byte aligned", name, fasgd::dtype_size(dtype));
    if (rows > 1 && (ld < cols || ld > kMaxElements / rows))
        return fail(FASGD_ERR_ARG, "%s: row stride %lld is not in [cols = %lld, 2^40 / rows]", name, (long long)ld,
                    (long long)cols);
    return FASGD_OK;
}

// Key of a dropout over n elements (include/fasgd_client.h).
fasgd_status drop_key(double p, uint64_t seed, int64_t T, int32_t client, int32_t site, int64_t index_base, int64_t n,
                      fasgd::DropKey& k)
{
    if (!(p >= 0.0 && p <= 1.0)) return fail(FASGD_ERR_ARG, "p must be in [0, 1]");
    if (T < 0 || T > int64_t(UINT32_MAX)) return fail(FASGD_ERR_ARG, "T = %lld is not in [0, 2^32)", (long long)T);
    if (client < 0) return fail(FASGD_ERR_CLIENT, "client = %d must be >= 0", client);
    if (site < 0 || site >= 16384) return fail(FASGD_ERR_ARG, "site = %d is not in [0, 16384)", site);
    if (index_base < 0 || (index_base & 7) != 0 || index_base > (int64_t(1) << 51) - n)
        return fail(FASGD_ERR_ARG, "index_base = %lld must be a multiple of 8 in [0, 2^51 - rows x cols]",
                    (long long)index_base);
    k.key0 = static_cast<uint32_t>(seed);
    k.key1 = static_cast<uint32_t>(seed >> 32);
    k.ctr1 = 0x40000000u | static_cast<uint32_t>(site) << 16;
    k.ctr_T = static_cast<uint32_t>(T);
    k.ctr_client = static_cast<uint32_t>(client);
    k.thr = static_cast<uint32_t>(floor(p * 65536.0 + 0.5));
    k.scale = k.thr < 65536u ? 65536.0f / static_cast<float>(65536u - k.thr) : 0.0f;
    k.chunk_base = index_base / 8;
    return FASGD_OK;
}

fasgd_status check_vector(const char* name, const float* p, bool required)
{
    if (!p) return required ? fail(FASGD_ERR_NULL, "%s is NULL", name) : FASGD_OK;
    return aligned(p, 4) ? FASGD_OK : fail(FASGD_ERR_ALIGN, "%s is not 4-byte aligned", name);
}

// What both passes of a residual norm share.
fasgd_status norm_setup(const client_residual_norm* op, fasgd::NormArgs& a)
{
    if (!op) return fail(FASGD_ERR_NULL, "the operator's description is NULL");
    FASGD_TRY(check_shape(op->rows, op->cols, op->dtype));
    if (op->cols < 1 || op->cols > (int64_t(1) << 30))
        return fail(FASGD_ERR_ARG, "cols = %lld is not in [1, 2^30]", (long long)op->cols);
    if (op->kind != CLIENT_NORM_RMS && op->kind != CLIENT_NORM_LAYER)
        return fail(FASGD_ERR_ARG, "kind = %d is not a client_norm_kind value", op->kind);
    if (op->gate_form < CLIENT_GATE_NONE || op->gate_form > CLIENT_GATE_FULL)
        return fail(FASGD_ERR_ARG, "gate_form = %d is not a client_gate_form value", op->gate_form);
    if (op->gate_act < CLIENT_GATE_IDENTITY || op->gate_act > CLIENT_GATE_TANH)
        return fail(FASGD_ERR_ARG, "gate_act = %d is not a client_gate_act value", op->gate_act);
    if (!isfinite(op->residual_scale)) return fail(FASGD_ERR_ARG, "residual_scale must be finite");
    if (!(isfinite(op->eps) && op->eps > 0.0f)) return fail(FASGD_ERR_ARG, "eps must be finite and > 0");
    FASGD_TRY(check_vector("w_post", op->w_post, false));
    FASGD_TRY(check_vector("b_post", op->b_post, false));
    FASGD_TRY(check_vector("w_pre", op->w_pre, false));
    FASGD_TRY(check_vector("b_pre", op->b_pre, false));
    if ((op->b_post && !op->w_post) || (op->b_pre && !op->w_pre))
        return fail(FASGD_ERR_NULL, "a bias needs its norm's weights");
    memset(&a, 0, sizeof a);
    FASGD_TRY(drop_key(op->p, op->seed, op->T, op->client, op->site, op->index_base, op->rows * op->cols, a.key));
    if (op->rows > 0) {
        if (op->gate_form == CLIENT_GATE_FULL)
            FASGD_TRY(check_matrix("gate", op->gate, op->ld_gate, op->rows, op->cols, op->dtype));
        else if (op->gate_form != CLIENT_GATE_NONE)
            FASGD_TRY(check_vector("gate", static_cast<const float*>(op->gate), true));
    }
    a.rows = op->rows;
    a.cols = static_cast<int32_t>(op->cols);
    a.n_cols = static_cast<float>(op->cols);
    a.inv_cols = 1.0f / static_cast<float>(op->cols);
    a.layer = op->kind == CLIENT_NORM_LAYER;
    a.gate_form = op->gate_form;
    a.gate_act = op->gate_act;
    a.drop = a.key.thr != 0;
    a.rho = op->residual_scale;
    a.eps = op->eps;
    a.w_post = op->w_post;
    a.b_post = op->b_post;
    a.w_pre = op->w_pre;
    a.b_pre = op->b_pre;
    a.gate = op->gate;
    a.ld_gate = op->ld_gate;
    return FASGD_OK;
}

constexpr int64_t kMaxK = int64_t(1) << 23;    // of an operand: 256 rows of it stay within 32-bit offsets

constexpr int64_t kMaxOperandRows = int64_t(1) << 27;   // every product's launch stays below 2^32 threads

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// An 8-bit operand; its arrays are needed where it holds anything.
fasgd_status check_operand(const char* name, const client_fp8_operand* op, fasgd::Fp8View& v)
{
    if (!op) return fail(FASGD_ERR_NULL, "%s is NULL", name);
    if (op->format != CLIENT_FP8_E4M3 && op->format != CLIENT_FP8_E5M2)
        return fail(FASGD_ERR_ARG, "%s: format = %d is not a client_fp8_format value", name, op->format);
    if (op->rows < 0 || op->rows > kMaxOperandRows)
        return fail(FASGD_ERR_ARG, "%s: rows = %lld is not in [0, 2^27]", name, (long long)op->rows);
    if (op->k < 0 || op->k > kMaxK) return fail(FASGD_ERR_ARG, "%s: k = %lld is not in [0, 2^23]", name, (long long)op->k);
    v = fasgd::Fp8View{op->data, op->scales, op->rows, op->k, op->ld, op->lds, op->format};
    if (op->rows == 0 || op->k == 0) return FASGD_OK;
    if (!op->data || !op->scales) return fail(FASGD_ERR_NULL, "%s: data or scales is NULL", name);
    if (!aligned(op->data, 16) || !aligned(op->scales, 4))
        return fail(FASGD_ERR_ALIGN, "%s: data must be 16-byte and scales 4-byte aligned", name);
    if (op->ld < round_up(op->k, 128) || op->ld % 128 != 0 || op->ld > kMaxK)
        return fail(FASGD_ERR_ARG, "%s: ld = %lld must be a multiple of 128 in [k = %lld rounded up, 2^23]", name,
                    (long long)op->ld, (long long)op->k);
    if (op->lds < op->rows || op->lds % 4 != 0 || op->lds > kMaxElements)
        return fail(FASGD_ERR_ARG, "%s: lds = %lld must be a multiple of 4 of at least rows = %lld", name,
                    (long long)op->lds, (long long)op->rows);
    return FASGD_OK;
}

fasgd_status check_workspace(const void* workspace, size_t bytes, size_t need)
{
    if (need == 0) return FASGD_OK;
    if (!workspace) return fail(FASGD_ERR_NULL, "workspace is NULL");
    if (!aligned(workspace, 16)) return fail(FASGD_ERR_ALIGN, "workspace must be 16-byte aligned");
    if (bytes < need)
        return fail(FASGD_ERR_CAPACITY, "workspace of %zu bytes is smaller than the %zu needed", bytes, need);
    return FASGD_OK;
}

// Takes the choice of short sums out of an output's type.
fasgd_status take_short_sums(int32_t& dtype, int32_t& short_sums)
{
    short_sums = (dtype & CLIENT_FP8_SHORT_SUMS) != 0;
    dtype &= ~CLIENT_FP8_SHORT_SUMS;
    if (short_sums && dtype == CLIENT_F32) return fail(FASGD_ERR_ARG, "short sums are of 16-bit outputs");
    return FASGD_OK;
}

// client_fp8_linear's quantized x at the front of its workspace.
size_t linear_operand_bytes(int64_t m, int64_t k)
{
    return static_cast<size_t>(round_up(m * round_up(k, 128) + round_up(k, 128) / 128 * round_up(m, 4), 256));
}

}  // namespace

extern "C" {

fasgd_status client_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, void* y, int64_t ldy,
                            int64_t rows, int64_t cols, int32_t dtype, double p, uint64_t seed, int64_t T,
                            int32_t client, int32_t site, int64_t index_base, hipStream_t stream)
{
    FASGD_TRY(check_shape(rows, cols, dtype));
    fasgd::DropoutArgs a;
    memset(&a, 0, sizeof a);
    FASGD_TRY(drop_key(p, seed, T, client, site, index_base, rows * cols, a.key));
    if (rows == 0 || cols == 0) return ok();
    FASGD_TRY(check_matrix("x", x, ldx, rows, cols, dtype));
    FASGD_TRY(check_matrix("y", y, ldy, rows, cols, dtype));
    if (residual) FASGD_TRY(check_matrix("residual", residual, ldr, rows, cols, dtype));
    a.x = x;
    a.residual = residual;
    a.y = y;
    a.ldx = ldx;
    a.ldr = ldr;
    a.ldy = ldy;
    a.rows = rows;
    a.cols = cols;
    const hipError_t e = fasgd::launch_dropout(a, dtype, stream);
    if (e != hipSuccess) return hip_fail(e, "client_dropout");
    return ok();
}

size_t client_residual_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return 0;
    return fasgd::norm_workspace_bytes(rows, cols);
}

fasgd_status client_residual_norm_forward(const client_residual_norm* op, const void* branch, int64_t ld_branch,
                                          const void* residual, int64_t ld_residual, void* sum, int64_t ld_sum,
                                          void* normed, int64_t ld_normed, float* stats, hipStream_t stream)
{
    fasgd::NormArgs a;
    FASGD_TRY(norm_setup(op, a));
    if (a.rows == 0) return ok();
    FASGD_TRY(check_matrix("branch", branch, ld_branch, op->rows, op->cols, op->dtype));
    if (residual) FASGD_TRY(check_matrix("residual", residual, ld_residual, op->rows, op->cols, op->dtype));
    FASGD_TRY(check_matrix("sum", sum, ld_sum, op->rows, op->cols, op->dtype));
    if (op->w_pre) FASGD_TRY(check_matrix("normed", normed, ld_normed, op->rows, op->cols, op->dtype));
    FASGD_TRY(check_vector("stats", stats, true));
    a.branch = branch;
    a.residual = residual;
    a.sum = sum;
    a.normed = normed;
    a.stats = stats;
    a.ld_branch = ld_branch;
    a.ld_residual = ld_residual;
    a.ld_sum = ld_sum;
    a.ld_normed = ld_normed;
    const hipError_t e = fasgd::launch_norm_forward(a, op->dtype, stream);
    if (e != hipSuccess) return hip_fail(e, "client_residual_norm_forward");
    return ok();
}

fasgd_status client_residual_norm_backward(const client_residual_norm* op, const void* branch, int64_t ld_branch,
                                           const void* sum, int64_t ld_sum, const float* stats, const void* dsum,
                                           int64_t ld_dsum, const void* dnormed, int64_t ld_dnormed, void* dbranch,
                                           int64_t ld_dbranch, void* dresidual, int64_t ld_dresidual, float* dw_post,
                                           float* db_post, void* dgate, int64_t ld_dgate, float* dw_pre,
                                           float* db_pre, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    fasgd::NormArgs a;
    FASGD_TRY(norm_setup(op, a));
    if ((dw_post && !op->w_post) || (db_post && !op->b_post) || (dw_pre && !op->w_pre) || (db_pre && !op->b_pre))
        return fail(FASGD_ERR_ARG, "a gradient is asked for a parameter that is absent");
    FASGD_TRY(check_vector("dw_post", dw_post, false));
    FASGD_TRY(check_vector("db_post", db_post, false));
    FASGD_TRY(check_vector("dw_pre", dw_pre, false));
    FASGD_TRY(check_vector("db_pre", db_pre, false));
    if (op->gate_form == CLIENT_GATE_CHANNEL) FASGD_TRY(check_vector("dgate", static_cast<float*>(dgate), false));
    if (op->rows > 0) {
        FASGD_TRY(check_matrix("branch", branch, ld_branch, op->rows, op->cols, op->dtype));
        if (op->w_pre) {
            FASGD_TRY(check_matrix("sum", sum, ld_sum, op->rows, op->cols, op->dtype));
            FASGD_TRY(check_matrix("dnormed", dnormed, ld_dnormed, op->rows, op->cols, op->dtype));
        } else if (dnormed) {
            return fail(FASGD_ERR_ARG, "dnormed is given without w_pre");
        }
        if (dsum) FASGD_TRY(check_matrix("dsum", dsum, ld_dsum, op->rows, op->cols, op->dtype));
        FASGD_TRY(check_matrix("dbranch", dbranch, ld_dbranch, op->rows, op->cols, op->dtype));
        if (dresidual) FASGD_TRY(check_matrix("dresidual", dresidual, ld_dresidual, op->rows, op->cols, op->dtype));
        if (op->gate_form == CLIENT_GATE_FULL)
            FASGD_TRY(check_matrix("dgate", dgate, ld_dgate, op->rows, op->cols, op->dtype));
        if (op->gate_form == CLIENT_GATE_ROW) FASGD_TRY(check_vector("dgate", static_cast<float*>(dgate), true));
        FASGD_TRY(check_vector("stats", stats, true));
        if (!workspace) return fail(FASGD_ERR_NULL, "workspace is NULL");
        if (!aligned(workspace, 16)) return fail(FASGD_ERR_ALIGN, "workspace must be 16-byte aligned");
        const size_t need = fasgd::norm_workspace_bytes(op->rows, op->cols);
        if (workspace_bytes < need)
            return fail(FASGD_ERR_CAPACITY, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    }
    a.branch = branch;
    a.sum = const_cast<void*>(sum);
    a.stats = const_cast<float*>(stats);
    a.dsum = dsum;
    a.dnormed = dnormed;
    a.dbranch = dbranch;
    a.dresidual = dresidual;
    a.dgate = dgate;
    a.ld_branch = ld_branch;
    a.ld_sum = ld_sum;
    a.ld_dsum = ld_dsum;
    a.ld_dnormed = ld_dnormed;
    a.ld_dbranch = ld_dbranch;
    a.ld_dresidual = ld_dresidual;
    a.ld_dgate = ld_dgate;
    a.dw_post = dw_post;
    a.db_post = db_post;
    a.dw_pre = dw_pre;
    a.db_pre = db_pre;
    a.partial = static_cast<float*>(workspace);
    const hipError_t e = fasgd::launch_norm_backward(a, op->dtype, stream);
    if (e != hipSuccess) return hip_fail(e, "client_residual_norm_backward");
    return ok();
}

size_t client_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m < 1 || n < 1 || k < 1 || k > kMaxK || m > kMaxElements / n || m > kMaxElements / k) return 0;
    return linear_operand_bytes(m, k) + fasgd::fp8_workspace_bytes(m, n, k);
}

fasgd_status client_fp8_quantize(const void* x, int64_t ldx, int64_t rows, int64_t cols, int32_t dtype,
                                 int32_t block_rows, const client_fp8_operand* by_rows,
                                 const client_fp8_operand* by_cols, hipStream_t stream)
{
    FASGD_TRY(check_shape(rows, cols, dtype));
    if (block_rows != 1 && block_rows != 128) return fail(FASGD_ERR_ARG, "block_rows = %d is neither 1 nor 128", block_rows);
    if (!by_rows && !by_cols) return fail(FASGD_ERR_NULL, "by_rows and by_cols are both NULL");
    fasgd::QuantizeArgs a;
    memset(&a, 0, sizeof a);
    if (by_rows) FASGD_TRY(check_operand("by_rows", by_rows, a.row));
    if (by_cols) FASGD_TRY(check_operand("by_cols", by_cols, a.col));
    if (by_rows && (by_rows->rows != rows || by_rows->k != cols))
        return fail(FASGD_ERR_ARG, "by_rows is %lld x %lld, x is %lld x %lld", (long long)by_rows->rows,
                    (long long)by_rows->k, (long long)rows, (long long)cols);
    if (by_cols && (by_cols->rows != cols || by_cols->k != rows))
        return fail(FASGD_ERR_ARG, "by_cols is %lld x %lld, x transposed is %lld x %lld", (long long)by_cols->rows,
                    (long long)by_cols->k, (long long)cols, (long long)rows);
    if (by_rows && by_cols && by_rows->format != by_cols->format)
        return fail(FASGD_ERR_ARG, "by_rows and by_cols differ in format");
    if (rows == 0 || cols == 0) return ok();
    FASGD_TRY(check_matrix("x", x, ldx, rows, cols, dtype));
    a.x = x;
    a.ldx = ldx;
    a.rows = rows;
    a.cols = cols;
    a.whole = block_rows == 128;
    const hipError_t e = fasgd::launch_quantize(a, dtype, stream);
    if (e != hipSuccess) return hip_fail(e, "client_fp8_quantize");
    return ok();
}

fasgd_status client_fp8_matmul(const client_fp8_operand* a, const client_fp8_operand* b, void* c, int64_t ldc,
                               int32_t c_dtype, int32_t accumulate, void* workspace, size_t workspace_bytes,
                               hipStream_t stream)
{
    fasgd::Fp8Product p;
    memset(&p, 0, sizeof p);
    FASGD_TRY(take_short_sums(c_dtype, p.short_sums));
    FASGD_TRY(check_operand("a", a, p.a));
    FASGD_TRY(check_operand("b", b, p.b));
    if (a->k != b->k)
        return fail(FASGD_ERR_ARG, "a and b differ in k: %lld and %lld", (long long)a->k, (long long)b->k);
    FASGD_TRY(check_shape(a->rows, b->rows, c_dtype));
    if (a->rows == 0 || b->rows == 0) return ok();
    FASGD_TRY(check_matrix("c", c, ldc, a->rows, b->rows, c_dtype));
    FASGD_TRY(check_workspace(workspace, workspace_bytes, fasgd::fp8_workspace_bytes(a->rows, b->rows, a->k)));
    if (a->k == 0 && accumulate) return ok();
    p.c = c;
    p.ldc = ldc;
    p.c_dtype = c_dtype;
    p.accumulate = accumulate != 0;
    p.partial = static_cast<float*>(workspace);
    const hipError_t e = fasgd::launch_fp8_product(p, stream);
    if (e != hipSuccess) return hip_fail(e, "client_fp8_matmul");
    return ok();
}

fasgd_status client_fp8_linear(const void* x, int64_t ldx, int64_t m, const client_fp8_operand* w, void* y,
                               int64_t ldy, int32_t dtype, void* workspace, size_t workspace_bytes,
                               hipStream_t stream)
{
    fasgd::Fp8Product p;
    memset(&p, 0, sizeof p);
    FASGD_TRY(take_short_sums(dtype, p.short_sums));
    FASGD_TRY(check_operand("w", w, p.b));
    FASGD_TRY(check_shape(m, w->rows, dtype));
    FASGD_TRY(check_shape(m, w->k, dtype));
    if (m > kMaxOperandRows) return fail(FASGD_ERR_ARG, "m = %lld is not in [0, 2^27]", (long long)m);
    if (m == 0 || w->rows == 0) return ok();
    FASGD_TRY(check_matrix("y", y, ldy, m, w->rows, dtype));
    if (w->k > 0) {
        FASGD_TRY(check_matrix("x", x, ldx, m, w->k, dtype));
        FASGD_TRY(check_workspace(workspace, workspace_bytes, client_fp8_workspace_bytes(m, w->rows, w->k)));
    }
    const int64_t ld = round_up(w->k, 128);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    p.a = fasgd::Fp8View{base, base + m * ld, m, w->k, ld, round_up(m, 4), fasgd::FP8_E4M3};
    p.c = y;
    p.ldc = ldy;
    p.c_dtype = dtype;
    p.partial = reinterpret_cast<float*>(base + (w->k > 0 ? linear_operand_bytes(m, w->k) : 0));
    hipError_t e = hipSuccess;
    const bool few = w->k > 0 && fasgd::fp8_linear_few(m, w->k);
    if (few) {
        e = fasgd::launch_fp8_linear_few(x, ldx, p, stream);
    } else if (w->k > 0) {
        fasgd::QuantizeArgs q;
        memset(&q, 0, sizeof q);
        q.x = x;
        q.ldx = ldx;
        q.rows = m;
        q.cols = w->k;
        q.row = p.a;
        e = fasgd::launch_quantize(q, dtype, stream);
    }
    if (e == hipSuccess && !few) e = fasgd::launch_fp8_product(p, stream);
    if (e != hipSuccess) return hip_fail(e, "client_fp8_linear");
    return ok();
}

}  // extern "C"
