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

}  // extern "C"
