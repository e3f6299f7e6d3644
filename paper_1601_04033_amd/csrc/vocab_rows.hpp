// What the kernels of the losses over a vocabulary share: the entries that rows
// are held to, their coefficients, and the end of the forward pass.
#pragma once

#include <float.h>

#include "vocab_kernels.hpp"

#define VOCAB_TRY(call)                                 \
    do {                                                \
        const hipError_t try_error = (call);            \
        if (try_error != hipSuccess) return try_error;  \
    } while (0)

namespace fasgd {
namespace {

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / 64;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLog2eRest = 1.92596303e-8f;    // what fp32 leaves of log2(e)

__device__ __forceinline__ float wave_sum(float x)
{
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ float wave_max(float x)
{
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}
__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger of x in this lane and the one `apart` away.
__device__ __forceinline__ float larger_of(float x, int apart) { return fmaxf(x, __shfl_xor(x, apart)); }

// ---- entries

__device__ __forceinline__ float teacher_logit(const VocabArgs& a, int64_t at)
{
    if (a.dtype == DTYPE_F32) return static_cast<const float*>(a.teacher)[at];
    if (a.dtype == DTYPE_BF16) return to_float(static_cast<const bf16*>(a.teacher)[at]);
    return to_float(static_cast<const f16*>(a.teacher)[at]);
}

// Whether entry `at` of the index counts: a class of the vocabulary, to which
// the teacher gives any weight.
__device__ __forceinline__ bool counts(const VocabArgs& a, int64_t at)
{
    const int64_t i = a.index[at];
    return i >= 0 && i < a.vocab && !(a.teacher && teacher_logit(a, at) == -INFINITY);
}

// A row's teacher: weights are exp(s_t t - top) by.  A whole wave's work.
struct Teacher {
    float top, by;
};
__device__ __forceinline__ Teacher teacher_of(const VocabArgs& a, int64_t row, int lane)
{
    if (!a.teacher) return Teacher{0.0f, 1.0f - a.smoothing};
    if (a.teacher_lse) return Teacher{a.teacher_lse[row], 1.0f};
    float top = -INFINITY, sum = 0.0f;
    for (int k = lane; k < a.entries; k += 64)
        if (counts(a, row * a.entries + k)) top = fmaxf(top, teacher_logit(a, row * a.entries + k) * a.teacher_scale);
    const float all = wave_max(top);
    for (int k = lane; k < a.entries; k += 64)
        if (counts(a, row * a.entries + k))
            sum += power((teacher_logit(a, row * a.entries + k) * a.teacher_scale - all) * kLog2e);
    return Teacher{all, 1.0f / wave_sum(sum)};
}
// log of the weight before `by`, for an entry that counts
__device__ __forceinline__ float log_weight(const VocabArgs& a, const Teacher& t, int64_t at)
{
    return a.teacher ? teacher_logit(a, at) * a.teacher_scale - t.top : 0.0f;
}
__device__ __forceinline__ float weight(const VocabArgs& a, const Teacher& t, int64_t at)
{
    return power(log_weight(a, t, at) * kLog2e) * t.by;
}

// dz at a class with logit `picked` and weight q.
__device__ __forceinline__ float entry_value(const VocabRow& row, float picked, float q)
{
    const float p = power(__builtin_fmaf(picked, kLog2e, -row.l));
    return __builtin_fmaf(row.f, p, -row.b) - row.g * q;
}

// dz at entry k of a row, for the first of those that name a class (the
// weights of the same class add up); false for the others.
__device__ __forceinline__ bool entry_gradient(const VocabArgs& a, const VocabRow& row, const Teacher& t, int64_t r,
                                               int k, float* dz)
{
    const int64_t base = r * a.entries;
    if (!counts(a, base + k)) return false;
    const int64_t i = a.index[base + k];
    float q = 0.0f;
    if (a.entries == 1) {
        q = weight(a, t, base);
    } else {
        for (int j = 0; j < a.entries; ++j) {
            if (a.index[base + j] != i || !counts(a, base + j)) continue;
            if (j < k) return false;
            q += weight(a, t, base + j);
        }
    }
    *dz = entry_value(row, a.picked[base + k], q);
    return true;
}

// A row's coefficients of the backward pass.  A whole wave's work.
__device__ __forceinline__ VocabRow coefficients_of(const VocabArgs& a, int64_t r, const Teacher& t, int lane)
{
    VocabRow c;
    const float lse = a.lse[r];
    c.g = a.grad_scale * (a.dloss ? a.dloss[r] : 1.0f);
    c.l = lse * kLog2e;
    if (!a.teacher) {
        c.f = c.g * (1.0f + 2.0f * a.z_loss * lse);
        c.b = c.g * (a.smoothing / static_cast<float>(a.vocab));
    } else {
        float q = 0.0f;
        for (int k = lane; k < a.entries; k += 64)
            if (counts(a, r * a.entries + k)) q += weight(a, t, r * a.entries + k);
        c.f = c.g * wave_sum(q);
        c.b = 0.0f;
    }
    // What rounding took from l, the same in all of the row's probabilities: into
    // their factor.  (A log-sum-exp of 12 or more: up to 6.6e-7 of each.)
    const float rest = __builtin_fmaf(lse, kLog2eRest, __builtin_fmaf(lse, kLog2e, -c.l));
    if (fabsf(rest) < 1.0f) c.f = __builtin_fmaf(c.f, -rest * kLn2, c.f);
    return c;
}

// The outputs of row r from its log-sum-exp and the mean of its logits.  taken:
// known to take part; else that is found here, and what takes no part gets zeros.
// A whole wave's work.
__device__ __forceinline__ void finish_row(const VocabArgs& a, int64_t r, float lse, float mean, bool taken, int lane)
{
    if (!taken) {
        bool any = false;
        for (int k = lane; k < a.entries; k += 64) {
            const bool in = counts(a, r * a.entries + k);
            if (!in) a.picked[r * a.entries + k] = 0.0f;
            any |= in;
        }
        if (__ballot(any) == 0) {
            if (lane == 0) a.loss[r] = a.lse[r] = 0.0f;
            return;
        }
    }
    float loss = 0.0f;
    if (!a.teacher) {
        // without smoothing the mean plays no part: that of logits beside masked classes is -infinity, and 0 times it NaN
        if (lane == 0) loss = lse - (1.0f - a.smoothing) * a.picked[r] - (a.smoothing != 0.0f ? a.smoothing * mean : 0.0f) + a.z_loss * lse * lse;
    } else {
        const Teacher t = teacher_of(a, r, lane);
        const float log_by = logf(t.by);
        for (int k = lane; k < a.entries; k += 64)
            if (counts(a, r * a.entries + k)) {
                const float lw = log_weight(a, t, r * a.entries + k), q = power(lw * kLog2e) * t.by;
                loss += q == 0.0f ? 0.0f : q * (lw + log_by - (a.picked[r * a.entries + k] - lse));
            }
        loss = wave_sum(loss);
    }
    if (lane == 0) {
        a.loss[r] = loss;
        a.lse[r] = lse;
    }
}

// Rows' losses from the statistics of their logits: 8 rows a block, the slots
// in 32 parts, joined in order.  list: the rows that take part (NULL: all are
// here, and those that take none are told apart).
static __global__ __launch_bounds__(kBlock) void finish(VocabArgs a, const int32_t* list, const int32_t* active, const float2* partial,
                                                 const float* partial_sum, int64_t slots, int64_t padded)
{
    __shared__ float2 part[32][8];
    __shared__ float part_sum[32][8];
    __shared__ float lse_of[8], mean_of[8];
    const int64_t n = list ? *active : a.rows, first = static_cast<int64_t>(blockIdx.x) * 8;
    if (first >= n) return;
    const int at = threadIdx.x & 7, slice = threadIdx.x >> 3;
    float top = -FLT_MAX, sum = 0.0f, all = 0.0f;
#pragma unroll 4
    for (int64_t s = slice; s < slots; s += 32) {
        const float2 x = partial[s * padded + first + at];
        const float next = fmaxf(top, x.x);
        sum = sum * power(top - next) + x.y * power(x.x - next);
        top = next;
        if (partial_sum) all += partial_sum[s * padded + first + at];
    }
    part[slice][at] = make_float2(top, sum);
    part_sum[slice][at] = all;
    __syncthreads();
    if (threadIdx.x < 8) {
        top = -FLT_MAX;
        for (int s = 0; s < 32; ++s) top = fmaxf(top, part[s][at].x);
        sum = all = 0.0f;
        for (int s = 0; s < 32; ++s) {
            sum += part[s][at].y * power(part[s][at].x - top);
            all += part_sum[s][at];
        }
        lse_of[at] = __builtin_fmaf(top, kLn2, logf(sum));
        mean_of[at] = all * a.scale / static_cast<float>(a.vocab);
    }
    __syncthreads();
    for (int i = threadIdx.x >> 6; i < 8 && first + i < n; i += kWaves)
        finish_row(a, list ? list[first + i] : first + i, lse_of[i], mean_of[i], list != nullptr, threadIdx.x & 63);
}

}  // namespace
}  // namespace fasgd
