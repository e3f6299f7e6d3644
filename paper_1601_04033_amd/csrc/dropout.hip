// client_dropout: y = [residual +] drop(x), the mask drawn where it is used.
//
// Bound by memory: one read and one write an element, and the ten rounds of
// Philox for each 8 elements fit beside them.  16,384 x 4,096: fp16 41 us, 6.6
// TB/s; bf16 with a residual 70 us, 5.7 TB/s.
#include "client_kernels.hpp"

namespace fasgd {
namespace {

constexpr int kBlock = 256;
constexpr int kChunk = 8;

// One chunk of 8 consecutive matrix elements per thread: one Philox call and
// one wide access each way.  A chunk that crosses a row's end (rows of a
// length that is no multiple of 8) goes element by element.
template <typename T>
__global__ __launch_bounds__(kBlock) void dropout(DropoutArgs a)
{
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.residual);
    T* y = static_cast<T*>(a.y);
    const int64_t n = a.rows * a.cols;
    const int64_t i = a.first + (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * kChunk;
    if (i >= n) return;
    int64_t r = 0, c = i;
    if (a.rows == 1) {          // one row, or rows without gaps: nothing to divide
    } else if (n <= UINT32_MAX) {      // a 64-bit division costs as much as the draw
        r = static_cast<uint32_t>(i) / static_cast<uint32_t>(a.cols);
        c = i - r * a.cols;
    } else {
        r = i / a.cols;
        c = i - r * a.cols;
    }
    const uint32_t keep = keep_bits(a.key, a.key.chunk_base + i / kChunk);
    if (c + kChunk <= a.cols) {
        Pack<T, kChunk> v = load_pack<T, kChunk>(x + r * a.ldx + c);
        Pack<T, kChunk> q;
        if (res) q = load_pack<T, kChunk>(res + r * a.ldr + c);
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            float f = kept(to_float(v.v[e]) * a.key.scale, keep, kChunk - 1 - e);
            if (res) f += to_float(q.v[e]);
            v.v[e] = from_float<T>(f);
        }
        store_pack(y + r * a.ldy + c, v);
        // keeps the compiler from joining this store's last element with the other way's
        asm volatile("" ::: "memory");
        return;
    }
    if (a.cols >= kChunk) {     // at most one row ends here: the loads are under way together
        float f[kChunk];
        const T* xr = x + r * a.ldx + c;
        const T* rr = res + r * a.ldr + c;
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const bool next = c + e >= a.cols, in = i + e < n;
            f[e] = in ? to_float(xr[next ? a.ldx - a.cols + e : e]) : 0.0f;
        }
        T* yr = y + r * a.ldy + c;
#pragma unroll
        for (int e = 0; e < kChunk; ++e) {
            const bool next = c + e >= a.cols, in = i + e < n;
            f[e] = kept(f[e] * a.key.scale, keep, kChunk - 1 - e);
            if (res) f[e] += in ? to_float(rr[next ? a.ldr - a.cols + e : e]) : 0.0f;
            if (in) yr[next ? a.ldy - a.cols + e : e] = from_float<T>(f[e]);
        }
        return;
    }
    for (int e = 0; e < kChunk && i + e < n; ++e) {
        float f = kept(to_float(x[r * a.ldx + c]) * a.key.scale, keep, kChunk - 1 - e);
        if (res) f += to_float(res[r * a.ldr + c]);
        y[r * a.ldy + c] = from_float<T>(f);
        if (++c == a.cols) {
            c = 0;
            ++r;
        }
    }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& args, int dtype, hipStream_t s)
{
    DropoutArgs a = args;
    // Rows without gaps are one row: no row's end cuts a chunk (4,099 x 1,001
    // fp16: 5.7 against 7.6 us).
    if (a.ldx == a.cols && a.ldy == a.cols && (!a.residual || a.ldr == a.cols)) {
        a.cols *= a.rows;
        a.rows = 1;
    }
    constexpr int64_t kElements = int64_t(kBlock) * kChunk;
    const int64_t blocks = (a.rows * a.cols + kElements - 1) / kElements;
    hipError_t e = hipSuccess;
    for (int64_t b = 0; b < blocks && e == hipSuccess; b += kLaunchBlocks) {
        a.first = b * kElements;
        const unsigned n = static_cast<unsigned>(blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks);
        if (dtype == DTYPE_F32) dropout<float><<<n, kBlock, 0, s>>>(a);
        else if (dtype == DTYPE_BF16) dropout<bf16><<<n, kBlock, 0, s>>>(a);
        else dropout<f16><<<n, kBlock, 0, s>>>(a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace fasgd
