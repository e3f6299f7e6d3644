// client_residual_norm_forward / _backward: the norm after a block, its gate,
// dropout, the scaled residual sum and the norm before the next block, one
// pass over the rows each way.
//
//   xh1 = (x - mean1) rstd1,  z = xh1 w_post + b_post,  u = m a z,
//   s = rho r + u,  xh2 = (s - mean2) rstd2,  h = xh2 w_pre + b_pre
// with m the dropout factor and a = act(gate).  Backward, from ds' and dh:
//   q = dh w_pre,  ds = ds' + rstd2 (q - mean(q) - xh2 mean(q xh2)),
//   dr = rho ds,  du = m ds,  t = du a w_post,
//   dx = rstd1 (t - mean(t) - xh1 mean(t xh1))
// (mean(q), mean(t) in a layer norm only).  The parameters' gradients need
// four column sums: of du xh1 and du (with a, where it is not a column's own),
// and of dh xh2 and dh: w_post, b_post and a channel gate share the first two.
//
// Each row is read once into registers, 8 columns a thread, and stays there
// through its reductions.  A thread keeps its columns over all its rows, so
// parameters are read once per block and the column sums stay in its
// registers, written once per block and joined in a fixed order by a second
// small kernel.
//
// Measured at 16,384 x 4,096 bf16, rms, channel gate, dropout: forward 109 us
// (4.9 TB/s; 103 without dropout), backward 157 us (6 matrices: 5.1 TB/s),
// column sums 6 us; fp32 205 and 313 us (5.2 TB/s).  The vector unit is busy
// two thirds of the forward pass.  Biases and full gates cost most (2,053 x
// 5,003 fp16: 59 and 77 us): their registers leave room for two rows a CU
// forward and one backward, too few to hide a row's reductions.
#include "client_kernels.hpp"

namespace fasgd {
namespace {

constexpr int kAcc = 4;             // column sums of the backward pass
constexpr int kLoopThreads = 1024;  // threads per row where a row does not fit the registers

constexpr int kCols = 8;            // columns of a row per thread: one or two 16-byte vectors
// waves per SIMD, for which the kernels' registers are limited (8 for 16-bit
// types without biases and full gates: 8,192 x 8,192 bf16, forward 119 against
// 138 us at 6)
template <typename T> constexpr int kForwardWaves = sizeof(T) == 2 ? 8 : 6;
constexpr int kForwardGeneralWaves = 5;
constexpr int kBackwardWaves = 4;
constexpr int kSubThreads = 512;    // threads of a block whose waves hold whole rows

template <typename T> constexpr int kVec = 16 / static_cast<int>(sizeof(T));
template <typename T> constexpr int kVecs = kCols / kVec<T>;

// ---- sums over the lanes of a row

// Sum over groups of LANES consecutive lanes, in every lane of the group.
template <int LANES> __device__ __forceinline__ float lane_sum(float x)
{
    if constexpr (LANES >= 2) x += dpp<0xB1>(x);        // quad_perm 1 0 3 2
    if constexpr (LANES >= 4) x += dpp<0x4E>(x);        // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) x += dpp<0x141>(x);       // row_half_mirror
    if constexpr (LANES >= 16) x += dpp<0x140>(x);      // row_mirror
    if constexpr (LANES >= 32) {
        const Pair p = across<16>(x);
        x = p.x + p.y;
    }
    if constexpr (LANES >= 64) {
        const Pair p = across<32>(x);
        x = p.x + p.y;
    }
    return x;
}

// Sums of N values over the threads of a row.  SUB > 0: SUB lanes hold a
// row.  SUB = 0: the block's threads do; the waves' sums pass through one of
// two LDS buffers taken in turn, so that one barrier per reduction is enough
// (a buffer is written again only after the other one's barrier), and each
// group of 16 lanes joins them (a loop over the waves would wait for LDS once
// for each: 2,053 x 5,003 fp16 with full gate, training step 146 against
// 134 us).
typedef float WaveSums[2][16][2];
template <int SUB, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], WaveSums& buf, int& turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane_sum<SUB ? SUB : 64>(v[i]);
    if constexpr (SUB == 0) {
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 15;
        float(*b)[2] = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) b[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lane_sum<16>(lane < waves ? b[lane][i] : 0.0f);
    }
}

__device__ __forceinline__ float activate(float g, int act)
{
    if (act == ACT_SIGMOID) return 1.0f / (1.0f + expf(-g));
    if (act == ACT_TANH) return tanhf(g);
    return g;
}
// Activations of V gates in place, the kind of activation decided once.  (From
// the hardware's exponential and reciprocal alone a sigmoid is 30 ulps of fp32
// off at a gate of -40; it took 2,053 x 5,003 fp16 from 142 to 127 us.)
template <int V> __device__ __forceinline__ void activate_all(float (&g)[V], int act)
{
    if (act == ACT_SIGMOID) {
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = activate(g[j], ACT_SIGMOID);
    } else if (act == ACT_TANH) {
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = activate(g[j], ACT_TANH);
    }
}
// the derivative, from the activation's value
__device__ __forceinline__ float slope(float a, int act)
{
    if (act == ACT_SIGMOID) return a * (1.0f - a);
    if (act == ACT_TANH) return 1.0f - a * a;
    return 1.0f;
}

// Up to V elements at column c of a row of `cols` (0 beyond its end).
template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_cols(const T* row, int c, int cols)
{
    if (c + V <= cols) return load_pack<T, V>(row + c);
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = c + j < cols ? row[c + j] : from_float<T>(0.0f);
    return r;
}
template <typename T, int V> __device__ __forceinline__ Pack<T, V> zero_pack()
{
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = from_float<T>(0.0f);
    return r;
}
template <typename T, int V>
__device__ __forceinline__ void store_cols(T* row, int c, int cols, const Pack<T, V>& x)
{
    if (c + V <= cols) {
        store_pack(row + c, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (c + j < cols) row[c + j] = x.v[j];
}
// fp32 parameters of columns c .. c + V - 1; `none` where there are none
template <int V>
__device__ __forceinline__ void load_params(const float* p, int c, int cols, float none, float (&out)[V])
{
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = none;
    if (p == nullptr) return;
    const Pack<float, V> x = load_cols<float, V>(p, c, cols);
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = x.v[j];
}

// s / n, from 1 / n and one correction: a row of one value has that mean.
// (The general division and square root are some 30 instructions in every
// wave of a row, and no nearer: of 20,000 rows whose sums are exact, means
// are within half an ulp and inverse roots within 1.01 x 2^-23, where the
// loops below, which divide, reach 0.97.)
__device__ __forceinline__ float mean_of(float s, const NormArgs& a)
{
    const float q = s * a.inv_cols;
    return fmaf(fmaf(-q, a.n_cols, s), a.inv_cols, q);
}
// 1 / sqrt(x) to an ulp; the hardware's has no subnormal arguments.
__device__ __forceinline__ float inverse_root(float x)
{
    return x < 0x1p-100f ? 1.0f / sqrtf(x) : __builtin_amdgcn_rsqf(x);
}

// mean and 1 / sqrt(variance + eps) of a row held as NV vectors of V in d
// (0 beyond the row's end); d becomes d - mean there.  The variance is that
// of the centred values.
template <int SUB, int NV, int V>
__device__ __forceinline__ void row_stats(float (&d)[NV][V], const NormArgs& a, int t, int tpr, float& mean,
                                          float& rstd, WaveSums& buf, int& turn)
{
    mean = 0.0f;
    if (a.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += d[v][j];
        row_sum<SUB>(s, buf, turn);
        mean = mean_of(s[0], a);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int left = a.cols - (v * tpr + t) * V;
            if (left >= V) {
#pragma unroll
                for (int j = 0; j < V; ++j) d[v][j] -= mean;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) d[v][j] = j < left ? d[v][j] - mean : 0.0f;
            }
        }
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < V; ++j) q[0] = fmaf(d[v][j], d[v][j], q[0]);
    row_sum<SUB>(q, buf, turn);
    rstd = inverse_root(fmaf(q[0], a.inv_cols, a.eps));
}

// Where a thread stands: its row's group of threads and its columns.  SUB > 0:
// SUB lanes of a block of kSubThreads hold a row; SUB = 0: the block does.
template <typename T, int SUB> struct Place {
    int tpr, t, rpb, group;     // threads per row, this one among them; rows per block, this one among them
    __device__ Place()
    {
        constexpr int S = SUB ? SUB : 1;
        tpr = SUB ? S : blockDim.x;
        t = SUB ? threadIdx.x % S : threadIdx.x;
        rpb = SUB ? kSubThreads / S : 1;
        group = SUB ? threadIdx.x / S : 0;
    }
    __device__ int column(int v) const { return (v * tpr + t) * kVec<T>; }
};

// Parameters of a thread's columns: in registers, or (IN_LDS) in LDS, WHICH
// of them.
template <typename T, int SUB, int MAXT, int WHICH, bool IN_LDS> struct Params {
    static constexpr int V = kVec<T>, NV = kVecs<T>;
    float reg[IN_LDS ? 1 : WHICH][NV][V];
    static __device__ float* lds(int which)
    {
        if constexpr (SUB == 0 && MAXT == 512) {
            // as much as the block's threads need: small blocks share a CU
            extern __shared__ __attribute__((aligned(16))) float dynamic[];
            return dynamic + which * (blockDim.x * kCols);
        } else {
            __shared__ __attribute__((aligned(16))) float x[WHICH][(SUB ? SUB : MAXT) * kCols];
            return x[which];
        }
    }
    __device__ void set(int which, int v, const Place<T, SUB>& at, const float (&x)[V])
    {
        if constexpr (IN_LDS) {
            if (at.group == 0) {
#pragma unroll
                for (int j = 0; j < V; ++j) lds(which)[at.column(v) + j] = x[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) reg[which][v][j] = x[j];
        }
    }
    __device__ void get(int which, int v, const Place<T, SUB>& at, float (&x)[V]) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = IN_LDS ? lds(which)[at.column(v) + j] : reg[which][v][j];
    }
};

// Keep bits of a thread's columns of a row (all kept without dropout).
template <typename T, int SUB>
__device__ __forceinline__ void row_keep(const NormArgs& a, const Place<T, SUB>& at, int64_t row, int cols,
                                         uint32_t (&keep)[kVecs<T>])
{
#pragma unroll
    for (int v = 0; v < kVecs<T>; ++v) keep[v] = ~0u;
    if (!a.drop) return;
    if constexpr (kVec<T> == 8 && (SUB == 0 || SUB == 64)) {
        // A wave's lanes hold neighbouring runs of 8, which begin `off` into
        // a chunk of the draws: a lane's run ends in its right neighbour's
        // first chunk, and only the last lane's in one that no lane has drawn,
        // which the scalar unit draws.
        const int64_t first = row * a.cols + at.column(0);
        const uint64_t chunk = static_cast<uint64_t>(a.key.chunk_base) + static_cast<uint64_t>(first >> 3);
        const uint32_t mine = keep_bits(a.key, chunk);
        const int off = __builtin_amdgcn_readfirstlane(static_cast<int>(first & 7));
        keep[0] = mine;
        if (off == 0) return;
        const uint32_t low = __builtin_amdgcn_readlane(static_cast<uint32_t>(chunk), 63);
        const uint32_t high = __builtin_amdgcn_readlane(static_cast<uint32_t>(chunk >> 32), 63);
        const uint32_t last = keep_bits(a.key, (static_cast<uint64_t>(high) << 32 | low) + 1);
        uint32_t next = __shfl_down(mine, 1);
        if ((threadIdx.x & 63) == 63) next = last;
        keep[0] = (mine << 8 | next) >> (8 - off);
        return;
    }
#pragma unroll
    for (int v = 0; v < kVecs<T>; ++v)
        if (at.column(v) < cols) keep[v] = keep_run<kVec<T>>(a.key, row * a.cols + at.column(v));
}

// GENERAL kernels take biases and a gate of every element.  Both cost
// registers in every thread, so operators without them have kernels of their
// own, and the general backward kernel has its parameters in LDS: with at
// most 128 registers two blocks of 512 threads share a CU, and one computes
// while the other waits for its row or its reduction.  (A row loaded ahead
// into registers instead cost more in waves than it gave.)

// ---- forward

template <typename T, int SUB, int MAXT, bool GENERAL>
__global__ __launch_bounds__(MAXT, GENERAL ? kForwardGeneralWaves : kForwardWaves<T>) void norm_forward(NormArgs a)
{
    constexpr int V = kVec<T>, NV = kVecs<T>;
    constexpr int kPost = 0, kPre = 1, kPostBias = 2, kPreBias = 3;
    __shared__ __attribute__((aligned(8))) WaveSums buf;
    int turn = 0;
    const Place<T, SUB> at;
    // the dropout's scale and a channel gate are folded into the first norm's weights and bias
    Params<T, SUB, MAXT, GENERAL ? 4 : 2, false> params;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = at.column(v);
        float f[V], x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = 1.0f;
        if (a.gate_form == GATE_CHANNEL) {
            load_params<V>(static_cast<const float*>(a.gate), c, a.cols, 0.0f, f);
            activate_all(f, a.gate_act);
        }
        const float scale = a.drop ? a.key.scale : 1.0f;
        load_params<V>(a.w_post, c, a.cols, 1.0f, x);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] *= f[j] * scale;
        params.set(kPost, v, at, x);
        load_params<V>(a.w_pre, c, a.cols, 1.0f, x);
        params.set(kPre, v, at, x);
        if constexpr (GENERAL) {
            load_params<V>(a.b_post, c, a.cols, 0.0f, x);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] *= f[j] * scale;
            params.set(kPostBias, v, at, x);
            load_params<V>(a.b_pre, c, a.cols, 0.0f, x);
            params.set(kPreBias, v, at, x);
        }
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * at.rpb;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * at.rpb; base < a.rows; base += step) {
        const int64_t row = base + at.group;
        const int cols = row < a.rows ? a.cols : 0;
        Pack<T, V> x[NV], r[NV], g[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = at.column(v);
            x[v] = load_cols<T, V>(static_cast<const T*>(a.branch) + row * a.ld_branch, c, cols);
            if (a.residual) r[v] = load_cols<T, V>(static_cast<const T*>(a.residual) + row * a.ld_residual, c, cols);
            else r[v] = zero_pack<T, V>();
            if (GENERAL && a.gate_form == GATE_FULL)
                g[v] = load_cols<T, V>(static_cast<const T*>(a.gate) + row * a.ld_gate, c, cols);
        }
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW && row < a.rows)
            row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        uint32_t keep[NV];
        row_keep<T, SUB>(a, at, row, cols, keep);
        float d[NV][V];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) d[v][j] = to_float(x[v].v[j]);
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (a.w_post) row_stats<SUB>(d, a, at.t, at.tpr, mean1, rstd1, buf, turn);
        const float k = rstd1 * row_gate;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = at.column(v);
            float w[V], b[V];
            params.get(kPost, v, at, w);
            if constexpr (GENERAL) params.get(kPostBias, v, at, b);
#pragma unroll
            for (int j = 0; j < V; ++j)
                d[v][j] = GENERAL ? fmaf(d[v][j] * k, w[j], b[j] * row_gate) : d[v][j] * k * w[j];
            if (GENERAL && a.gate_form == GATE_FULL) {
                float f[V];
#pragma unroll
                for (int j = 0; j < V; ++j) f[j] = to_float(g[v].v[j]);
                activate_all(f, a.gate_act);
#pragma unroll
                for (int j = 0; j < V; ++j) d[v][j] *= f[j];
            }
            Pack<T, V> out;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                out.v[j] = from_float<T>(scaled_sum(a.rho, to_float(r[v].v[j]), kept(d[v][j], keep[v], V - 1 - j)));
                // the norm is of the sum as it is stored, so that the
                // backward pass, which reads it, differentiates this function
                d[v][j] = to_float(out.v[j]);
            }
            if (c + V > cols) {
#pragma unroll
                for (int j = 0; j < V; ++j) d[v][j] = c + j < cols ? d[v][j] : 0.0f;
            }
            store_cols<T, V>(static_cast<T*>(a.sum) + row * a.ld_sum, c, cols, out);
        }
        if (a.w_pre) {
            row_stats<SUB>(d, a, at.t, at.tpr, mean2, rstd2, buf, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[V], b[V];
                params.get(kPre, v, at, w);
                if constexpr (GENERAL) params.get(kPreBias, v, at, b);
                Pack<T, V> out;
#pragma unroll
                for (int j = 0; j < V; ++j)
                    out.v[j] = from_float<T>(GENERAL ? fmaf(d[v][j] * rstd2, w[j], b[j]) : d[v][j] * rstd2 * w[j]);
                store_cols<T, V>(static_cast<T*>(a.normed) + row * a.ld_normed, at.column(v), cols, out);
            }
        }
        if (at.t == 0 && row < a.rows) {
            const float st[4] = {mean1, rstd1, mean2, rstd2};
            __builtin_memcpy(a.stats + row * 4, st, sizeof st);
        }
    }
}

// ---- backward

template <typename T, int SUB, int MAXT, bool GENERAL>
__global__ __launch_bounds__(MAXT, SUB && GENERAL ? 2 : kBackwardWaves) void norm_backward(NormArgs a)
{
    constexpr int V = kVec<T>, NV = kVecs<T>;
    constexpr int kPost = 0, kPre = 1, kPostBias = 2;   // kPost: w_post, times the gate where it is the column's
    __shared__ __attribute__((aligned(8))) WaveSums buf;
    int turn = 0;
    const Place<T, SUB> at;
    // A row is loaded where its registers come free, at the end of the row
    // before it (16,384 x 4,096 bf16: 195 against 216 us), except where two
    // blocks do not share a CU or registers are short (5,003 columns: 61
    // against 51 us; with biases, 1,000 fp32 columns: 138 against 116).
    constexpr bool kAhead = SUB == 0 && MAXT == 512 && !GENERAL;
    Pack<T, V> x[NV], s[NV], dh[NV], up[NV], g[NV];
    float st[4];
    auto fetch = [&](int64_t row) {
        const int cols = row < a.rows ? a.cols : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = at.column(v);
            if (a.w_pre) {
                s[v] = load_cols<T, V>(static_cast<const T*>(a.sum) + row * a.ld_sum, c, cols);
                dh[v] = load_cols<T, V>(static_cast<const T*>(a.dnormed) + row * a.ld_dnormed, c, cols);
            }
            if (a.dsum) up[v] = load_cols<T, V>(static_cast<const T*>(a.dsum) + row * a.ld_dsum, c, cols);
            else up[v] = zero_pack<T, V>();
            x[v] = load_cols<T, V>(static_cast<const T*>(a.branch) + row * a.ld_branch, c, cols);
            if (GENERAL && a.gate_form == GATE_FULL)
                g[v] = load_cols<T, V>(static_cast<const T*>(a.gate) + row * a.ld_gate, c, cols);
        }
        if (cols) __builtin_memcpy(st, a.stats + row * 4, sizeof st);
        else st[0] = st[1] = st[2] = st[3] = 0.0f;
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * at.rpb;
    if (kAhead) fetch(static_cast<int64_t>(blockIdx.x) * at.rpb + at.group);
    Params<T, SUB, MAXT, GENERAL ? 3 : 2, GENERAL> params;
    float post1[NV][V], post2[NV][V], pre1[NV][V], pre2[NV][V];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = at.column(v);
        float x[V];
#pragma unroll
        for (int j = 0; j < V; ++j) post1[v][j] = post2[v][j] = pre1[v][j] = pre2[v][j] = 0.0f;
        load_params<V>(a.w_post, c, a.cols, 1.0f, x);
        if (a.gate_form == GATE_CHANNEL) {
            float f[V];
            load_params<V>(static_cast<const float*>(a.gate), c, a.cols, 0.0f, f);
            activate_all(f, a.gate_act);
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] *= f[j];
        }
        params.set(kPost, v, at, x);
        load_params<V>(a.w_pre, c, a.cols, 1.0f, x);
        params.set(kPre, v, at, x);
        if constexpr (GENERAL) {
            load_params<V>(a.b_post, c, a.cols, 0.0f, x);
            params.set(kPostBias, v, at, x);
        }
    }
    if (GENERAL) __syncthreads();
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * at.rpb; base < a.rows; base += step) {
        const int64_t row = base + at.group;
        const int cols = row < a.rows ? a.cols : 0;
        if (!kAhead) fetch(row);
        const float mean1 = st[0], rstd1 = st[1], mean2 = st[2], rstd2 = st[3];
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW && row < a.rows)
            row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        uint32_t keep[NV];
        row_keep<T, SUB>(a, at, row, cols, keep);
        float ds[NV][V], q[NV][V], xh[NV][V];
        float two[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) ds[v][j] = to_float(up[v].v[j]);
        if (a.w_pre) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float w[V];
                params.get(kPre, v, at, w);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float h = to_float(dh[v].v[j]);
                    xh[v][j] = (to_float(s[v].v[j]) - mean2) * rstd2;
                    q[v][j] = h * w[j];
                    pre1[v][j] = fmaf(h, xh[v][j], pre1[v][j]);
                    if (GENERAL) pre2[v][j] += h;
                    two[0] = fmaf(q[v][j], xh[v][j], two[0]);
                }
                if (a.layer) {
#pragma unroll
                    for (int j = 0; j < V; ++j) two[1] += q[v][j];
                }
            }
            row_sum<SUB>(two, buf, turn);
            const float m0 = two[0] * a.inv_cols * rstd2, m1 = a.layer ? two[1] * a.inv_cols * rstd2 : 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) ds[v][j] += fmaf(rstd2, q[v][j], fmaf(-m0, xh[v][j], -m1));
        }
        const float scale = a.drop ? a.key.scale : 1.0f;
        two[0] = two[1] = 0.0f;
        float dg_row[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = at.column(v);
            Pack<T, V> out;
#pragma unroll
            for (int j = 0; j < V; ++j) out.v[j] = from_float<T>(a.rho * ds[v][j]);
            if (a.dresidual) store_cols<T, V>(static_cast<T*>(a.dresidual) + row * a.ld_dresidual, c, cols, out);
            if (c + V > cols) {
#pragma unroll
                for (int j = 0; j < V; ++j) ds[v][j] = c + j < cols ? ds[v][j] : 0.0f;
            }
            // ds becomes du, and then the gradient of z
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ds[v][j] = kept(ds[v][j], keep[v], V - 1 - j) * scale;
                xh[v][j] = (to_float(x[v].v[j]) - mean1) * rstd1;
            }
            if (a.drop && !a.w_post) {
                // what is dropped takes no part, were it infinite or NaN
#pragma unroll
                for (int j = 0; j < V; ++j) xh[v][j] = kept(xh[v][j], keep[v], V - 1 - j);
            }
            float w[V], b[V];
            params.get(kPost, v, at, w);
            if constexpr (GENERAL) params.get(kPostBias, v, at, b);
            if (GENERAL && a.gate_form == GATE_FULL) {
                float f[V], z[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    f[j] = to_float(g[v].v[j]);
                    z[j] = ds[v][j] * fmaf(xh[v][j], w[j], b[j]);
                }
                activate_all(f, a.gate_act);
                if (a.gate_act == ACT_SIGMOID) {
#pragma unroll
                    for (int j = 0; j < V; ++j) z[j] *= slope(f[j], ACT_SIGMOID);
                } else if (a.gate_act == ACT_TANH) {
#pragma unroll
                    for (int j = 0; j < V; ++j) z[j] *= slope(f[j], ACT_TANH);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    out.v[j] = from_float<T>(z[j]);
                    ds[v][j] *= f[j];
                }
                if (a.drop) {
                    // nor does the gate of what is dropped, were it infinite or NaN
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        out.v[j] = from_float<T>(kept(z[j], keep[v], V - 1 - j));
                        ds[v][j] = kept(ds[v][j], keep[v], V - 1 - j);
                    }
                }
                store_cols<T, V>(static_cast<T*>(a.dgate) + row * a.ld_dgate, c, cols, out);
            } else if (a.gate_form == GATE_ROW) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    dg_row[0] = fmaf(ds[v][j], GENERAL ? fmaf(xh[v][j], w[j], b[j]) : xh[v][j] * w[j], dg_row[0]);
                    ds[v][j] *= row_gate;
                }
            }
            // a channel gate is the column's own: the column sums go without it
#pragma unroll
            for (int j = 0; j < V; ++j) {
                post1[v][j] = fmaf(ds[v][j], xh[v][j], post1[v][j]);
                if (GENERAL) post2[v][j] += ds[v][j];
                q[v][j] = ds[v][j] * w[j];
                two[0] = fmaf(q[v][j], xh[v][j], two[0]);
            }
            if (a.layer) {
#pragma unroll
                for (int j = 0; j < V; ++j) two[1] += q[v][j];
            }
        }
        if (a.gate_form == GATE_ROW) {
            row_sum<SUB>(dg_row, buf, turn);
            if (at.t == 0 && row < a.rows) static_cast<float*>(a.dgate)[row] = dg_row[0] * slope(row_gate, a.gate_act);
        }
        if (a.w_post) {
            row_sum<SUB>(two, buf, turn);
            const float m0 = two[0] * a.inv_cols * rstd1, m1 = a.layer ? two[1] * a.inv_cols * rstd1 : 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) q[v][j] = fmaf(rstd1, q[v][j], fmaf(-m0, xh[v][j], -m1));
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Pack<T, V> out;
#pragma unroll
            for (int j = 0; j < V; ++j) out.v[j] = from_float<T>(q[v][j]);
            store_cols<T, V>(static_cast<T*>(a.dbranch) + row * a.ld_dbranch, at.column(v), cols, out);
        }
        if (kAhead) fetch(row + step);
    }
    // column sums: groups of a wave, then the block's waves, then one row of the partial sums per block
    auto put = [&](int which, float (&acc)[NV][V]) {
        float* out = a.partial + (static_cast<int64_t>(which) * gridDim.x + blockIdx.x) * a.cols;
        if constexpr (SUB == 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Pack<float, V> p;
#pragma unroll
                for (int j = 0; j < V; ++j) p.v[j] = acc[v][j];
                store_cols<float, V>(out, at.column(v), a.cols, p);
            }
        } else {
            constexpr int kWaves = kSubThreads / 64;
            __shared__ float join[kWaves][SUB * kCols];
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float x = acc[v][j];
#pragma unroll
                    for (int lanes = SUB; lanes < 64; lanes *= 2) x += __shfl_xor(x, lanes);
                    if ((threadIdx.x & 63) < SUB) join[threadIdx.x >> 6][at.column(v) + j] = x;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += kSubThreads) {
                float x = join[0][c];
                for (int w = 1; w < kWaves; ++w) x += join[w][c];
                out[c] = x;
            }
        }
    };
    put(0, post1);
    put(1, pre1);
    if (GENERAL) {
        put(2, post2);
        put(3, pre2);
    }
}

// The column sums of `blocks` blocks joined: each of the block's 16 waves
// takes every 16th, and the waves' sums are added in order, so the order is
// fixed.  blockIdx.y: the norm after the block, or the one before the next.
__global__ __launch_bounds__(1024) void norm_columns(NormArgs a, int blocks, int bias, int first)
{
    __shared__ float part[2][16][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, pre = blockIdx.y;
    const int c = first + blockIdx.x * 64 + lane;
    float s[2] = {0.0f, 0.0f};
    if (c < a.cols) {
        const float* p = a.partial + static_cast<int64_t>(pre) * blocks * a.cols + c;
#pragma unroll 8
        for (int b = slice; b < blocks; b += 16) s[0] += p[static_cast<int64_t>(b) * a.cols];
        if (bias) {
            p += static_cast<int64_t>(2) * blocks * a.cols;
#pragma unroll 8
            for (int b = slice; b < blocks; b += 16) s[1] += p[static_cast<int64_t>(b) * a.cols];
        }
    }
    part[0][slice][lane] = s[0];
    part[1][slice][lane] = s[1];
    __syncthreads();
    if (slice != 0 || c >= a.cols) return;
    for (int k = 1; k < 16; ++k) {
        s[0] += part[0][k][lane];
        s[1] += part[1][k][lane];
    }
    if (pre) {
        if (a.dw_pre) a.dw_pre[c] = s[0];
        if (a.db_pre) a.db_pre[c] = s[1];
        return;
    }
    float f = 1.0f;
    if (a.gate_form == GATE_CHANNEL) {
        f = activate(static_cast<const float*>(a.gate)[c], a.gate_act);
        const float w = a.w_post ? a.w_post[c] : 1.0f, b = a.b_post ? a.b_post[c] : 0.0f;
        if (a.dgate) static_cast<float*>(a.dgate)[c] = slope(f, a.gate_act) * (w * s[0] + b * s[1]);
    }
    if (a.dw_post) a.dw_post[c] = f * s[0];
    if (a.db_post) a.db_post[c] = f * s[1];
}

// 16 threads a column and norm, so a launch takes 2^26 columns of the 2^30
// that there may be: it may have fewer than 2^32 threads.
void launch_columns(const NormArgs& a, int blocks, int bias, hipStream_t s)
{
    constexpr int kColumns = 1 << 26;
    for (int first = 0; first < a.cols; first += kColumns) {
        const int n = a.cols - first < kColumns ? a.cols - first : kColumns;
        norm_columns<<<dim3((n + 63) / 64, a.w_pre ? 2 : 1), 1024, 0, s>>>(a, blocks, bias, first);
        if (hipPeekAtLastError() != hipSuccess) return;     // the launcher's caller takes it
    }
}

// ---- rows too long for the registers: the same sums with the row read again

template <typename T> __global__ __launch_bounds__(kLoopThreads) void norm_forward_loop(NormArgs a)
{
    __shared__ __attribute__((aligned(8))) WaveSums buf;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.branch) + row * a.ld_branch;
        const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.ld_residual : nullptr;
        T* sum = static_cast<T*>(a.sum) + row * a.ld_sum;
        float st[4] = {0.0f, 1.0f, 0.0f, 1.0f};
        auto stats = [&](const T* p, float& mean, float& rstd) {
            float s[1] = {0.0f};
            if (a.layer) {
                for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) s[0] += to_float(p[c]);
                row_sum<0>(s, buf, turn);
            }
            mean = s[0] / a.n_cols;      // divided, so that a row of one value has that mean
            s[0] = 0.0f;
            for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
                const float d = to_float(p[c]) - mean;
                s[0] = fmaf(d, d, s[0]);
            }
            row_sum<0>(s, buf, turn);
            rstd = 1.0f / sqrtf(s[0] / a.n_cols + a.eps);
        };
        if (a.w_post) stats(x, st[0], st[1]);
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW) row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            float u = (to_float(x[c]) - st[0]) * st[1];
            u = fmaf(u, a.w_post ? a.w_post[c] : 1.0f, a.b_post ? a.b_post[c] : 0.0f) * row_gate;
            if (a.gate_form == GATE_CHANNEL) u *= activate(static_cast<const float*>(a.gate)[c], a.gate_act);
            if (a.gate_form == GATE_FULL)
                u *= activate(to_float(static_cast<const T*>(a.gate)[row * a.ld_gate + c]), a.gate_act);
            if (a.drop) u = kept(u * a.key.scale, keep_run<1>(a.key, row * a.cols + c), 0);
            if (r) u = scaled_sum(a.rho, to_float(r[c]), u);
            sum[c] = from_float<T>(u);
        }
        if (a.w_pre) {
            // each thread reads back only what it wrote
            stats(sum, st[2], st[3]);
            T* h = static_cast<T*>(a.normed) + row * a.ld_normed;
            for (int c = threadIdx.x; c < a.cols; c += kLoopThreads)
                h[c] = from_float<T>(fmaf((to_float(sum[c]) - st[2]) * st[3], a.w_pre[c], a.b_pre ? a.b_pre[c] : 0.0f));
        }
        if (threadIdx.x == 0) __builtin_memcpy(a.stats + row * 4, st, sizeof st);
    }
}

template <typename T> __global__ __launch_bounds__(kLoopThreads) void norm_backward_loop(NormArgs a)
{
    __shared__ __attribute__((aligned(8))) WaveSums buf;
    int turn = 0;
    float* acc[kAcc];
    for (int i = 0; i < kAcc; ++i) acc[i] = a.partial + (static_cast<int64_t>(i) * gridDim.x + blockIdx.x) * a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const bool first = row == blockIdx.x;
        const T* x = static_cast<const T*>(a.branch) + row * a.ld_branch;
        const T* s = static_cast<const T*>(a.sum) + row * a.ld_sum;
        const T* dh = static_cast<const T*>(a.dnormed) + row * a.ld_dnormed;
        float st[4];
        __builtin_memcpy(st, a.stats + row * 4, sizeof st);
        float two[2] = {0.0f, 0.0f};
        if (a.w_pre) {
            for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
                const float xh = (to_float(s[c]) - st[2]) * st[3], q = to_float(dh[c]) * a.w_pre[c];
                two[0] = fmaf(q, xh, two[0]);
                two[1] += q;
            }
            row_sum<0>(two, buf, turn);
        }
        const float m0 = two[0] * a.inv_cols, m1 = a.layer ? two[1] * a.inv_cols : 0.0f;
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW) row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        // ds, du, the normed branch value and the gate of one element; what is
        // dropped takes no part, were it or its own gate infinite or NaN
        auto element = [&](int c, float& ds, float& du, float& xh1, float& xa, float& g) {
            ds = a.dsum ? to_float(static_cast<const T*>(a.dsum)[row * a.ld_dsum + c]) : 0.0f;
            if (a.w_pre) {
                const float xh = (to_float(s[c]) - st[2]) * st[3];
                ds = fmaf(st[3], to_float(dh[c]) * a.w_pre[c] - m1 - xh * m0, ds);
            }
            du = ds;
            g = row_gate;
            if (a.gate_form == GATE_CHANNEL) g = activate(static_cast<const float*>(a.gate)[c], a.gate_act);
            if (a.gate_form == GATE_FULL)
                g = activate(to_float(static_cast<const T*>(a.gate)[row * a.ld_gate + c]), a.gate_act);
            xa = xh1 = (to_float(x[c]) - st[0]) * st[1];
            if (a.drop) {
                const uint32_t keep = keep_run<1>(a.key, row * a.cols + c);
                du = kept(du * a.key.scale, keep, 0);
                xa = kept(xa, keep, 0);
                if (a.gate_form == GATE_FULL) g = kept(g, keep, 0);
            }
        };
        float three[2] = {0.0f, 0.0f}, dg_row[1] = {0.0f};
        for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            float ds, du, xh, xa, g;
            element(c, ds, du, xh, xa, g);
            const float w = a.w_post ? a.w_post[c] : 1.0f;
            const float z = fmaf(xa, w, a.b_post ? a.b_post[c] : 0.0f);
            if (a.gate_form == GATE_ROW) dg_row[0] = fmaf(du, z, dg_row[0]);
            const float own = a.gate_form == GATE_CHANNEL ? du : du * g;
            acc[0][c] = fmaf(own, xa, first ? 0.0f : acc[0][c]);
            acc[2][c] = own + (first ? 0.0f : acc[2][c]);
            float d = 0.0f, xh2 = 0.0f;
            if (a.w_pre) {
                d = to_float(dh[c]);
                xh2 = (to_float(s[c]) - st[2]) * st[3];
            }
            acc[1][c] = fmaf(d, xh2, first ? 0.0f : acc[1][c]);
            acc[3][c] = d + (first ? 0.0f : acc[3][c]);
            const float q = du * g * w;
            three[0] = fmaf(q, xa, three[0]);
            three[1] += q;
        }
        if (a.w_post) row_sum<0>(three, buf, turn);
        if (a.gate_form == GATE_ROW) {
            row_sum<0>(dg_row, buf, turn);
            if (threadIdx.x == 0) static_cast<float*>(a.dgate)[row] = dg_row[0] * slope(row_gate, a.gate_act);
        }
        const float k0 = a.w_post ? three[0] * a.inv_cols : 0.0f;
        const float k1 = a.w_post && a.layer ? three[1] * a.inv_cols : 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            float ds, du, xh, xa, g;
            element(c, ds, du, xh, xa, g);
            const float w = a.w_post ? a.w_post[c] : 1.0f;
            const float z = fmaf(xa, w, a.b_post ? a.b_post[c] : 0.0f);
            if (a.dresidual) static_cast<T*>(a.dresidual)[row * a.ld_dresidual + c] = from_float<T>(a.rho * ds);
            if (a.gate_form == GATE_FULL)
                static_cast<T*>(a.dgate)[row * a.ld_dgate + c] = from_float<T>(du * z * slope(g, a.gate_act));
            static_cast<T*>(a.dbranch)[row * a.ld_dbranch + c] =
                from_float<T>(a.w_post ? st[1] * (du * g * w - k1 - xh * k0) : du * g);
        }
    }
}

// ---- launches

// Blocks loop over their rows, so there are as many as fit the 256 CUs at
// once: more would wait for the first ones to end.
int64_t resident_blocks(int waves_per_simd, int64_t cols)
{
    const int64_t waves = cols <= 64 * kCols ? kSubThreads / 64 : (cols + 64 * kCols - 1) / (64 * kCols);
    const int64_t per_cu = 4 * waves_per_simd / waves;
    return 256 * (per_cu > 0 ? per_cu : 1);
}

// Blocks of the backward pass: fewer where a block would have less than 8
// rows to write its column sums for (but 256 if there are the rows).
int64_t backward_blocks(int64_t groups, int64_t cols)
{
    int64_t blocks = resident_blocks(kBackwardWaves, cols);
    const int64_t eighth = groups / 8 > 256 ? groups / 8 : 256;
    if (blocks > eighth) blocks = eighth;
    return blocks < groups ? blocks : groups;
}

template <typename T, int SUB, int MAXT, bool GENERAL>
void launch_kernel(const NormArgs& a, int threads, bool backward, hipStream_t s)
{
    const int64_t rpb = SUB ? kSubThreads / (SUB ? SUB : 1) : 1;
    const int64_t groups = (a.rows + rpb - 1) / rpb;
    if (!backward) {
        const int64_t most = resident_blocks(GENERAL ? kForwardGeneralWaves : kForwardWaves<T>, a.cols);
        norm_forward<T, SUB, MAXT, GENERAL><<<static_cast<unsigned>(groups < most ? groups : most), threads, 0, s>>>(a);
    } else {
        const int blocks = static_cast<int>(backward_blocks(groups, a.cols));
        const size_t lds = GENERAL && SUB == 0 && MAXT == 512 ? 3 * sizeof(float) * kCols * threads : 0;
        norm_backward<T, SUB, MAXT, GENERAL><<<blocks, threads, lds, s>>>(a);
        launch_columns(a, blocks, GENERAL, s);
    }
}

template <typename T, int SUB, int MAXT>
hipError_t launch_layout(const NormArgs& a, int threads, bool backward, hipStream_t s)
{
    if (a.b_post || a.b_pre || a.gate_form == GATE_FULL) launch_kernel<T, SUB, MAXT, true>(a, threads, backward, s);
    else launch_kernel<T, SUB, MAXT, false>(a, threads, backward, s);
    return hipGetLastError();
}

template <typename T> hipError_t launch_type(const NormArgs& a, bool backward, hipStream_t s)
{
    // threads that a row needs
    const int need = (a.cols + kCols - 1) / kCols;
    if (need <= 8) return launch_layout<T, 8, kSubThreads>(a, kSubThreads, backward, s);
    if (need <= 16) return launch_layout<T, 16, kSubThreads>(a, kSubThreads, backward, s);
    if (need <= 32) return launch_layout<T, 32, kSubThreads>(a, kSubThreads, backward, s);
    if (need <= 64) return launch_layout<T, 64, kSubThreads>(a, kSubThreads, backward, s);
    const int threads = (need + 63) / 64 * 64;
    if (need <= 512) return launch_layout<T, 0, 512>(a, threads, backward, s);
    if (need <= 1024) return launch_layout<T, 0, 1024>(a, threads, backward, s);
    const int blocks = static_cast<int>(a.rows < 256 ? a.rows : 256);
    if (!backward) {
        norm_forward_loop<T><<<blocks, kLoopThreads, 0, s>>>(a);
    } else {
        norm_backward_loop<T><<<blocks, kLoopThreads, 0, s>>>(a);
        launch_columns(a, blocks, 1, s);
    }
    return hipGetLastError();
}

__global__ void norm_no_rows(NormArgs a)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    if (a.gate_form == GATE_CHANNEL && a.dgate) static_cast<float*>(a.dgate)[c] = 0.0f;
    if (a.dw_post) a.dw_post[c] = 0.0f;
    if (a.db_post) a.db_post[c] = 0.0f;
    if (a.dw_pre) a.dw_pre[c] = 0.0f;
    if (a.db_pre) a.db_pre[c] = 0.0f;
}

hipError_t launch(const NormArgs& a, int dtype, bool backward, hipStream_t s)
{
    if (dtype == DTYPE_F32) return launch_type<float>(a, backward, s);
    if (dtype == DTYPE_BF16) return launch_type<bf16>(a, backward, s);
    return launch_type<f16>(a, backward, s);
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int64_t cols)
{
    return sizeof(float) * kAcc * static_cast<size_t>(backward_blocks(rows, cols)) * static_cast<size_t>(cols);
}

hipError_t launch_norm_forward(const NormArgs& a, int dtype, hipStream_t s) { return launch(a, dtype, false, s); }

hipError_t launch_norm_backward(const NormArgs& a, int dtype, hipStream_t s)
{
    if (a.rows == 0) {
        norm_no_rows<<<(a.cols + 255) / 256, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    return launch(a, dtype, true, s);
}

}  // namespace fasgd
