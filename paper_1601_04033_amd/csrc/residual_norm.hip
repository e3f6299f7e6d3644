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
// Each row is read once into registers and stays there through its
// reductions; the next row's loads are issued before the first of them.  A
// thread keeps its columns over all its rows, so parameters are read once per
// block and the column sums stay in its registers, written once per block and
// joined in a fixed order by a second small kernel.
#include "client_kernels.hpp"

namespace fasgd {
namespace {

constexpr int kAcc = 4;             // column sums of the backward pass
constexpr int kMaxBlocks = 512;     // of the backward pass (its column sums: [kAcc][blocks][cols])
constexpr int kLoopThreads = 1024;  // threads per row where a row does not fit the registers

template <typename T> constexpr int kVec = 16 / static_cast<int>(sizeof(T));

// ---- sums over the lanes of a row

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// Sum over groups of LANES consecutive lanes, in every lane of the group.
template <int LANES> __device__ __forceinline__ float lane_sum(float x)
{
    if constexpr (LANES >= 2) x += dpp<0xB1>(x);        // quad_perm 1 0 3 2
    if constexpr (LANES >= 4) x += dpp<0x4E>(x);        // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) x += dpp<0x141>(x);       // row_half_mirror
    if constexpr (LANES >= 16) x += dpp<0x140>(x);      // row_mirror
    if constexpr (LANES >= 32) x += __shfl_xor(x, 16);
    if constexpr (LANES >= 64) x += __shfl_xor(x, 32);
    return x;
}

// Sums of N values over the threads of a row.  SUB > 0: SUB lanes hold a
// row.  SUB = 0: the block's threads do; the waves' sums pass through one of
// two LDS buffers taken in turn, so that one barrier per reduction is enough
// (a buffer is written again only after the other one's barrier).
template <int SUB, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*buf)[16][2], int& turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane_sum<SUB ? SUB : 64>(v[i]);
    if constexpr (SUB == 0) {
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
        float(*b)[2] = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) b[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.0f;
        for (int w = 0; w < waves; ++w) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += b[w][i];
        }
    }
}

__device__ __forceinline__ float activate(float g, int act)
{
    if (act == ACT_SIGMOID) return 1.0f / (1.0f + expf(-g));
    if (act == ACT_TANH) return tanhf(g);
    return g;
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

// Dropout factors of V elements from matrix index i on.
template <int V> __device__ __forceinline__ void drop_factors(const DropKey& k, int64_t i, float (&m)[V])
{
    const uint64_t chunk = static_cast<uint64_t>(k.chunk_base) + static_cast<uint64_t>(i >> 3);
    const int off = static_cast<int>(i & 7);
    uint32_t bits = keep_bits(k, chunk);
    if (off + V > 8) bits |= keep_bits(k, chunk + 1) << 8;
    bits >>= off;
#pragma unroll
    for (int j = 0; j < V; ++j) m[j] = (bits >> j) & 1 ? k.scale : 0.0f;
}

// Dropped elements are 0 whatever is dropped (0 times NaN would not be).
__device__ __forceinline__ float dropped(float x, float m) { return m == 0.0f ? 0.0f : x * m; }

// mean and 1 / sqrt(variance + eps) of a row held as NV vectors of V in d
// (0 beyond the row's end); d becomes d - mean there.  The variance is that
// of the centred values.
template <int SUB, int NV, int V>
__device__ __forceinline__ void row_stats(float (&d)[NV][V], const NormArgs& a, int t, int tpr, float& mean,
                                          float& rstd, float (*buf)[16][2], int& turn)
{
    mean = 0.0f;
    if (a.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += d[v][j];
        row_sum<SUB>(s, buf, turn);
        mean = s[0] / a.n_cols;      // divided, so that a row of one value has that mean
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int left = a.cols - (v * tpr + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) d[v][j] = j < left ? d[v][j] - mean : 0.0f;
        }
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < V; ++j) q[0] = fmaf(d[v][j], d[v][j], q[0]);
    row_sum<SUB>(q, buf, turn);
    rstd = 1.0f / sqrtf(q[0] / a.n_cols + a.eps);
}

// ---- forward

template <typename T, int SUB, int NV>
__global__ __launch_bounds__(SUB ? 256 : 512) void norm_forward(NormArgs a)
{
    constexpr int V = kVec<T>;
    __shared__ float buf[2][16][2];
    int turn = 0;
    const int tpr = SUB ? SUB : blockDim.x;
    const int t = SUB ? threadIdx.x % (SUB ? SUB : 1) : threadIdx.x;
    const int rpb = SUB ? 256 / (SUB ? SUB : 1) : 1;
    const int group = SUB ? threadIdx.x / (SUB ? SUB : 1) : 0;
    const T* branch = static_cast<const T*>(a.branch);
    const T* residual = static_cast<const T*>(a.residual);
    const T* gate = static_cast<const T*>(a.gate);
    float wp[NV][V], bp[NV][V], wn[NV][V], bn[NV][V];      // a channel gate is folded into wp and bp
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * tpr + t) * V;
        load_params<V>(a.w_post, c, a.cols, 1.0f, wp[v]);
        load_params<V>(a.b_post, c, a.cols, 0.0f, bp[v]);
        load_params<V>(a.w_pre, c, a.cols, 1.0f, wn[v]);
        load_params<V>(a.b_pre, c, a.cols, 0.0f, bn[v]);
        if (a.gate_form == GATE_CHANNEL) {
            float g[V];
            load_params<V>(static_cast<const float*>(a.gate), c, a.cols, 0.0f, g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float f = activate(g[j], a.gate_act);
                wp[v][j] *= f;
                bp[v][j] *= f;
            }
        }
    }
    Pack<T, V> x[NV], r[NV], g[NV];
    auto fetch = [&](int64_t row) {
        const int cols = row < a.rows ? a.cols : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * V;
            x[v] = load_cols<T, V>(branch + row * a.ld_branch, c, cols);
            if (residual) r[v] = load_cols<T, V>(residual + row * a.ld_residual, c, cols);
            if (a.gate_form == GATE_FULL) g[v] = load_cols<T, V>(gate + row * a.ld_gate, c, cols);
        }
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * rpb;
    fetch(static_cast<int64_t>(blockIdx.x) * rpb + group);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * rpb; base < a.rows; base += step) {
        const int64_t row = base + group;
        const int cols = row < a.rows ? a.cols : 0;
        float d[NV][V], res[NV][V], ga[NV][V];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                d[v][j] = to_float(x[v].v[j]);
                res[v][j] = residual ? a.rho * to_float(r[v].v[j]) : 0.0f;
                ga[v][j] = a.gate_form == GATE_FULL ? activate(to_float(g[v].v[j]), a.gate_act) : 1.0f;
            }
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW && row < a.rows)
            row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        fetch(row + step);
        float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
        if (a.w_post) row_stats<SUB>(d, a, t, tpr, mean1, rstd1, buf, turn);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * V;
            float m[V];
#pragma unroll
            for (int j = 0; j < V; ++j) m[j] = 1.0f;
            if (a.drop && c < cols) drop_factors<V>(a.key, row * a.cols + c, m);
            Pack<T, V> out;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float u = fmaf(d[v][j] * rstd1, wp[v][j], bp[v][j]) * (ga[v][j] * row_gate);
                if (a.drop) u = dropped(u, m[j]);
                out.v[j] = from_float<T>(res[v][j] + u);
                // the norm is of the sum as it is stored, so that the
                // backward pass, which reads it, differentiates this function
                d[v][j] = j < cols - c ? to_float(out.v[j]) : 0.0f;
            }
            store_cols<T, V>(static_cast<T*>(a.sum) + row * a.ld_sum, c, cols, out);
        }
        if (a.w_pre) {
            row_stats<SUB>(d, a, t, tpr, mean2, rstd2, buf, turn);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Pack<T, V> out;
#pragma unroll
                for (int j = 0; j < V; ++j) out.v[j] = from_float<T>(fmaf(d[v][j] * rstd2, wn[v][j], bn[v][j]));
                store_cols<T, V>(static_cast<T*>(a.normed) + row * a.ld_normed, (v * tpr + t) * V, cols, out);
            }
        }
        if (t == 0 && row < a.rows) {
            const float st[4] = {mean1, rstd1, mean2, rstd2};
            __builtin_memcpy(a.stats + row * 4, st, sizeof st);
        }
    }
}

// ---- backward

template <typename T, int SUB, int NV>
__global__ __launch_bounds__(SUB ? 256 : 512) void norm_backward(NormArgs a)
{
    constexpr int V = kVec<T>;
    __shared__ float buf[2][16][2];
    int turn = 0;
    const int tpr = SUB ? SUB : blockDim.x;
    const int t = SUB ? threadIdx.x % (SUB ? SUB : 1) : threadIdx.x;
    const int rpb = SUB ? 256 / (SUB ? SUB : 1) : 1;
    const int group = SUB ? threadIdx.x / (SUB ? SUB : 1) : 0;
    const T* branch = static_cast<const T*>(a.branch);
    const T* sum = static_cast<const T*>(a.sum);
    const T* gate = static_cast<const T*>(a.gate);
    const T* dsum = static_cast<const T*>(a.dsum);
    const T* dnormed = static_cast<const T*>(a.dnormed);
    float wp[NV][V], bp[NV][V], wn[NV][V], gc[NV][V];
    float post1[NV][V], post2[NV][V], pre1[NV][V], pre2[NV][V];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * tpr + t) * V;
        load_params<V>(a.w_post, c, a.cols, 1.0f, wp[v]);
        load_params<V>(a.b_post, c, a.cols, 0.0f, bp[v]);
        load_params<V>(a.w_pre, c, a.cols, 1.0f, wn[v]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            gc[v][j] = 1.0f;
            post1[v][j] = post2[v][j] = pre1[v][j] = pre2[v][j] = 0.0f;
        }
        if (a.gate_form == GATE_CHANNEL) {
            load_params<V>(static_cast<const float*>(a.gate), c, a.cols, 0.0f, gc[v]);
#pragma unroll
            for (int j = 0; j < V; ++j) gc[v][j] = activate(gc[v][j], a.gate_act);
        }
    }
    Pack<T, V> px[NV], ps[NV], pds[NV], pdh[NV], pg[NV];
    float st[4];
    auto fetch = [&](int64_t row) {
        const int cols = row < a.rows ? a.cols : 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * V;
            px[v] = load_cols<T, V>(branch + row * a.ld_branch, c, cols);
            if (a.w_pre) {
                ps[v] = load_cols<T, V>(sum + row * a.ld_sum, c, cols);
                pdh[v] = load_cols<T, V>(dnormed + row * a.ld_dnormed, c, cols);
            }
            if (dsum) pds[v] = load_cols<T, V>(dsum + row * a.ld_dsum, c, cols);
            if (a.gate_form == GATE_FULL) pg[v] = load_cols<T, V>(gate + row * a.ld_gate, c, cols);
        }
        if (cols) __builtin_memcpy(st, a.stats + row * 4, sizeof st);
        else st[0] = st[1] = st[2] = st[3] = 0.0f;
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * rpb;
    fetch(static_cast<int64_t>(blockIdx.x) * rpb + group);
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * rpb; base < a.rows; base += step) {
        const int64_t row = base + group;
        const int cols = row < a.rows ? a.cols : 0;
        const float mean1 = st[0], rstd1 = st[1], mean2 = st[2], rstd2 = st[3];
        float ds[NV][V], xh1[NV][V], q[NV][V], xh2[NV][V];
        float ga[NV][V];
        float two[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                ds[v][j] = dsum ? to_float(pds[v].v[j]) : 0.0f;
                xh1[v][j] = (to_float(px[v].v[j]) - mean1) * rstd1;
                ga[v][j] = a.gate_form == GATE_FULL ? activate(to_float(pg[v].v[j]), a.gate_act) : gc[v][j];
                if (a.w_pre) {
                    const float dh = to_float(pdh[v].v[j]);
                    xh2[v][j] = (to_float(ps[v].v[j]) - mean2) * rstd2;
                    q[v][j] = dh * wn[v][j];
                    pre1[v][j] = fmaf(dh, xh2[v][j], pre1[v][j]);
                    pre2[v][j] += dh;
                    two[0] = fmaf(q[v][j], xh2[v][j], two[0]);
                    two[1] += q[v][j];
                }
            }
        float row_gate = 1.0f;
        if (a.gate_form == GATE_ROW && row < a.rows)
            row_gate = activate(static_cast<const float*>(a.gate)[row], a.gate_act);
        fetch(row + step);
        if (a.w_pre) {
            row_sum<SUB>(two, buf, turn);
            const float m0 = two[0] * a.inv_cols, m1 = a.layer ? two[1] * a.inv_cols : 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) ds[v][j] = fmaf(rstd2, q[v][j] - m1 - xh2[v][j] * m0, ds[v][j]);
        }
        float dg_row[1] = {0.0f};
        two[0] = two[1] = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * tpr + t) * V;
            float m[V];
#pragma unroll
            for (int j = 0; j < V; ++j) m[j] = 1.0f;
            if (a.drop && c < cols) drop_factors<V>(a.key, row * a.cols + c, m);
            Pack<T, V> dr, dgp;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool in = j < cols - c;
                dr.v[j] = from_float<T>(a.rho * ds[v][j]);
                float du = in ? ds[v][j] : 0.0f;
                if (a.drop) du = dropped(du, m[j]);
                // what is dropped takes no part, were it infinite or NaN
                const float xa = a.drop && m[j] == 0.0f ? 0.0f : xh1[v][j];
                const float z = fmaf(xa, wp[v][j], bp[v][j]);
                if (a.gate_form == GATE_FULL) dgp.v[j] = from_float<T>(du * z * slope(ga[v][j], a.gate_act));
                if (a.gate_form == GATE_ROW) {
                    dg_row[0] = fmaf(du, z, dg_row[0]);
                    du *= row_gate;
                }
                // a channel gate's a is the column's own: its sums go without it
                const float dz = du * ga[v][j];
                const float acc = a.gate_form == GATE_CHANNEL ? du : dz;
                post1[v][j] = fmaf(acc, xa, post1[v][j]);
                post2[v][j] += acc;
                q[v][j] = dz * wp[v][j];
                two[0] = fmaf(q[v][j], xa, two[0]);
                two[1] += q[v][j];
            }
            if (a.dresidual) store_cols<T, V>(static_cast<T*>(a.dresidual) + row * a.ld_dresidual, c, cols, dr);
            if (a.gate_form == GATE_FULL) store_cols<T, V>(static_cast<T*>(a.dgate) + row * a.ld_dgate, c, cols, dgp);
        }
        if (a.w_post) row_sum<SUB>(two, buf, turn);
        if (a.gate_form == GATE_ROW) {
            row_sum<SUB>(dg_row, buf, turn);
            if (t == 0 && row < a.rows) static_cast<float*>(a.dgate)[row] = dg_row[0] * slope(row_gate, a.gate_act);
        }
        const float m0 = a.w_post ? two[0] * a.inv_cols : 0.0f;
        const float m1 = a.w_post && a.layer ? two[1] * a.inv_cols : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            Pack<T, V> out;
#pragma unroll
            for (int j = 0; j < V; ++j)
                out.v[j] = from_float<T>(a.w_post ? rstd1 * (q[v][j] - m1 - xh1[v][j] * m0) : q[v][j]);
            store_cols<T, V>(static_cast<T*>(a.dbranch) + row * a.ld_dbranch, (v * tpr + t) * V, cols, out);
        }
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
                store_cols<float, V>(out, (v * tpr + t) * V, a.cols, p);
            }
        } else {
            __shared__ float join[4][SUB * NV * V];
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float x = acc[v][j];
#pragma unroll
                    for (int lanes = SUB; lanes < 64; lanes *= 2) x += __shfl_xor(x, lanes);
                    if ((threadIdx.x & 63) < SUB) join[threadIdx.x >> 6][(v * SUB + t) * V + j] = x;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += 256)
                out[c] = (join[0][c] + join[1][c]) + (join[2][c] + join[3][c]);
        }
    };
    put(0, post1);
    put(1, post2);
    put(2, pre1);
    put(3, pre2);
}

// The column sums of `blocks` blocks joined in block order within each of
// the wave's slices and then slice by slice: a fixed order.
__global__ __launch_bounds__(1024) void norm_columns(NormArgs a, int blocks)
{
    __shared__ float part[kAcc][16][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    float s[kAcc] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < a.cols) {
        for (int b = slice; b < blocks; b += 16)
#pragma unroll
            for (int i = 0; i < kAcc; ++i) s[i] += a.partial[(static_cast<int64_t>(i) * blocks + b) * a.cols + c];
    }
#pragma unroll
    for (int i = 0; i < kAcc; ++i) part[i][slice][lane] = s[i];
    __syncthreads();
    if (slice != 0 || c >= a.cols) return;
#pragma unroll
    for (int i = 0; i < kAcc; ++i)
        for (int k = 1; k < 16; ++k) s[i] += part[i][k][lane];
    float f = 1.0f;
    if (a.gate_form == GATE_CHANNEL) {
        f = activate(static_cast<const float*>(a.gate)[c], a.gate_act);
        const float w = a.w_post ? a.w_post[c] : 1.0f, b = a.b_post ? a.b_post[c] : 0.0f;
        if (a.dgate) static_cast<float*>(a.dgate)[c] = slope(f, a.gate_act) * (w * s[0] + b * s[1]);
    }
    if (a.dw_post) a.dw_post[c] = f * s[0];
    if (a.db_post) a.db_post[c] = f * s[1];
    if (a.dw_pre) a.dw_pre[c] = s[2];
    if (a.db_pre) a.db_pre[c] = s[3];
}

// ---- rows too long for the registers: the same sums with the row read again

template <typename T> __global__ __launch_bounds__(kLoopThreads) void norm_forward_loop(NormArgs a)
{
    __shared__ float buf[2][16][2];
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
            if (a.drop) {
                float m[1];
                drop_factors<1>(a.key, row * a.cols + c, m);
                u = dropped(u, m[0]);
            }
            if (r) u += a.rho * to_float(r[c]);
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
    __shared__ float buf[2][16][2];
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
        // ds, du and the normed branch value of one element
        auto element = [&](int c, float& ds, float& du, float& xh1, float& xa) {
            ds = a.dsum ? to_float(static_cast<const T*>(a.dsum)[row * a.ld_dsum + c]) : 0.0f;
            if (a.w_pre) {
                const float xh = (to_float(s[c]) - st[2]) * st[3];
                ds = fmaf(st[3], to_float(dh[c]) * a.w_pre[c] - m1 - xh * m0, ds);
            }
            du = ds;
            xa = xh1 = (to_float(x[c]) - st[0]) * st[1];
            if (a.drop) {
                float m[1];
                drop_factors<1>(a.key, row * a.cols + c, m);
                du = dropped(du, m[0]);
                if (m[0] == 0.0f) xa = 0.0f;
            }
        };
        auto gate_of = [&](int c) {
            if (a.gate_form == GATE_CHANNEL) return activate(static_cast<const float*>(a.gate)[c], a.gate_act);
            if (a.gate_form == GATE_FULL)
                return activate(to_float(static_cast<const T*>(a.gate)[row * a.ld_gate + c]), a.gate_act);
            return row_gate;
        };
        float three[2] = {0.0f, 0.0f}, dg_row[1] = {0.0f};
        for (int c = threadIdx.x; c < a.cols; c += kLoopThreads) {
            float ds, du, xh, xa;
            element(c, ds, du, xh, xa);
            const float w = a.w_post ? a.w_post[c] : 1.0f, g = gate_of(c);
            const float z = fmaf(xa, w, a.b_post ? a.b_post[c] : 0.0f);
            if (a.gate_form == GATE_ROW) dg_row[0] = fmaf(du, z, dg_row[0]);
            const float own = a.gate_form == GATE_CHANNEL ? du : du * g;
            acc[0][c] = fmaf(own, xa, first ? 0.0f : acc[0][c]);
            acc[1][c] = own + (first ? 0.0f : acc[1][c]);
            float d = 0.0f, xh2 = 0.0f;
            if (a.w_pre) {
                d = to_float(dh[c]);
                xh2 = (to_float(s[c]) - st[2]) * st[3];
            }
            acc[2][c] = fmaf(d, xh2, first ? 0.0f : acc[2][c]);
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
            float ds, du, xh, xa;
            element(c, ds, du, xh, xa);
            const float w = a.w_post ? a.w_post[c] : 1.0f, g = gate_of(c);
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

template <typename T, int SUB, int NV>
hipError_t launch_form(const NormArgs& a, int threads, bool backward, hipStream_t s)
{
    const int64_t rpb = SUB ? 256 / (SUB ? SUB : 1) : 1;
    const int64_t need = (a.rows + rpb - 1) / rpb;
    if (!backward) {
        const int64_t most = 256 * (2048 / threads);
        norm_forward<T, SUB, NV><<<static_cast<unsigned>(need < most ? need : most), threads, 0, s>>>(a);
        return hipGetLastError();
    }
    const int blocks = static_cast<int>(need < kMaxBlocks ? need : kMaxBlocks);
    norm_backward<T, SUB, NV><<<blocks, threads, 0, s>>>(a);
    norm_columns<<<(a.cols + 63) / 64, 1024, 0, s>>>(a, blocks);
    return hipGetLastError();
}

template <typename T> hipError_t launch_type(const NormArgs& a, bool backward, hipStream_t s)
{
    const int nvec = (a.cols + kVec<T> - 1) / kVec<T>;
    if (nvec <= 8) return launch_form<T, 8, 1>(a, 256, backward, s);
    if (nvec <= 16) return launch_form<T, 16, 1>(a, 256, backward, s);
    if (nvec <= 32) return launch_form<T, 32, 1>(a, 256, backward, s);
    if (nvec <= 64) return launch_form<T, 64, 1>(a, 256, backward, s);
    // whole waves share a row: at most 8 of them
    const auto threads = [&](int nv) { return (nvec + 64 * nv - 1) / (64 * nv) * 64; };
    if (nvec <= 512) return launch_form<T, 0, 1>(a, threads(1), backward, s);
    if (nvec <= 1024) return launch_form<T, 0, 2>(a, threads(2), backward, s);
    if (nvec <= 2048) return launch_form<T, 0, 4>(a, threads(4), backward, s);
    const int blocks = static_cast<int>(a.rows < kMaxBlocks ? a.rows : kMaxBlocks);
    if (!backward) {
        norm_forward_loop<T><<<blocks, kLoopThreads, 0, s>>>(a);
    } else {
        norm_backward_loop<T><<<blocks, kLoopThreads, 0, s>>>(a);
        norm_columns<<<(a.cols + 63) / 64, 1024, 0, s>>>(a, blocks);
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
    const int64_t blocks = rows < kMaxBlocks ? rows : kMaxBlocks;
    return sizeof(float) * kAcc * static_cast<size_t>(blocks) * static_cast<size_t>(cols);
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
