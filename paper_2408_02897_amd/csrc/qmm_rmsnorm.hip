// qmm_rmsnorm_quantize and qmm_rmsnorm_backward: the root-mean-square norm in front of a quantized product, with the
// residual stream's addition before it and the quantization of its result (Eq. 1, one step size per token) behind it, and its
// backward pass.
//
// Forward, row i:  h = x + r rounded to the tensor's type (the residual stream as the next layer sees it),
//   rstd = 1 / sqrt(mean h^2 + eps),  y_j = (h_j w_j) rstd,  delta = max |y| / qmax,  codes = round(y fl(1 / delta)).
// y is rounded by the encoder alone: going through bfloat16 first would round twice.  Multiplying by rstd > 0 keeps order, rounding
// included, so max |y| is fl(max |h w| rstd): the sum and the maximum are one reduction, and a row is read once and
// held in registers in between.
// Backward:  a = w dy,  n = h rstd,  dx = rstd (a - n mean(a n)) + dr,  dw = sum over rows of dy n.
// A thread keeps its columns' share of dw in registers over all rows of its workgroup; the workgroups' shares are added by a second
// kernel in a fixed order, so dw does not depend on timing.
// All of it is bound by memory traffic.  bfloat16 16384 x 4096, back to back on changing tensors: forward with residual, h and y (604 MB) 100 us, 6.0 TB/s;
// backward with a residual's gradient (537 MB) 91 us, 5 of them the fold of dw, 5.9 TB/s; a plain copy of 1 GB runs at 6.0.  One row of 4096: 4 us,
// a launch and two trips to memory and back.
#include <type_traits>
#include "qmm_rows.h"

namespace qmm {
namespace {

struct NormArgs {
    const void* x; const void* r;              // r: the residual, or null
    int64_t x_batch, x_row, r_batch, r_row;    // strides in elements
    const void* w; int w_bf16;
    float eps;
    void* h; void* y; float* rstd;             // dense, or null
    float* delta; uint8_t* codes;
    int64_t batch, rows, cols;
    uint64_t seed, offset;
    float qmax; int fmt;
};

// 1 / sqrt(mean + eps), both operations correctly rounded
QMM_DEV float rstd_of(float sum, int64_t cols, float eps)
{
    const float mean = cols > 0 ? sum / (float)cols : 0.0f;
    return 1.0f / sqrtf(mean + eps);
}
// What the products h w are multiplied by: 1 / rms.  A row without any (all zero: m, their largest magnitude, is 0) stays what it is where the root is zero
// too (eps = 0), whose reciprocal times zero would be no number.
QMM_DEV float factor_of(float rstd, uint32_t m) { return m == 0u ? 1.0f : rstd; }
// A row whose squares are beyond binary32 has rstd 0 and is zero, unless an element is infinite.  Where h w is beyond binary32 as well, m = infinity does not tell
// the two apart: the kernels then look at h and w again, each lane at the elements that it has read or written (elements c .. end - 1; one by one, so that
// this costs the other rows nothing: with vectors, or h kept in registers for it, ten registers more).
constexpr uint32_t kInfBits = 0x7F800000u;
template <typename T> QMM_DEV bool finite_elements(const T* h, const void* w, int w_bf16, int c, int end)
{
    uint32_t m = 0;
#pragma unroll 1
    for (; c < end; ++c) {
        m = max(m, mag_bits<T>(h[c]));
        if (w) m = max(m, w_bf16 ? mag_bits<uint16_t>(static_cast<const uint16_t*>(w)[c]) : mag_bits<float>(static_cast<const float*>(w)[c]));
    }
    return m < kInfBits;
}

// Rows of up to kRowElements: LPR lanes hold one, NV vectors a lane.
// STREAM: x and r are read, h and y written past the caches (host).
template <typename T, int MODE, int LPR, int NV, bool STREAM> __global__ void __launch_bounds__(LPR > 256 ? LPR : 256)
rmsnorm_rows(NormArgs a)
{
    constexpr int V = Vec<T>::V, THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
    __shared__ typename RowReduce<LPR>::Shared sh;
    const int64_t total = a.batch * a.rows;
    const int c0 = (int)(threadIdx.x % LPR) * V;
    int turn = 0;
    for (int64_t blk = blockIdx.x; blk * RPB < total; blk += gridDim.x, turn ^= 1) {
        const int64_t id = blk * RPB + threadIdx.x / LPR;
        const bool live = id < total;
        const int64_t b = live && a.batch > 1 ? id / a.rows : 0, i = live ? id - b * a.rows : 0;
        const int cols = live ? (int)a.cols : 0;
        const T* x = static_cast<const T*>(a.x) + b * a.x_batch + i * a.x_row;
        u32x4 w[NV];
        Weights weight[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) weight[k] = fetch_weights<V>(a.w, a.w_bf16, c0 + k * LPR * V, cols);
#pragma unroll
        for (int k = 0; k < NV; ++k) w[k] = fetch_row<T, LPR == 8, STREAM>(x, c0 + k * LPR * V, cols);
        if (a.r) {
            const T* r = static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row;
            T* h = static_cast<T*>(a.h) + id * a.cols;
            u32x4 q[NV];
#pragma unroll
            for (int k = 0; k < NV; ++k) q[k] = fetch_row<T, LPR == 8, STREAM>(r, c0 + k * LPR * V, cols);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                // (both shifted alike: the sum of the vectors is the vector of the sums)
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = Vec<T>::at(w[k], e) + Vec<T>::at(q[k], e);
                w[k] = settle_row<T, LPR == 8, STREAM>(pack_row<T>(v), c0 + k * LPR * V, cols);
                put_row<T, STREAM>(h + c0 + k * LPR * V, w[k], cols - c0 - k * LPR * V);
            }
        }
        else {
#pragma unroll
            for (int k = 0; k < NV; ++k) w[k] = settle_row<T, LPR == 8, STREAM>(w[k], c0 + k * LPR * V, cols);
        }
        float y[NV][V], sum = 0.0f;
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            weight_values<V>(weight[k], a.w, a.w_bf16, c0 + k * LPR * V, cols, y[k]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float h = Vec<T>::at(w[k], e);
                sum = fmaf(h, h, sum);
                y[k][e] *= h;
                m = max(m, mag_bits(y[k][e]));
            }
        }
        RowReduce<LPR>::run(sum, m, sh, turn);
        if (!live) continue;                                 // (LPR > 64: never, a workgroup's only row is live)
        const float rstd = rstd_of(sum, a.cols, a.eps);
        if (rstd == 0.0f && m == kInfBits) {
            bool finite = true;
#pragma unroll 1
            for (int k = 0; k < NV; ++k)
                finite &= finite_elements<T>(a.r ? static_cast<const T*>(a.h) + id * a.cols : x, a.w, a.w_bf16, c0 + k * LPR * V, min(c0 + k * LPR * V + V, cols));
            m = finite ? 0u : kInfBits;
            if constexpr (LPR > kWave) __syncthreads();      // the words of the reduction above have been read
            RowReduce<LPR>::run(sum, m, sh, turn);
            if (m == 0u) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) y[k][e] = 0.0f;
            }
        }
        const float factor = factor_of(rstd, m);
        const float d = delta_from_absmax_bits(mag_bits(__uint_as_float(m) * factor), a.qmax);
        if (threadIdx.x % LPR == 0) {
            a.delta[id] = d;
            if (a.rstd) a.rstd[id] = rstd;
        }
        const float rho = 1.0f / d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V, left = cols - c;
            if (left <= 0) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) y[k][e] *= factor;
            const int64_t p = id * a.cols + c;
            if (a.y) put_row<T, STREAM>(static_cast<T*>(a.y) + p, pack_row<T>(y[k]), left);
            store_row_codes<T>(a.codes + p, encode_values<V, MODE>(y[k], rho, a.fmt, (uint64_t)p + a.offset, a.seed), left);
        }
    }
}

// Longer rows: a workgroup goes over its row twice, the second time out of the L2.
template <typename T, int MODE> __global__ void __launch_bounds__(kRowLanes)
rmsnorm_long(NormArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ typename RowReduce<kRowLanes>::Shared sh;
    const int64_t total = a.batch * a.rows;
    int turn = 0;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x, turn ^= 1) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const T* x = static_cast<const T*>(a.x) + b * a.x_batch + i * a.x_row;
        const T* r = a.r ? static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row : nullptr;
        T* h = a.r ? static_cast<T*>(a.h) + id * a.cols : nullptr;
        float sum = 0.0f;
        uint32_t m = 0;
        for (int64_t c = (int64_t)threadIdx.x * V; c < a.cols; c += kRowLanes * V) {
            const int left = (int)min((int64_t)V, a.cols - c);
            u32x4 w = load_row<T>(x, (int)c, (int)a.cols);
            if (r) {
                const u32x4 q = load_row<T>(r, (int)c, (int)a.cols);
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = Vec<T>::at(w, e) + Vec<T>::at(q, e);
                w = pack_row<T>(v);
                store_row<T>(h + c, w, left);
            }
            float y[V];
            load_weight<V>(a.w, a.w_bf16, (int)c, (int)a.cols, y);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v = Vec<T>::at(w, e);
                sum = fmaf(v, v, sum);
                m = max(m, mag_bits(v * y[e]));
            }
        }
        RowReduce<kRowLanes>::run(sum, m, sh, turn);
        const float rstd = rstd_of(sum, a.cols, a.eps);
        const T* src = h ? h : x;                            // a thread's own stores where there is a residual
        bool zero = false;
        if (rstd == 0.0f && m == kInfBits) {
            bool finite = true;
            for (int64_t c = (int64_t)threadIdx.x * V; c < a.cols; c += kRowLanes * V)
                finite &= finite_elements<T>(src, a.w, a.w_bf16, (int)c, (int)min(c + V, a.cols));
            m = finite ? 0u : kInfBits;
            __syncthreads();
            RowReduce<kRowLanes>::run(sum, m, sh, turn);
            zero = m == 0u;
        }
        const float factor = factor_of(rstd, m);
        const float d = delta_from_absmax_bits(mag_bits(__uint_as_float(m) * factor), a.qmax);
        if (threadIdx.x == 0) {
            a.delta[id] = d;
            if (a.rstd) a.rstd[id] = rstd;
        }
        const float rho = 1.0f / d;
        for (int64_t c = (int64_t)threadIdx.x * V; c < a.cols; c += kRowLanes * V) {
            const int left = (int)min((int64_t)V, a.cols - c);
            const u32x4 w = load_row<T>(src, (int)c, (int)a.cols);
            float y[V];
            load_weight<V>(a.w, a.w_bf16, (int)c, (int)a.cols, y);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = zero ? 0.0f : (Vec<T>::at(w, e) * y[e]) * factor;
            const int64_t p = id * a.cols + c;
            if (a.y) store_row<T>(static_cast<T*>(a.y) + p, pack_row<T>(y), left);
            store_row_codes<T>(a.codes + p, encode_values<V, MODE>(y, rho, a.fmt, (uint64_t)p + a.offset, a.seed), left);
        }
    }
}

struct NormGradArgs {
    const void* dy; const void* h; const void* r;      // r: the gradient that reaches h past the norm, or null
    int64_t dy_batch, dy_row, h_batch, h_row, r_batch, r_row;
    const float* rstd;
    const void* w; int w_bf16;
    void* dx;
    float* partial;                                    // [gridDim.x][cols] shares of dw, or null
    float* dw;
    int64_t batch, rows, cols;
    int64_t shares;                                    // of them
};

// A thread's next row is on its way while it works on the current one; workgroups of 1024 threads, whose threads have 128 registers, do without,
// and fetch the weights anew for every row.
// STREAM: dy, h and r are read past the caches (host).
template <typename T, int LPR, int NV, bool STREAM> __global__ void __launch_bounds__(LPR > 256 ? LPR : 256)
rmsnorm_grad_rows(NormGradArgs a)
{
    constexpr int V = Vec<T>::V, THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
    constexpr bool AHEAD = LPR < 1024;
    __shared__ typename RowReduce<LPR>::Shared sh;
    __shared__ float s_dw[RPB > 1 ? RPB : 1][RPB > 1 ? LPR * NV * V : 1];
    const int64_t total = a.batch * a.rows;
    const int c0 = (int)(threadIdx.x % LPR) * V;
    float weight[NV][V], dw[NV][V];
    auto load_weights = [&]() {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_weight<V>(a.w, a.w_bf16, c0 + k * LPR * V, (int)a.cols, weight[k]);
    };
    if constexpr (AHEAD) load_weights();
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[k][e] = 0.0f;
    struct Row { u32x4 g[NV], w[NV], q[NV]; float rstd; };      // dy, h, dresidual
    auto fetch = [&](int64_t blk, Row& r) {
        const int64_t id = blk * RPB + threadIdx.x / LPR;
        const bool live = id < total;
        const int64_t b = live && a.batch > 1 ? id / a.rows : 0, i = live ? id - b * a.rows : 0;
        const int cols = live ? (int)a.cols : 0;
        const T* dy = static_cast<const T*>(a.dy) + b * a.dy_batch + i * a.dy_row;
        const T* h = static_cast<const T*>(a.h) + b * a.h_batch + i * a.h_row;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            r.g[k] = fetch_row<T, LPR == 8, STREAM>(dy, c, cols);
            r.w[k] = fetch_row<T, LPR == 8, STREAM>(h, c, cols);
            r.q[k] = u32x4{0u, 0u, 0u, 0u};
            if (a.r) r.q[k] = fetch_row<T, LPR == 8, STREAM>(static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row, c, cols);
        }
        r.rstd = live ? a.rstd[id] : 0.0f;
    };
    Row row;
    if (AHEAD && (int64_t)blockIdx.x * RPB < total) fetch(blockIdx.x, row);
    int turn = 0;
    for (int64_t blk = blockIdx.x; blk * RPB < total; blk += gridDim.x, turn ^= 1) {
        const int64_t id = blk * RPB + threadIdx.x / LPR;
        const int cols = id < total ? (int)a.cols : 0;
        Row next;
        if constexpr (AHEAD) { if ((blk + gridDim.x) * RPB < total) fetch(blk + gridDim.x, next); }
        else { fetch(blk, row); load_weights(); }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            row.g[k] = settle_row<T, LPR == 8, STREAM>(row.g[k], c, cols); row.w[k] = settle_row<T, LPR == 8, STREAM>(row.w[k], c, cols); row.q[k] = settle_row<T, LPR == 8, STREAM>(row.q[k], c, cols);
        }
        const float rstd = row.rstd;
        float sum = 0.0f;
        uint32_t none = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = Vec<T>::at(row.g[k], e), n = Vec<T>::at(row.w[k], e) * rstd;
                sum = fmaf(d * weight[k][e], n, sum);
                dw[k][e] = fmaf(d, n, dw[k][e]);
            }
        RowReduce<LPR>::run(sum, none, sh, turn);
        const float mean = sum / (float)a.cols;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V, left = cols - c;
            if (left <= 0) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float n = Vec<T>::at(row.w[k], e) * rstd;
                v[e] = fmaf(rstd, fmaf(-n, mean, Vec<T>::at(row.g[k], e) * weight[k][e]), Vec<T>::at(row.q[k], e));
            }
            store_row<T>(static_cast<T*>(a.dx) + id * a.cols + c, pack_row<T>(v), left);
        }
        if constexpr (AHEAD) row = next;
    }
    if (!a.partial) return;
    if constexpr (RPB > 1) {
        // the workgroup's rows side by side: added in order
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) s_dw[threadIdx.x / LPR][c0 + k * LPR * V + e] = dw[k][e];
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += THREADS) {
            float s = 0.0f;
#pragma unroll
            for (int q = 0; q < RPB; ++q) s += s_dw[q][c];
            a.partial[(int64_t)blockIdx.x * a.cols + c] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
#pragma unroll
            for (int q = 0; q < V / 4; ++q)
                store_row<float>(a.partial + (int64_t)blockIdx.x * a.cols + c + 4 * q, pack_row<float>(dw[k] + 4 * q), (int)a.cols - c - 4 * q);
        }
    }
}

// Longer rows: dx by workgroups that go over their row twice, the shares of dw by another pass down the columns.
template <typename T> __global__ void __launch_bounds__(kRowLanes)
rmsnorm_grad_long(NormGradArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ typename RowReduce<kRowLanes>::Shared sh;
    const int64_t total = a.batch * a.rows;
    int turn = 0;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x, turn ^= 1) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const T* dy = static_cast<const T*>(a.dy) + b * a.dy_batch + i * a.dy_row;
        const T* h = static_cast<const T*>(a.h) + b * a.h_batch + i * a.h_row;
        const T* r = a.r ? static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row : nullptr;
        const float rstd = a.rstd[id];
        float sum = 0.0f;
        uint32_t none = 0;
        for (int64_t c = (int64_t)threadIdx.x * V; c < a.cols; c += kRowLanes * V) {
            const u32x4 g = load_row<T>(dy, (int)c, (int)a.cols), w = load_row<T>(h, (int)c, (int)a.cols);
            float weight[V];
            load_weight<V>(a.w, a.w_bf16, (int)c, (int)a.cols, weight);
#pragma unroll
            for (int e = 0; e < V; ++e) sum = fmaf(Vec<T>::at(g, e) * weight[e], Vec<T>::at(w, e) * rstd, sum);
        }
        RowReduce<kRowLanes>::run(sum, none, sh, turn);
        const float mean = sum / (float)a.cols;
        for (int64_t c = (int64_t)threadIdx.x * V; c < a.cols; c += kRowLanes * V) {
            const int left = (int)min((int64_t)V, a.cols - c);
            const u32x4 g = load_row<T>(dy, (int)c, (int)a.cols), w = load_row<T>(h, (int)c, (int)a.cols);
            const u32x4 q = r ? load_row<T>(r, (int)c, (int)a.cols) : u32x4{0u, 0u, 0u, 0u};
            float weight[V], v[V];
            load_weight<V>(a.w, a.w_bf16, (int)c, (int)a.cols, weight);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float n = Vec<T>::at(w, e) * rstd;
                v[e] = fmaf(rstd, fmaf(-n, mean, Vec<T>::at(g, e) * weight[e]), Vec<T>::at(q, e));
            }
            store_row<T>(static_cast<T*>(a.dx) + id * a.cols + c, pack_row<T>(v), left);
        }
    }
}
template <typename T> __global__ void __launch_bounds__(kThreads)
rmsnorm_grad_columns(NormGradArgs a)                   // grid (columns, shares): every share-th row
{
    constexpr int V = Vec<T>::V;
    const int64_t total = a.batch * a.rows;
    const int64_t c = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * V;
    if (c >= a.cols) return;
    const int left = (int)min((int64_t)V, a.cols - c);
    float dw[V] = {};
    for (int64_t id = blockIdx.y; id < total; id += gridDim.y) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const u32x4 g = load_row<T>(static_cast<const T*>(a.dy) + b * a.dy_batch + i * a.dy_row, (int)c, (int)a.cols);
        const u32x4 w = load_row<T>(static_cast<const T*>(a.h) + b * a.h_batch + i * a.h_row, (int)c, (int)a.cols);
        const float rstd = a.rstd[id];
#pragma unroll
        for (int e = 0; e < V; ++e) dw[e] = fmaf(Vec<T>::at(g, e), Vec<T>::at(w, e) * rstd, dw[e]);
    }
#pragma unroll
    for (int q = 0; q < V / 4; ++q)
        store_row<float>(a.partial + (int64_t)blockIdx.y * a.cols + c + 4 * q, pack_row<float>(dw + 4 * q), left - 4 * q);
}

// dw = the sum of the shares, in an order fixed by their number: a workgroup takes 16 columns, sixty-four lanes a column every sixty-fourth share each.
// (64 columns and sixteen lanes a column, a quarter of the workgroups: 512 shares of 1000 columns 3.9 us, of 4096 4.8.)
__global__ void __launch_bounds__(1024)
rmsnorm_grad_fold(NormGradArgs a)
{
    constexpr int C = 16, L = 1024 / C;
    __shared__ float part[L][C + 1];
    const int c_in = threadIdx.x % C, l = threadIdx.x / C;
    const int64_t c = (int64_t)blockIdx.x * C + c_in;
    float s = 0.0f;
    if (c < a.cols) {
#pragma unroll 8
        for (int64_t p = l; p < a.shares; p += L) s += a.partial[p * a.cols + c];
    }
    part[l][c_in] = s;
    __syncthreads();
    if (threadIdx.x < kWave) {                               // four lanes a column
        const int k = threadIdx.x % C, first = threadIdx.x / C * (L / 4);
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < L / 4; ++i) s += part[first + i][k];
        s += __shfl_xor(s, 16, kWave);
        s += __shfl_xor(s, 32, kWave);
        const int64_t f = (int64_t)blockIdx.x * C + k;
        if (threadIdx.x < C && f < a.cols) a.dw[f] = s;
    }
}

// Shares of dw: workgroups that go over rows, of columns' parts of rows where rows are long.  Two workgroups a CU, one of 1024 threads: enough to keep
// the rows coming, and every further one is a share more to write and fold (bfloat16 16384 x 4096, 256 / 384 / 512 / 768 / 1024 workgroups 135 / 109 / 104 / 108 /
// 119 us; binary32 1000 x 12000, 1024 threads, 256 / 512: 53 / 61).  Where up to four would work one does, and its share is dw: no fold, no workspace.
int64_t shares_of(const qmm_tensor* t)
{
    const int64_t total = t->batch * t->rows;
    if (t->cols > kRowElements) return total <= 4 ? 1 : std::min<int64_t>(total, 64);
    int64_t blocks = 0, most = 512;
    auto count = [&](auto lpr, auto) {
        constexpr int rpb = lpr.value < 256 ? 256 / lpr.value : 1;
        blocks = (total + rpb - 1) / rpb;
        if (lpr.value == 1024) most = 256;
    };
    if (t->dtype == QMM_DT_BF16) for_row_size<uint16_t>(t->cols, count); else for_row_size<float>(t->cols, count);
    return blocks <= 4 ? 1 : std::min(blocks, most);
}

template <typename T, int MODE> qmm_status launch_norm(const NormArgs& a, bool stream, hipStream_t s)
{
    const int64_t total = a.batch * a.rows;
    if (a.cols > kRowElements) rmsnorm_long<T, MODE><<<row_blocks(total, 1), kRowLanes, 0, s>>>(a);
    else for_row_size<T>(a.cols, [&](auto lpr, auto nv) {
        constexpr int threads = lpr.value > 256 ? lpr.value : 256;
        if constexpr (lpr.value >= kWave) {
            if (stream) { rmsnorm_rows<T, MODE, lpr.value, nv.value, true><<<row_blocks(total, threads / lpr.value), threads, 0, s>>>(a); return; }
        }
        rmsnorm_rows<T, MODE, lpr.value, nv.value, false><<<row_blocks(total, threads / lpr.value), threads, 0, s>>>(a);
    });
    return launch_status();
}
template <typename T> qmm_status launch_norm_grad(NormGradArgs& a, bool stream, hipStream_t s)
{
    const int64_t total = a.batch * a.rows;
    if (a.cols > kRowElements) {
        // (down the columns first: dx may be written over dy)
        if (a.partial) {
            const unsigned strips = (unsigned)((a.cols + kThreads * Vec<T>::V - 1) / (kThreads * Vec<T>::V));
            rmsnorm_grad_columns<T><<<dim3(strips, (unsigned)a.shares), kThreads, 0, s>>>(a);
        }
        rmsnorm_grad_long<T><<<row_blocks(total, 1), kRowLanes, 0, s>>>(a);
    } else {
        for_row_size<T>(a.cols, [&](auto lpr, auto nv) {
            constexpr int threads = lpr.value > 256 ? lpr.value : 256;
            if constexpr (lpr.value >= kWave) {
                if (stream) { rmsnorm_grad_rows<T, lpr.value, nv.value, true><<<(unsigned)a.shares, threads, 0, s>>>(a); return; }
            }
            rmsnorm_grad_rows<T, lpr.value, nv.value, false><<<(unsigned)a.shares, threads, 0, s>>>(a);
        });
    }
    if (a.partial && a.partial != a.dw) {
        if (hipGetLastError() != hipSuccess) return QMM_ERR_LAUNCH;
        rmsnorm_grad_fold<<<(unsigned)((a.cols + 15) / 16), 1024, 0, s>>>(a);
    }
    return launch_status();
}

}  // namespace
}  // namespace qmm

using namespace qmm;

extern "C" qmm_status qmm_rmsnorm_quantize(const qmm_tensor* x, const qmm_tensor* residual, const void* weight, qmm_dtype weight_dtype, float eps,
                                           qmm_format fmt, qmm_round mode, uint64_t seed, uint64_t offset, void* h_out, void* y_out,
                                           float* rstd_out, float* delta_out, uint8_t* codes_out, void* stream)
{
    if (!x) return QMM_ERR_NULL;
    qmm_status st = check_rows(x);
    if (st != QMM_OK) return st;
    if (residual) {
        st = check_rows(residual);
        if (st != QMM_OK) return st;
        if (!same_extent(x, residual)) return QMM_ERR_SHAPE;
        if (residual->dtype != x->dtype) return QMM_ERR_UNSUPPORTED;
    }
    if (weight_dtype != QMM_DT_BF16 && weight_dtype != QMM_DT_F32) return QMM_ERR_ENUM;
    if (fmt != QMM_FMT_INT8 && fmt != QMM_FMT_E4M3 && fmt != QMM_FMT_E5M2) return QMM_ERR_ENUM;
    if (mode != QMM_ROUND_RTNE && mode != QMM_ROUND_STOCHASTIC) return QMM_ERR_ENUM;
    if (!(eps >= 0.0f && eps <= 3.402823466e38f)) return QMM_ERR_SHAPE;
    if (x->batch * x->rows == 0) return QMM_OK;
    if (!delta_out) return QMM_ERR_NULL;
    if (x->cols > 0 && (!x->data || !codes_out || (residual && (!residual->data || !h_out)))) return QMM_ERR_NULL;
    if (!element_aligned(x->data, x->dtype) || (residual && !element_aligned(residual->data, x->dtype)) || !element_aligned(h_out, x->dtype) ||
        !element_aligned(y_out, x->dtype) || !element_aligned(weight, weight_dtype) || !element_aligned(delta_out, QMM_DT_F32) ||
        !element_aligned(rstd_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    for (const void* out : {static_cast<const void*>(h_out), static_cast<const void*>(y_out)})      // over an input: element by element only
        if (out && ((out == x->data && !dense(x)) || (residual && out == residual->data && !dense(residual)))) return QMM_ERR_SHAPE;

    if (h_out && h_out == y_out && x->cols > 0) return QMM_ERR_SHAPE;

    NormArgs a{};
    a.x = x->data; a.x_batch = x->batch_stride; a.x_row = x->row_stride;
    if (residual) { a.r = residual->data; a.r_batch = residual->batch_stride; a.r_row = residual->row_stride; a.h = h_out; }
    a.w = weight; a.w_bf16 = weight_dtype == QMM_DT_BF16; a.eps = eps;
    a.y = y_out; a.rstd = rstd_out; a.delta = delta_out; a.codes = codes_out;
    a.batch = x->batch; a.rows = x->rows; a.cols = x->cols;
    a.seed = seed; a.offset = offset; a.qmax = host_qmax(fmt); a.fmt = fmt;
    if (a.cols == 0) a.r = nullptr;
    // The old residual stream is not read again, h is wanted by the next addition to it, y by the backward pass: where they are large they would fill the
    // caches for nothing and go past them; the codes, which the next product reads, do not (bfloat16 16384 x 4096 with y 115 -> 102 us, 8192 x 8192 97 -> 86;
    // 16384 x 1024, 33 MB, 22.5 -> 25.1).
    const bool streaming = residual && streams(x) && streams(residual) && aligned16(h_out) && aligned16(y_out);
    hipStream_t s = as_stream(stream);
    if (x->dtype == QMM_DT_BF16)
        return mode == QMM_ROUND_RTNE ? launch_norm<uint16_t, QMM_ROUND_RTNE>(a, streaming, s) : launch_norm<uint16_t, QMM_ROUND_STOCHASTIC>(a, streaming, s);
    return mode == QMM_ROUND_RTNE ? launch_norm<float, QMM_ROUND_RTNE>(a, streaming, s) : launch_norm<float, QMM_ROUND_STOCHASTIC>(a, streaming, s);
}

extern "C" size_t qmm_rmsnorm_backward_workspace_size(const qmm_tensor* dy)
{
    if (!dy || check_rows(dy) != QMM_OK || dy->batch * dy->rows * dy->cols == 0) return 0;
    const int64_t shares = shares_of(dy);
    return shares > 1 ? (size_t)shares * (size_t)dy->cols * sizeof(float) : 0;
}

extern "C" qmm_status qmm_rmsnorm_backward(const qmm_tensor* dy, const qmm_tensor* h, const float* rstd, const void* weight, qmm_dtype weight_dtype,
                                           const qmm_tensor* dresidual, void* dx_out, float* dw_out, void* workspace, size_t workspace_bytes,
                                           void* stream)
{
    if (!dy || !h) return QMM_ERR_NULL;
    for (const qmm_tensor* t : {dy, h, dresidual}) {
        if (!t) continue;
        const qmm_status st = check_rows(t);
        if (st != QMM_OK) return st;
        if (!same_extent(dy, t)) return QMM_ERR_SHAPE;
        if (t->dtype != dy->dtype) return QMM_ERR_UNSUPPORTED;
    }
    if (weight_dtype != QMM_DT_BF16 && weight_dtype != QMM_DT_F32) return QMM_ERR_ENUM;
    if (dy->cols == 0) return QMM_OK;
    NormGradArgs a{};
    a.batch = dy->batch; a.rows = dy->rows; a.cols = dy->cols;
    const bool empty = dy->batch * dy->rows == 0;
    if (!empty && (!dy->data || !h->data || !rstd || !dx_out || (dresidual && !dresidual->data))) return QMM_ERR_NULL;
    for (const qmm_tensor* t : {dy, h, dresidual}) {
        if (!t) continue;
        if (!element_aligned(t->data, t->dtype)) return QMM_ERR_ALIGN;
        if (dx_out && dx_out == t->data && !dense(t)) return QMM_ERR_SHAPE;
    }
    if (!element_aligned(dx_out, dy->dtype) || !element_aligned(weight, weight_dtype) || !element_aligned(rstd, QMM_DT_F32) ||
        !element_aligned(dw_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    if (dw_out && !empty) {
        const size_t need = qmm_rmsnorm_backward_workspace_size(dy);
        a.partial = dw_out;                                  // a single share
        if (need > 0) {
            if (!workspace || workspace_bytes < need) return QMM_ERR_WORKSPACE;
            if (!aligned16(workspace)) return QMM_ERR_ALIGN;
            a.partial = static_cast<float*>(workspace);
        }
    }
    a.dw = dw_out;
    hipStream_t s = as_stream(stream);
    if (empty) {                                             // no rows: dw is a sum of none
        if (dw_out) rmsnorm_grad_fold<<<(unsigned)((a.cols + 15) / 16), 1024, 0, s>>>(a);
        return launch_status();
    }
    a.shares = shares_of(dy);
    a.dy = dy->data; a.dy_batch = dy->batch_stride; a.dy_row = dy->row_stride;
    a.h = h->data; a.h_batch = h->batch_stride; a.h_row = h->row_stride;
    if (dresidual) { a.r = dresidual->data; a.r_batch = dresidual->batch_stride; a.r_row = dresidual->row_stride; }
    a.rstd = rstd; a.w = weight; a.w_bf16 = weight_dtype == QMM_DT_BF16; a.dx = dx_out;
    const bool streaming = streams(dy) && streams(h) && (!dresidual || streams(dresidual));       // (bfloat16 16384 x 4096 104 -> 95 us, 8192 x 8192 112 -> 108)
    return dy->dtype == QMM_DT_BF16 ? launch_norm_grad<uint16_t>(a, streaming, s) : launch_norm_grad<float>(a, streaming, s);
}
