// qmm_layernorm_quantize and qmm_layernorm_backward: what a BERT layer has behind each of its two blocks -- dropout of the block's result, addition to the residual
// stream, layer norm -- with the quantization (Eq. 1) of the norm's result for the next product behind it, and its backward pass.
//
// Forward, row i:  h = x kept / (1 - p) + r, one rounding to binary32 and one to the tensor's type;  mean = sum h / n;
//   with d = h - mean and c = sum d / n (what the rounding of the sum left of the mean):  rstd = 1 / sqrt(sum d^2 / n - c^2 + eps),
//   v = (d - c) rstd,  y = v w + b (one rounding),  delta = max |y| / qmax over the row or over each 128 columns of it,  codes = round(y fl(1 / delta)).
// The mean comes first and the squares are those of the differences, so a row far from zero keeps its variance; the row stays in registers in between.
// Backward:  n = (h - mean) rstd,  a = w dy,  dh = rstd (a - mean(a) - n mean(a n)) + dr,  dx = dh kept / (1 - p),  dw = sum over rows of dy n,  db = sum of dy.
// The decisions of dropout are computed again.  A thread keeps its columns' shares of dw and db in registers over all rows of its workgroup; the
// workgroups' shares are added by a second kernel in a fixed order.
#include <type_traits>
#include "qmm_blocks.h"
#include "qmm_dropout.h"

namespace qmm {
namespace {

struct LayerArgs {
    const void* x; const void* r;              // r: the residual, or null
    int64_t x_batch, x_row, r_batch, r_row;    // strides in elements
    const void* w; const void* bias; int w_bf16;
    float eps;
    Drop drop;
    void* h; void* y; float* mean; float* rstd;        // dense, or null
    float* delta; uint8_t* codes;              // delta null: no codes
    int64_t batch, rows, cols;
    uint64_t seed, offset;
    float qmax; int fmt;
};

// Sums of two values and a maximum over the LPR lanes that hold a row; above 64 lanes over the workgroup.
template <int LPR> struct RowSums {
    static constexpr int WAVES = LPR > kWave ? LPR / kWave : 1, IN_WAVE = LPR > kWave ? kWave : LPR;
    struct Shared { float s[WAVES], t[WAVES]; };
    static QMM_DEV void run(float& s, float& t, Shared& sh)
    {
        s = over_lanes<IN_WAVE>(s, Plus());
        t = over_lanes<IN_WAVE>(t, Plus());
        if constexpr (LPR > kWave) {
            if ((threadIdx.x & (kWave - 1)) == 0) { sh.s[threadIdx.x / kWave] = s; sh.t[threadIdx.x / kWave] = t; }
            __syncthreads();
            s = 0.0f; t = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) { s += sh.s[k]; t += sh.t[k]; }
        }
    }
    static QMM_DEV void run(uint32_t& m, Shared& sh)
    {
        m = over_lanes<IN_WAVE>(m, Most());
        if constexpr (LPR > kWave) {
            if ((threadIdx.x & (kWave - 1)) == 0) sh.s[threadIdx.x / kWave] = __uint_as_float(m);
            __syncthreads();
            m = 0u;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) m = max(m, __float_as_uint(sh.s[k]));
        }
    }
};
// The order of `units` of PER neighbouring rows that a launch's workgroups take.  Several rows a workgroup: runs of 32 rows to one XCD (workgroups go to the eight in turn), so that the
// step sizes of a block of columns, which lie row by row, are put together to lines in its L2 (16384 x 1024 in blocks of 128, rows in turn: 39 us instead of 33).  One row a workgroup: in
// turn, 1 to 2 % faster than that (16384 x 4096 without dropout 116 -> 114 us, 8192 x 4096 binary32 99 -> 97).
template <int PER> QMM_DEV int64_t unit_of(int64_t blk, int64_t units)
{
    constexpr int RUN = PER == 1 || PER >= 32 ? 1 : 32 / PER, PERIOD = 8 * RUN;
    if (RUN == 1 || blk / PERIOD >= units / PERIOD) return blk;
    const int r = (int)(blk % PERIOD);
    return blk - r + (r % 8) * RUN + r / 8;
}

// 1 / root as what multiplies the differences: of a row without a spread (variance 0 and eps 0, infinite) they count as zero in both passes, not as zero times infinity.
QMM_DEV float slope_of(float rstd) { return rstd == __uint_as_float(0x7F800000u) ? 0.0f : rstd; }
struct Stats { float mean, rest, rstd, factor; };
// From the sums of d and d^2.
QMM_DEV Stats stats_of(float mean, float sum_d, float sum_d2, int64_t cols, float eps)
{
    const float n = cols > 0 ? (float)cols : 1.0f, off = sum_d / n, var = fmaf(-off, off, sum_d2 / n);
    // What the differences to the mean still sum to is the mean's error only where it is more than their own roundings make, up to 2^-24 of each, and nearly the same in all
    // that have one exponent (16384 x 4096 bfloat16, taken out always: the mean off by 1.3e-6 in the 2-norm, now 4e-8).  Not a number stays one.
    const float rest = off * off <= 0x1p-46f * var ? 0.0f : off;
    Stats s;
    s.mean = mean + rest; s.rest = rest;
    s.rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);                  // (NaN stays)
    s.factor = slope_of(s.rstd);
    return s;
}

// x (dropped, if it is) plus the residual, in binary32, as a vector of the tensor's type.
template <typename T> QMM_DEV u32x4 stream_vector(const u32x4& x, const u32x4& r, const Drop& drop, uint64_t n)
{
    constexpr int V = Vec<T>::V;
    float v[V];
    if (drop.least) {
        const Kept keep = kept<V>(drop, n);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = fmaf(keep[e] ? Vec<T>::at(x, e) : 0.0f, drop.scale, Vec<T>::at(r, e));
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = Vec<T>::at(x, e) + Vec<T>::at(r, e);
    }
    return pack_row<T>(v);
}

// Rows of up to kRowElements: LPR lanes hold one, NV vectors a lane.  STREAM: x and r are read, h and y written past the caches (host).
// BLOCKS: a step size per 128 columns instead of one per row.
template <typename T, int MODE, int LPR, int NV, bool STREAM, bool BLOCKS> __global__ void __launch_bounds__(LPR > 256 ? LPR : 256)
layernorm_rows(LayerArgs a)
{
    constexpr int V = Vec<T>::V, THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
    __shared__ typename RowSums<LPR>::Shared sh_sum, sh_squares;
    __shared__ typename RowSums<LPR>::Shared sh_max;
    constexpr bool AHEAD = LPR < 1024;
    const int64_t total = a.batch * a.rows, units = (total + RPB - 1) / RPB;
    const int c0 = (int)(threadIdx.x % LPR) * V;
    Weights weight[NV], bias[NV];
    auto fetch_both = [&]() {
#pragma unroll
        for (int k = 0; k < NV; ++k) weight[k] = fetch_weights<V>(a.w, a.w_bf16, c0 + k * LPR * V, (int)a.cols);
#pragma unroll
        for (int k = 0; k < NV; ++k) bias[k] = fetch_weights<V>(a.bias, a.w_bf16, c0 + k * LPR * V, (int)a.cols);
    };
    if constexpr (AHEAD) fetch_both();
    struct Row { u32x4 x[NV], r[NV]; };
    auto row_id = [&](int64_t blk) { return (BLOCKS ? unit_of<RPB>(blk, units) : blk) * RPB + threadIdx.x / LPR; };
    auto fetch = [&](int64_t blk, Row& row) {
        const int64_t id = row_id(blk);
        const bool live = id < total;
        const int64_t b = live && a.batch > 1 ? id / a.rows : 0, i = live ? id - b * a.rows : 0;
        const int cols = live ? (int)a.cols : 0;
        const T* x = static_cast<const T*>(a.x) + b * a.x_batch + i * a.x_row;
#pragma unroll
        for (int k = 0; k < NV; ++k) row.x[k] = fetch_row<T, LPR == 8, STREAM>(x, c0 + k * LPR * V, cols);
        if (a.r) {
            const T* r = static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row;
#pragma unroll
            for (int k = 0; k < NV; ++k) row.r[k] = fetch_row<T, LPR == 8, STREAM>(r, c0 + k * LPR * V, cols);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) row.r[k] = u32x4{0u, 0u, 0u, 0u};
        }
    };
    Row row;
    if (AHEAD && blockIdx.x < units) fetch(blockIdx.x, row);
    for (int64_t blk = blockIdx.x; blk < units; blk += gridDim.x) {
        const int64_t id = row_id(blk);
        const bool live = id < total;
        const int64_t b = live && a.batch > 1 ? id / a.rows : 0, i = live ? id - b * a.rows : 0;
        const int cols = live ? (int)a.cols : 0;
        Row next;
        if constexpr (AHEAD) { if (blk + gridDim.x < units) fetch(blk + gridDim.x, next); }
        else { fetch(blk, row); fetch_both(); }
        u32x4 w[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            w[k] = settle_row<T, LPR == 8, STREAM>(row.x[k], c, cols);
            if (a.h) {
                const u32x4 q = settle_row<T, LPR == 8, STREAM>(row.r[k], c, cols);
                w[k] = stream_vector<T>(w[k], q, a.drop, (uint64_t)(id * a.cols + c) + a.drop.offset);
                put_row<T, STREAM>(static_cast<T*>(a.h) + id * a.cols + c, w[k], cols - c);
            }
        }
        if constexpr (AHEAD) row = next;
        float y[NV][V], sum = 0.0f, none = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[k][e] = Vec<T>::at(w[k], e);
                sum += y[k][e];                              // (zeros behind the row's end)
            }
        RowSums<LPR>::run(sum, none, sh_sum);
        const float mean = cols > 0 ? sum / (float)a.cols : 0.0f;
        float sum_d = 0.0f, sum_d2 = 0.0f;
        // (what lies behind the row's end stays zero: a select a vector, and one an element where a vector is cut)
        auto take_out = [&](int k, float value) {
            const int left = cols - c0 - k * LPR * V;
            const float whole = left >= V ? value : 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) y[k][e] -= whole;
            if (!STREAM && left > 0 && left < V) {
#pragma unroll
                for (int e = 0; e < V; ++e) y[k][e] -= e < left ? value : 0.0f;
            }
        };
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            take_out(k, mean);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sum_d += y[k][e];
                sum_d2 = fmaf(y[k][e], y[k][e], sum_d2);
            }
        }
        RowSums<LPR>::run(sum_d, sum_d2, sh_squares);
        const Stats st = stats_of(mean, sum_d, sum_d2, a.cols, a.eps);
        if (live && threadIdx.x % LPR == 0) {
            if (a.mean) a.mean[id] = st.mean;
            if (a.rstd) a.rstd[id] = st.rstd;
        }
        uint32_t m[NV], row_max = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float wv[V], bv[V];
            weight_values<V>(weight[k], a.w, a.w_bf16, c0 + k * LPR * V, (int)a.cols, wv);
            weight_values<V>(bias[k], a.bias, a.w_bf16, c0 + k * LPR * V, (int)a.cols, bv);
            m[k] = 0;
            take_out(k, st.rest);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[k][e] = fmaf(y[k][e] * st.factor, wv[e], a.bias ? bv[e] : 0.0f);
                m[k] = max(m[k], mag_bits(y[k][e]));           // (behind the row's end the weights are finite and the bias zero)
            }
            row_max = max(row_max, m[k]);
        }
        if (a.y) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = c0 + k * LPR * V;
                put_row<T, STREAM>(static_cast<T*>(a.y) + id * a.cols + c, pack_row<T>(y[k]), cols - c);
            }
        }
        if (!a.delta) continue;
        if constexpr (!BLOCKS) {
            RowSums<LPR>::run(row_max, sh_max);
            const float d = delta_from_absmax_bits(row_max, a.qmax);
            if (live && threadIdx.x % LPR == 0) a.delta[id] = d;
            const float rho = 1.0f / d;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = c0 + k * LPR * V, left = cols - c;
                if (left <= 0) continue;
                const int64_t p = id * a.cols + c;
                store_row_codes<T>(a.codes + p, encode_known<V, MODE>(y[k], row_max, rho, a.fmt, (uint64_t)p + a.offset, a.seed), left);
            }
        } else {
            constexpr int LB = LPR < kBlock / V ? LPR : kBlock / V;          // lanes of a block
            const int64_t blocks = (a.cols + kBlock - 1) / kBlock;
#pragma unroll
            for (int k = 0; k < NV; ++k) m[k] = over_lanes<LB>(m[k], Most());
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = c0 + k * LPR * V, left = cols - c;
                if (left <= 0) continue;
                const float d = delta_from_absmax_bits(m[k], a.qmax);
                if (threadIdx.x % LB == 0) a.delta[(b * blocks + c / kBlock) * a.rows + i] = d;
                const int64_t p = id * a.cols + c;
                store_row_codes<T>(a.codes + p, encode_known<V, MODE>(y[k], m[k], 1.0f / d, a.fmt, (uint64_t)p + a.offset, a.seed), left);
            }
        }
    }
}

// Longer rows: a workgroup goes over its row four times (three where no codes of a whole row are wanted), all but the first out of the L2.
template <typename T, int MODE, bool BLOCKS> __global__ void __launch_bounds__(kRowLanes)
layernorm_long(LayerArgs a)
{
    constexpr int V = Vec<T>::V, STEP = kRowLanes * V;
    __shared__ typename RowSums<kRowLanes>::Shared sh_sum, sh_squares;
    __shared__ typename RowSums<kRowLanes>::Shared sh_max;
    const int64_t total = a.batch * a.rows;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const int cols = (int)a.cols;
        const T* x = static_cast<const T*>(a.x) + b * a.x_batch + i * a.x_row;
        const T* r = a.r ? static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row : nullptr;
        T* h = a.h ? static_cast<T*>(a.h) + id * a.cols : nullptr;
        float sum = 0.0f, none = 0.0f;
        for (int c = (int)threadIdx.x * V; c < cols; c += STEP) {
            u32x4 w = load_row<T>(x, c, cols);
            if (h) {
                u32x4 q = {0u, 0u, 0u, 0u};
                if (r) q = load_row<T>(r, c, cols);
                w = stream_vector<T>(w, q, a.drop, (uint64_t)(id * a.cols + c) + a.drop.offset);
                store_row<T>(h + c, w, cols - c);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum += Vec<T>::at(w, e);
        }
        // what a thread reads below are its own elements and, in front of a row's end, some of another's that it shifts out
        __syncthreads();
        RowSums<kRowLanes>::run(sum, none, sh_sum);
        const T* src = h ? h : x;
        const float mean = sum / (float)a.cols;
        float sum_d = 0.0f, sum_d2 = 0.0f;
        for (int c = (int)threadIdx.x * V; c < cols; c += STEP) {
            const u32x4 w = load_row<T>(src, c, cols);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = c + e < cols ? Vec<T>::at(w, e) - mean : 0.0f;
                sum_d += d;
                sum_d2 = fmaf(d, d, sum_d2);
            }
        }
        RowSums<kRowLanes>::run(sum_d, sum_d2, sh_squares);
        const Stats st = stats_of(mean, sum_d, sum_d2, a.cols, a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[id] = st.mean;
            if (a.rstd) a.rstd[id] = st.rstd;
        }
        auto values = [&](int c, float (&y)[V]) -> uint32_t {
            const u32x4 w = load_row<T>(src, c, cols);
            float wv[V], bv[V];
            load_weight<V>(a.w, a.w_bf16, c, cols, wv);
            load_weight<V>(a.bias, a.w_bf16, c, cols, bv);
            uint32_t m = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[e] = fmaf(((Vec<T>::at(w, e) - mean) - st.rest) * st.factor, wv[e], a.bias ? bv[e] : 0.0f);
                if (c + e < cols) m = max(m, mag_bits(y[e]));
            }
            return m;
        };
        float rho = 0.0f;
        if (!BLOCKS && a.delta) {
            uint32_t m = 0;
            float y[V];
            for (int c = (int)threadIdx.x * V; c < cols; c += STEP) m = max(m, values(c, y));
            RowSums<kRowLanes>::run(m, sh_max);
            const float d = delta_from_absmax_bits(m, a.qmax);
            if (threadIdx.x == 0) a.delta[id] = d;
            rho = 1.0f / d;
        }
        const int64_t blocks = (a.cols + kBlock - 1) / kBlock;
        for (int base = 0; base < cols; base += STEP) {                      // (all lanes of a block go through the exchange)
            const int c = base + (int)threadIdx.x * V, left = min(V, cols - c);
            float y[V];
            uint32_t m = left > 0 ? values(c, y) : 0u;
            const int64_t p = id * a.cols + c;
            if (a.y && left > 0) store_row<T>(static_cast<T*>(a.y) + p, pack_row<T>(y), left);
            if (!a.delta) continue;
            if constexpr (BLOCKS) {
                m = over_lanes<kBlock / V>(m, Most());
                const float d = delta_from_absmax_bits(m, a.qmax);
                if (left > 0 && threadIdx.x % (kBlock / V) == 0) a.delta[(b * blocks + c / kBlock) * a.rows + i] = d;
                rho = 1.0f / d;
            }
            if (left > 0) store_row_codes<T>(a.codes + p, encode_values<V, MODE>(y, rho, a.fmt, (uint64_t)p + a.offset, a.seed), left);
        }
    }
}

struct LayerGradArgs {
    const void* dy; const void* h; const void* r;      // r: the gradient that reaches h past the norm, or null
    int64_t dy_batch, dy_row, h_batch, h_row, r_batch, r_row;
    const float* mean; const float* rstd;
    const void* w; int w_bf16;
    Drop drop;
    void* dh; void* dx;                                // dx: null where nothing was dropped
    float* partial;                                    // [2][shares][cols]: shares of dw, then of db; or null
    float* dw; float* db;
    int64_t batch, rows, cols, shares;
};

template <typename T> QMM_DEV void store_gradients(const LayerGradArgs& a, int64_t p, const float* v, int left)
{
    constexpr int V = Vec<T>::V;
    store_row<T>(static_cast<T*>(a.dh) + p, pack_row<T>(v), left);
    if (!a.dx) return;
    float u[V];
    drop_values<V>(a.drop, (uint64_t)p + a.drop.offset, v, u);
    store_row<T>(static_cast<T*>(a.dx) + p, pack_row<T>(u), left);
}

// A thread's next row is on its way while it works on the current one; workgroups of 1024 threads, whose threads have 128 registers, do without.
// STREAM: dy, h and r are read past the caches (host).
template <typename T, int LPR, int NV, bool STREAM> __global__ void __launch_bounds__(LPR > 256 ? LPR : 256)
layernorm_grad_rows(LayerGradArgs a)
{
    constexpr int V = Vec<T>::V, THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
    constexpr bool AHEAD = LPR < 1024;
    __shared__ typename RowSums<LPR>::Shared sh[2];
    __shared__ float s_share[2][RPB > 1 ? RPB : 1][RPB > 1 ? LPR * NV * V : 1];
    const int64_t total = a.batch * a.rows;
    const int c0 = (int)(threadIdx.x % LPR) * V;
    float weight[NV][V], dw[NV][V], db[NV][V];
    auto load_weights = [&]() {
#pragma unroll
        for (int k = 0; k < NV; ++k) load_weight<V>(a.w, a.w_bf16, c0 + k * LPR * V, (int)a.cols, weight[k]);
    };
    if constexpr (AHEAD) load_weights();
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[k][e] = db[k][e] = 0.0f;
    struct Row { u32x4 g[NV], w[NV], q[NV]; float mean, rstd; };      // dy, h, dresidual
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
        r.mean = live ? a.mean[id] : 0.0f;
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
        const float rstd = slope_of(row.rstd);
        float sum_a = 0.0f, sum_an = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            row.g[k] = settle_row<T, LPR == 8, STREAM>(row.g[k], c, cols);
            row.w[k] = settle_row<T, LPR == 8, STREAM>(row.w[k], c, cols);
            row.q[k] = settle_row<T, LPR == 8, STREAM>(row.q[k], c, cols);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                // (behind the row's end dy is zero; n may be anything finite or not, so it is left out there)
                const float d = Vec<T>::at(row.g[k], e), n = c + e < cols ? (Vec<T>::at(row.w[k], e) - row.mean) * rstd : 0.0f, g = d * weight[k][e];
                sum_a += g;
                sum_an = fmaf(g, n, sum_an);
                dw[k][e] = fmaf(d, n, dw[k][e]);
                db[k][e] += d;
            }
        }
        RowSums<LPR>::run(sum_a, sum_an, sh[turn]);
        const float mean_a = sum_a / (float)a.cols, mean_an = sum_an / (float)a.cols;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V, left = cols - c;
            if (left <= 0) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float n = (Vec<T>::at(row.w[k], e) - row.mean) * rstd;
                v[e] = fmaf(rstd, fmaf(-n, mean_an, Vec<T>::at(row.g[k], e) * weight[k][e] - mean_a), Vec<T>::at(row.q[k], e));
            }
            store_gradients<T>(a, id * a.cols + c, v, left);
        }
        if constexpr (AHEAD) row = next;
    }
    if (!a.partial) return;
    if constexpr (RPB > 1) {
        // the workgroup's rows side by side: added in order
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s_share[0][threadIdx.x / LPR][c0 + k * LPR * V + e] = dw[k][e];
                s_share[1][threadIdx.x / LPR][c0 + k * LPR * V + e] = db[k][e];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += THREADS)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < RPB; ++q) s += s_share[t][q][c];
                a.partial[(t * a.shares + blockIdx.x) * a.cols + c] = s;
            }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                store_row<float>(a.partial + (int64_t)blockIdx.x * a.cols + c + 4 * q, pack_row<float>(dw[k] + 4 * q), (int)a.cols - c - 4 * q);
                store_row<float>(a.partial + (a.shares + blockIdx.x) * a.cols + c + 4 * q, pack_row<float>(db[k] + 4 * q), (int)a.cols - c - 4 * q);
            }
        }
    }
}

// Longer rows: dh by workgroups that go over their row twice, the shares of dw and db by another pass down the columns.
template <typename T> __global__ void __launch_bounds__(kRowLanes)
layernorm_grad_long(LayerGradArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ typename RowSums<kRowLanes>::Shared sh[2];
    const int64_t total = a.batch * a.rows;
    int turn = 0;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x, turn ^= 1) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const int cols = (int)a.cols;
        const T* dy = static_cast<const T*>(a.dy) + b * a.dy_batch + i * a.dy_row;
        const T* h = static_cast<const T*>(a.h) + b * a.h_batch + i * a.h_row;
        const T* r = a.r ? static_cast<const T*>(a.r) + b * a.r_batch + i * a.r_row : nullptr;
        const float mean = a.mean[id], rstd = slope_of(a.rstd[id]);
        float sum_a = 0.0f, sum_an = 0.0f;
        for (int c = (int)threadIdx.x * V; c < cols; c += kRowLanes * V) {
            const u32x4 g = load_row<T>(dy, c, cols), w = load_row<T>(h, c, cols);
            float weight[V];
            load_weight<V>(a.w, a.w_bf16, c, cols, weight);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = Vec<T>::at(g, e) * weight[e], n = c + e < cols ? (Vec<T>::at(w, e) - mean) * rstd : 0.0f;
                sum_a += d;
                sum_an = fmaf(d, n, sum_an);
            }
        }
        RowSums<kRowLanes>::run(sum_a, sum_an, sh[turn]);
        const float mean_a = sum_a / (float)a.cols, mean_an = sum_an / (float)a.cols;
        for (int c = (int)threadIdx.x * V; c < cols; c += kRowLanes * V) {
            const u32x4 g = load_row<T>(dy, c, cols), w = load_row<T>(h, c, cols);
            const u32x4 q = r ? load_row<T>(r, c, cols) : u32x4{0u, 0u, 0u, 0u};
            float weight[V], v[V];
            load_weight<V>(a.w, a.w_bf16, c, cols, weight);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float n = (Vec<T>::at(w, e) - mean) * rstd;
                v[e] = fmaf(rstd, fmaf(-n, mean_an, Vec<T>::at(g, e) * weight[e] - mean_a), Vec<T>::at(q, e));
            }
            store_gradients<T>(a, id * a.cols + c, v, cols - c);
        }
    }
}
template <typename T> __global__ void __launch_bounds__(kThreads)
layernorm_grad_columns(LayerGradArgs a)                // grid (columns, shares): every share-th row
{
    constexpr int V = Vec<T>::V;
    const int64_t total = a.batch * a.rows;
    const int64_t c = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * V;
    if (c >= a.cols) return;
    const int left = (int)min((int64_t)V, a.cols - c);
    float dw[V] = {}, db[V] = {};
    for (int64_t id = blockIdx.y; id < total; id += gridDim.y) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const u32x4 g = load_row<T>(static_cast<const T*>(a.dy) + b * a.dy_batch + i * a.dy_row, (int)c, (int)a.cols);
        const u32x4 w = load_row<T>(static_cast<const T*>(a.h) + b * a.h_batch + i * a.h_row, (int)c, (int)a.cols);
        const float mean = a.mean[id], rstd = slope_of(a.rstd[id]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float d = Vec<T>::at(g, e);
            dw[e] = fmaf(d, (Vec<T>::at(w, e) - mean) * rstd, dw[e]);
            db[e] += d;
        }
    }
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
        store_row<float>(a.partial + (int64_t)blockIdx.y * a.cols + c + 4 * q, pack_row<float>(dw + 4 * q), left - 4 * q);
        store_row<float>(a.partial + (a.shares + blockIdx.y) * a.cols + c + 4 * q, pack_row<float>(db + 4 * q), left - 4 * q);
    }
}

// dw and db = the sums of the shares, in an order fixed by their number: a workgroup takes 16 columns of one, sixty-four lanes a column.
__global__ void __launch_bounds__(1024)
layernorm_grad_fold(LayerGradArgs a)
{
    constexpr int C = 16, L = 1024 / C;
    __shared__ float part[L][C + 1];
    const float* partial = a.partial + (int64_t)blockIdx.y * a.shares * a.cols;
    float* out = blockIdx.y ? a.db : a.dw;
    const int c_in = threadIdx.x % C, l = threadIdx.x / C;
    const int64_t c = (int64_t)blockIdx.x * C + c_in;
    float s = 0.0f;
    if (c < a.cols) {
#pragma unroll 8
        for (int64_t p = l; p < a.shares; p += L) s += partial[p * a.cols + c];
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
        if (threadIdx.x < C && f < a.cols) out[f] = s;
    }
}

// Shares of dw and db: workgroups that go over rows, as for the root-mean-square norm's backward pass.
int64_t shares_of(const qmm_tensor* t)
{
    const int64_t total = t->batch * t->rows;
    if (t->cols > kRowElements) return std::min<int64_t>(total, 64);
    int64_t blocks = 0, most = 512;
    auto count = [&](auto lpr, auto) {
        constexpr int rpb = lpr.value < 256 ? 256 / lpr.value : 1;
        blocks = (total + rpb - 1) / rpb;
        if (lpr.value == 1024) most = 256;
    };
    if (t->dtype == QMM_DT_BF16) for_row_size<uint16_t>(t->cols, count); else for_row_size<float>(t->cols, count);
    const int64_t turns = (blocks + most - 1) / most;        // the fewest that take no more turns
    return (blocks + turns - 1) / turns;
}

unsigned norm_blocks(int64_t total, int per, int lpr) { return (unsigned)std::min<int64_t>((total + per - 1) / per, lpr >= 1024 ? 1 << 21 : lpr == 512 ? 512 : 1024); }
template <typename T, int MODE, bool BLOCKS> qmm_status launch_layer(const LayerArgs& a, bool stream, hipStream_t s)
{
    const int64_t total = a.batch * a.rows;
    if (a.cols > kRowElements) layernorm_long<T, MODE, BLOCKS><<<row_blocks(total, 1), kRowLanes, 0, s>>>(a);
    else for_row_size<T>(a.cols, [&](auto lpr, auto nv) {
        constexpr int threads = lpr.value > 256 ? lpr.value : 256;
        if constexpr (lpr.value >= kWave) {
            if (stream) { layernorm_rows<T, MODE, lpr.value, nv.value, true, BLOCKS><<<norm_blocks(total, threads / lpr.value, lpr.value), threads, 0, s>>>(a); return; }
        }
        layernorm_rows<T, MODE, lpr.value, nv.value, false, BLOCKS><<<norm_blocks(total, threads / lpr.value, lpr.value), threads, 0, s>>>(a);
    });
    return launch_status();
}
template <typename T> qmm_status launch_layer_form(const LayerArgs& a, bool blocks, qmm_round mode, bool stream, hipStream_t s)
{
    if (mode == QMM_ROUND_RTNE) return blocks ? launch_layer<T, QMM_ROUND_RTNE, true>(a, stream, s) : launch_layer<T, QMM_ROUND_RTNE, false>(a, stream, s);
    return blocks ? launch_layer<T, QMM_ROUND_STOCHASTIC, true>(a, stream, s) : launch_layer<T, QMM_ROUND_STOCHASTIC, false>(a, stream, s);
}
template <typename T> qmm_status launch_layer_grad(LayerGradArgs& a, bool stream, hipStream_t s)
{
    const int64_t total = a.batch * a.rows;
    if (a.cols > kRowElements) {
        // (down the columns first: dh may be written over dy)
        if (a.partial) {
            const unsigned strips = (unsigned)((a.cols + kThreads * Vec<T>::V - 1) / (kThreads * Vec<T>::V));
            layernorm_grad_columns<T><<<dim3(strips, (unsigned)a.shares), kThreads, 0, s>>>(a);
            if (hipGetLastError() != hipSuccess) return QMM_ERR_LAUNCH;
        }
        layernorm_grad_long<T><<<row_blocks(total, 1), kRowLanes, 0, s>>>(a);
    } else {
        for_row_size<T>(a.cols, [&](auto lpr, auto nv) {
            constexpr int threads = lpr.value > 256 ? lpr.value : 256;
            if constexpr (lpr.value >= kWave) {
                if (stream) { layernorm_grad_rows<T, lpr.value, nv.value, true><<<(unsigned)a.shares, threads, 0, s>>>(a); return; }
            }
            layernorm_grad_rows<T, lpr.value, nv.value, false><<<(unsigned)a.shares, threads, 0, s>>>(a);
        });
    }
    if (a.partial) {
        if (hipGetLastError() != hipSuccess) return QMM_ERR_LAUNCH;
        layernorm_grad_fold<<<dim3((unsigned)((a.cols + 15) / 16), 2), 1024, 0, s>>>(a);
    }
    return launch_status();
}

}  // namespace
}  // namespace qmm

using namespace qmm;

extern "C" qmm_status qmm_layernorm_quantize(const qmm_tensor* x, const qmm_tensor* residual, const void* weight, const void* bias, qmm_dtype weight_dtype,
                                             float eps, float dropout, uint64_t dropout_seed, uint64_t dropout_offset, qmm_format fmt, int32_t block,
                                             qmm_round mode, uint64_t seed, uint64_t offset, void* h_out, void* y_out, float* mean_out, float* rstd_out,
                                             float* delta_out, uint8_t* codes_out, void* stream)
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
    const bool codes = codes_out || delta_out;
    if (codes) {
        if (fmt != QMM_FMT_INT8 && fmt != QMM_FMT_E4M3 && fmt != QMM_FMT_E5M2) return QMM_ERR_ENUM;
        if (mode != QMM_ROUND_RTNE && mode != QMM_ROUND_STOCHASTIC) return QMM_ERR_ENUM;
        if (block != 0 && block != kBlock) return QMM_ERR_ENUM;
    }
    LayerArgs a{};
    if (!(eps >= 0.0f && eps <= 3.402823466e38f) || !drop_of(dropout, dropout_seed, dropout_offset, &a.drop)) return QMM_ERR_SHAPE;
    const bool new_h = residual || dropout > 0.0f;
    if (x->batch * x->rows == 0) return QMM_OK;
    if (!codes && !y_out && !mean_out && !rstd_out && !(new_h && h_out)) return QMM_ERR_NULL;
    if (x->cols > 0 && (!x->data || (residual && !residual->data) || (new_h && !h_out) || (codes && (!codes_out || !delta_out)))) return QMM_ERR_NULL;
    if (codes && block == 0 && !delta_out) return QMM_ERR_NULL;
    if (!element_aligned(x->data, x->dtype) || (residual && !element_aligned(residual->data, x->dtype)) || !element_aligned(h_out, x->dtype) ||
        !element_aligned(y_out, x->dtype) || !element_aligned(weight, weight_dtype) || !element_aligned(bias, weight_dtype) ||
        !element_aligned(delta_out, QMM_DT_F32) || !element_aligned(mean_out, QMM_DT_F32) || !element_aligned(rstd_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    for (const void* out : {static_cast<const void*>(new_h ? h_out : nullptr), static_cast<const void*>(y_out)})      // over an input: element by element only
        if (out && ((out == x->data && !dense(x)) || (residual && out == residual->data && !dense(residual)))) return QMM_ERR_SHAPE;
    if (new_h && h_out == y_out && x->cols > 0) return QMM_ERR_SHAPE;

    a.x = x->data; a.x_batch = x->batch_stride; a.x_row = x->row_stride;
    if (residual) { a.r = residual->data; a.r_batch = residual->batch_stride; a.r_row = residual->row_stride; }
    if (new_h) a.h = h_out;
    a.w = weight; a.bias = bias; a.w_bf16 = weight_dtype == QMM_DT_BF16; a.eps = eps;
    a.y = y_out; a.mean = mean_out; a.rstd = rstd_out; a.delta = delta_out; a.codes = codes_out;
    a.batch = x->batch; a.rows = x->rows; a.cols = x->cols;
    a.seed = seed; a.offset = offset;
    if (codes) { a.qmax = host_qmax(fmt); a.fmt = fmt; }
    // As in qmm_rmsnorm_quantize, where a residual is read beside x.  Without one the rule is ordinary loads, though streaming is mostly faster there too (16384 x 4096
    // bfloat16, dropout and all outputs, 104 us by ordinary loads, 95 by streaming; without dropout 84 / 80; 65536 x 1024, codes alone, 65 / 68).
    const bool streaming = residual && streams(x) && streams(residual) && aligned16(h_out) && aligned16(y_out);
    hipStream_t s = as_stream(stream);
    return x->dtype == QMM_DT_BF16 ? launch_layer_form<uint16_t>(a, block == kBlock, mode, streaming, s) : launch_layer_form<float>(a, block == kBlock, mode, streaming, s);
}

extern "C" size_t qmm_layernorm_backward_workspace_size(const qmm_tensor* dy)
{
    if (!dy || check_rows(dy) != QMM_OK || dy->batch * dy->rows * dy->cols == 0) return 0;
    return 2u * (size_t)shares_of(dy) * (size_t)dy->cols * sizeof(float);
}

extern "C" qmm_status qmm_layernorm_backward(const qmm_tensor* dy, const qmm_tensor* h, const float* mean, const float* rstd, const void* weight,
                                             qmm_dtype weight_dtype, const qmm_tensor* dresidual, float dropout, uint64_t dropout_seed,
                                             uint64_t dropout_offset, void* dh_out, void* dx_out, float* dw_out, float* db_out, void* workspace,
                                             size_t workspace_bytes, void* stream)
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
    LayerGradArgs a{};
    if (!drop_of(dropout, dropout_seed, dropout_offset, &a.drop)) return QMM_ERR_SHAPE;
    if (!dw_out != !db_out) return QMM_ERR_NULL;
    if (dy->cols == 0) return QMM_OK;
    a.batch = dy->batch; a.rows = dy->rows; a.cols = dy->cols;
    const bool empty = dy->batch * dy->rows == 0;
    if (!empty && (!dy->data || !h->data || !mean || !rstd || !dh_out || (dropout > 0.0f && !dx_out) || (dresidual && !dresidual->data))) return QMM_ERR_NULL;
    if (dropout > 0.0f) a.dx = dx_out;
    for (const qmm_tensor* t : {dy, h, dresidual}) {
        if (!t) continue;
        if (!element_aligned(t->data, t->dtype)) return QMM_ERR_ALIGN;
        if ((dh_out && dh_out == t->data && !dense(t)) || (a.dx && a.dx == t->data && !dense(t))) return QMM_ERR_SHAPE;
    }
    if (!empty && a.dx && a.dx == dh_out) return QMM_ERR_SHAPE;
    if (!element_aligned(dh_out, dy->dtype) || !element_aligned(a.dx, dy->dtype) || !element_aligned(weight, weight_dtype) || !element_aligned(mean, QMM_DT_F32) ||
        !element_aligned(rstd, QMM_DT_F32) || !element_aligned(dw_out, QMM_DT_F32) || !element_aligned(db_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    a.dw = dw_out; a.db = db_out;
    hipStream_t s = as_stream(stream);
    if (empty) {                                             // no rows: sums of none
        if (dw_out) layernorm_grad_fold<<<dim3((unsigned)((a.cols + 15) / 16), 2), 1024, 0, s>>>(a);
        return launch_status();
    }
    if (dw_out) {
        const size_t need = qmm_layernorm_backward_workspace_size(dy);
        if (!workspace || workspace_bytes < need) return QMM_ERR_WORKSPACE;
        if (!aligned16(workspace)) return QMM_ERR_ALIGN;
        a.partial = static_cast<float*>(workspace);
    }
    a.shares = shares_of(dy);
    a.dy = dy->data; a.dy_batch = dy->batch_stride; a.dy_row = dy->row_stride;
    a.h = h->data; a.h_batch = h->batch_stride; a.h_row = h->row_stride;
    if (dresidual) { a.r = dresidual->data; a.r_batch = dresidual->batch_stride; a.r_row = dresidual->row_stride; }
    a.mean = mean; a.rstd = rstd; a.w = weight; a.w_bf16 = weight_dtype == QMM_DT_BF16; a.dh = dh_out;
    const bool streaming = streams(dy) && streams(h) && (!dresidual || streams(dresidual));
    return dy->dtype == QMM_DT_BF16 ? launch_layer_grad<uint16_t>(a, streaming, s) : launch_layer_grad<float>(a, streaming, s);
}
