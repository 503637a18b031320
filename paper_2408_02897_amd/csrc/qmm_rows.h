// Device code shared by the operators that keep a token's row in registers between a reduction over it and its output
// (qmm_rmsnorm.hip, qmm_gated.hip): vectors of a row, reductions over the lanes that hold one, codes of computed values.
#pragma once
#include <algorithm>
#include <type_traits>
#include "qmm_encode.h"

namespace qmm {
namespace {

// The vector of elements c .. c + V - 1 of a row of `cols`, zeros from there on; c a multiple of V.  In two steps, so that all of a row's loads are on their
// way before the first is waited for: fetch_row takes a row's last elements with the vector that ends there, settle_row shifts that one.  (One by one, each
// behind a branch and a wait, they were what a row of odd length took: bfloat16 8969 x 1491, the norm's backward pass 70 us against 28 of 1488 columns;
// shifted where they were loaded 50, now 30 and 26.)  SHORT: rows of less than a vector are possible.  STREAM: a large tensor of whole lines that is not read again; its
// lines are the first to leave the caches, else they take the place of what is still wanted.  (A constant of the kernel: chosen by a branch, the two loads
// were made one ordinary one, or with what kept them apart 133 us where the gated gradients of 16384 x 4096 take 119.)
template <typename T, bool SHORT = true, bool STREAM = false> QMM_DEV u32x4 fetch_row(const T* row, int c, int cols)
{
    constexpr int V = Vec<T>::V;
    if (c >= cols) return u32x4{0u, 0u, 0u, 0u};
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + c));
    if (SHORT && cols < V) return Vec<T>::partial_load(row, cols);
    return *reinterpret_cast<const u32x4_any*>(row + min(c, cols - V));
}
template <typename T, bool SHORT = true, bool STREAM = false> QMM_DEV u32x4 settle_row(u32x4 w, int c, int cols)
{
    constexpr int V = Vec<T>::V;
    if (!STREAM && c + V > cols && c < cols && (!SHORT || cols >= V)) {
        const uint32_t away = (uint32_t)(c + V - cols) * sizeof(T);      // bytes of the elements before c
        if (away & 8u) w = u32x4{w[2], w[3], 0u, 0u};
        if (away & 4u) w = u32x4{w[1], w[2], w[3], 0u};
        if constexpr (sizeof(T) == 2) { if (away & 2u) w = u32x4{(w[0] >> 16) | (w[1] << 16), (w[1] >> 16) | (w[2] << 16), (w[2] >> 16) | (w[3] << 16), w[3] >> 16}; }
    }
    return w;
}
template <typename T> QMM_DEV u32x4 load_row(const T* row, int c, int cols) { return settle_row<T>(fetch_row<T>(row, c, cols), c, cols); }
// binary32 values -> a vector of the tensor's type, rounded to nearest even
template <typename T> QMM_DEV u32x4 pack_row(const float* v)
{
    u32x4 w;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(v[e]);
    } else {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[2 * e], v[2 * e + 1]}, bf2));
    }
    return w;
}
template <typename T> QMM_DEV void store_row(T* p, const u32x4& w, int left)
{
    if (left >= Vec<T>::V) { *reinterpret_cast<u32x4_any*>(p) = w; return; }
    if (left > 0) store_bytes<16>(reinterpret_cast<uint8_t*>(p), w, left * (int)sizeof(T));
}
// The same of a vector's codes.
template <typename T> QMM_DEV void store_row_codes(uint8_t* p, u32x2 c, int left)
{
    if (left >= Vec<T>::V) store_codes<T>(p, c, left);
    else if (left > 0) store_bytes<8>(p, u32x4{c[0], c[1], 0u, 0u}, left);
}
// A vector's store, past the caches (STREAM; 16-byte boundaries) for outputs that are wanted again much later or do not fit them.
template <typename T, bool STREAM> QMM_DEV void put_row(T* p, const u32x4& w, int left)
{
    if constexpr (STREAM) { if (left > 0) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p)); }
    else store_row<T>(p, w, left);
}
// V of the norm's weights, of either type, ones where there is none: as they come from memory (so that they are requested in front of what is waited for
// first: the norm of bfloat16 16384 x 4096 112 -> 107 us), and as values.
struct Weights { u32x4 w[2]; };
template <int V> QMM_DEV Weights fetch_weights(const void* w, int bf16, int c, int cols)
{
    Weights r{};
    if (!w || c >= cols) return r;
    if (!bf16) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) r.w[q] = fetch_row<float>(static_cast<const float*>(w), c + 4 * q, cols);
    } else if constexpr (V == 8) r.w[0] = fetch_row<uint16_t>(static_cast<const uint16_t*>(w), c, cols);
    else {
        typedef unsigned int u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
        const uint16_t* p = static_cast<const uint16_t*>(w);
        if (cols >= V) {
            const u32x2_any q = *reinterpret_cast<const u32x2_any*>(p + min(c, cols - V));
            r.w[0][0] = q[0]; r.w[0][1] = q[1];
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) if (e < cols) r.w[0][e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        }
    }
    return r;
}
template <int V> QMM_DEV void weight_values(const Weights& r, const void* w, int bf16, int c, int cols, float (&out)[V])
{
    if (!w) {
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = 1.0f;
    } else if (!bf16) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const u32x4 v = settle_row<float>(r.w[q], c + 4 * q, cols);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[4 * q + e] = __uint_as_float(v[e]);
        }
    } else if constexpr (V == 8) {
        const u32x4 v = settle_row<uint16_t>(r.w[0], c, cols);
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = Vec<uint16_t>::at(v, e);
    } else {
        uint64_t q = r.w[0][0] | (uint64_t)r.w[0][1] << 32;
        if (c + V > cols && c < cols && cols >= V) q >>= 16 * (c + V - cols);
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = bf16_bits_to_f32((uint32_t)(q >> (16 * e)) & 0xFFFFu);
    }
}
template <int V> QMM_DEV void load_weight(const void* w, int bf16, int c, int cols, float (&out)[V])
{
    weight_values<V>(fetch_weights<V>(w, bf16, c, cols), w, bf16, c, cols, out);
}

// Sums and maxima over the LPR lanes that hold a row: within a wavefront by a butterfly, above 64 lanes over the workgroup (then
// all of it) through LDS.  The order of additions is fixed.  `turn` alternates between a workgroup's rows: with two
// sets of words one barrier a row is enough.
template <int LPR> struct RowReduce {
    static constexpr int WAVES = LPR > kWave ? LPR / kWave : 1;
    struct Shared { float sum[2][WAVES]; uint32_t max[2][WAVES]; };
    static QMM_DEV void lanes(float& s, uint32_t& m)
    {
#pragma unroll
        for (int off = (LPR < kWave ? LPR : kWave) / 2; off > 0; off >>= 1) {
            s += __shfl_xor(s, off, kWave);
            m = max(m, (uint32_t)__shfl_xor((int)m, off, kWave));
        }
    }
    static QMM_DEV void run(float& s, uint32_t& m, Shared& sh, int turn)
    {
        lanes(s, m);
        if constexpr (LPR > kWave) {
            if ((threadIdx.x & (kWave - 1)) == 0) { sh.sum[turn][threadIdx.x / kWave] = s; sh.max[turn][threadIdx.x / kWave] = m; }
            __syncthreads();
            s = 0.0f; m = 0u;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) { s += sh.sum[turn][k]; m = max(m, sh.max[turn][k]); }
        }
    }
};

// Codes of V = 4 or 8 computed values (times rho), the first of them element number g of the random stream.
template <int V, int MODE> QMM_DEV u32x2 encode_values(const float* y, float rho, int fmt, uint64_t g, uint64_t seed)
{
    constexpr int Q = V / 4;
    float t[V];
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = y[e] * rho;
    uint32_t c[Q];
    const bool whole = MODE == QMM_ROUND_STOCHASTIC && !__any((g & 3u) != 0u);
    if (fmt == QMM_FMT_INT8) encode_quads<QMM_FMT_INT8, MODE, Q>(t, g, seed, whole, c);
    else if (fmt == QMM_FMT_E4M3) encode_quads<QMM_FMT_E4M3, MODE, Q>(t, g, seed, whole, c);
    else encode_quads<QMM_FMT_E5M2, MODE, Q>(t, g, seed, whole, c);
    return u32x2{c[0], c[Q - 1]};
}

// Lanes and vectors of a row: the smallest that hold it.  f(lanes, vectors).
constexpr int kRowLanes = 1024, kRowElements = 16384;         // the longest row held in registers
template <typename T, typename F> void for_row_size(int64_t cols, F f)
{
    constexpr int V = Vec<T>::V;
    const int64_t nvec = (cols + V - 1) / V;
    auto run = [&](auto lpr, auto nv) { f(lpr, nv); };
#define QMM_ROW(L, N) run(std::integral_constant<int, L>{}, std::integral_constant<int, N>{})
    if (nvec <= 8) QMM_ROW(8, 1);
    else if (nvec <= 16) QMM_ROW(16, 1);
    else if (nvec <= 32) QMM_ROW(32, 1);
    else if (nvec <= 64) QMM_ROW(64, 1);
    else if (nvec <= 128) QMM_ROW(64, 2);
    else if (nvec <= 256) QMM_ROW(256, 1);
    else if (nvec <= 512) QMM_ROW(256, 2);
    else if (nvec <= 1024) QMM_ROW(512, 2);
    else if (nvec <= 2048) QMM_ROW(1024, 2);
    else if constexpr (V == 4) QMM_ROW(1024, 4);
#undef QMM_ROW
}

// ---- arguments (host)
constexpr int64_t kMaxColumns = int64_t(1) << 22;             // as a product's K
inline qmm_status check_rows(const qmm_tensor* t)
{
    if (t->dtype != QMM_DT_BF16 && t->dtype != QMM_DT_F32) return QMM_ERR_ENUM;
    if (t->contract_axis != 1) return t->contract_axis == 0 ? QMM_ERR_UNSUPPORTED : QMM_ERR_ENUM;
    if (t->batch < 0 || t->rows < 0 || t->cols < 0 || t->row_stride < t->cols) return QMM_ERR_SHAPE;
    if (t->batch > 1 && t->rows > 0 && t->batch_stride < (t->rows - 1) * t->row_stride + t->cols) return QMM_ERR_SHAPE;
    if (t->batch > 65535 || t->cols > kMaxColumns) return QMM_ERR_UNSUPPORTED;
    return QMM_OK;
}
inline bool element_aligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == QMM_DT_BF16 ? 1u : 3u)) == 0; }
inline bool same_extent(const qmm_tensor* a, const qmm_tensor* b) { return a->batch == b->batch && a->rows == b->rows && a->cols == b->cols; }
inline bool dense(const qmm_tensor* t)
{
    return (t->rows <= 1 || t->row_stride == t->cols) && (t->batch <= 1 || t->batch_stride == t->rows * t->cols);
}
// Whether a tensor is to be read by streaming loads: from 64 MB on, rows of whole lines (a line that two rows share would be fetched twice: binary32
// 16384 x 1000, the norm's backward pass 51.7 by ordinary loads, 54.9 by streaming ones).
inline bool streams(const qmm_tensor* t)
{
    const int64_t e = t->dtype == QMM_DT_BF16 ? 2 : 4;
    return t->batch * t->rows * t->cols * e >= (int64_t)64 << 20 && in_lines(t->data, (t->cols | t->row_stride | (t->batch > 1 ? t->batch_stride : 0)) * e);
}
// workgroups for `total` rows, `per` each (they go round where the grid would pass what a launch takes, 2^32 threads)
inline unsigned row_blocks(int64_t total, int per) { return (unsigned)std::min<int64_t>((total + per - 1) / per, 1 << 21); }

}  // namespace
}  // namespace qmm
