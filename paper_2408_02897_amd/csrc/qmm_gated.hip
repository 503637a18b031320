// qmm_gated_backward: the backward pass of h = act(g) u, up to the operand of the products behind it.
//   dg = dh u act'(g),  du = dh act(g)
// for a token's whole row (g | u), as values for the weight gradient and, quantized with one step size per token (Eq. 1), as the
// codes of the data gradient's operand.  A row is read once, its 2 F results stay in registers until their largest magnitude is known:
// the codes are of the binary32 results, not of their bfloat16 roundings.
// Bound by memory traffic: bfloat16 reads 6 bytes and writes 4 + 2 a pair; 16384 x 4096 (805 MB) 120 us, 6.7 TB/s; GELU's, with more
// vector work, 122 to 127.
#include "qmm_activation.h"
#include "qmm_rows.h"

namespace qmm {
namespace {

struct GatedGradArgs {
    const void* dh; const void* gu;
    int64_t dh_batch, dh_row, gu_batch, gu_row;
    void* dgu;                                 // dense, or null
    float* delta; uint8_t* codes;              // or null, both
    int64_t batch, rows, F;
    uint64_t seed, offset;
    float qmax; int fmt;
};

// V pairs of results
template <typename T, int ACT> QMM_DEV void gated_grad(const u32x4& dh, const u32x4& g, const u32x4& u, float* dg, float* du)
{
#pragma unroll
    for (int e = 0; e < Vec<T>::V; ++e) {
        const float d = Vec<T>::at(dh, e);
        float value, slope;
        activate_slope<ACT, sizeof(T) == 2>(Vec<T>::at(g, e), value, slope);
        dg[e] = (d * Vec<T>::at(u, e)) * slope;
        du[e] = d * value;
    }
}
template <typename T, int MODE, bool STREAM> QMM_DEV void gated_grad_out(const GatedGradArgs& a, int64_t p, const float* v, int left, float rho)
{
    if (a.dgu) put_row<T, STREAM>(static_cast<T*>(a.dgu) + p, pack_row<T>(v), left);
    if (a.codes) store_row_codes<T>(a.codes + p, encode_values<Vec<T>::V, MODE>(v, rho, a.fmt, (uint64_t)p + a.offset, a.seed), left);
}

// STREAM: dh and gu are read, dgu is written past the caches (host).
template <typename T, int MODE, int ACT, int LPR, int NV, bool STREAM> __global__ void __launch_bounds__(LPR > 256 ? LPR : 256)
gated_grad_rows(GatedGradArgs a)
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
        const int F = live ? (int)a.F : 0;
        const T* dh = static_cast<const T*>(a.dh) + b * a.dh_batch + i * a.dh_row;
        const T* g = static_cast<const T*>(a.gu) + b * a.gu_batch + i * a.gu_row;
        u32x4 wd[NV], wg[NV], wu[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            wd[k] = fetch_row<T, LPR == 8, STREAM>(dh, c, F);
            wg[k] = fetch_row<T, LPR == 8, STREAM>(g, c, F);
            wu[k] = fetch_row<T, LPR == 8, STREAM>(g + a.F, c, F);
        }
        float dg[NV][V], du[NV][V], none = 0.0f;
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V;
            gated_grad<T, ACT>(settle_row<T, LPR == 8, STREAM>(wd[k], c, F), settle_row<T, LPR == 8, STREAM>(wg[k], c, F), settle_row<T, LPR == 8, STREAM>(wu[k], c, F), dg[k], du[k]);
#pragma unroll
            for (int e = 0; e < V; ++e) m = max(m, max(mag_bits(dg[k][e]), mag_bits(du[k][e])));
        }
        RowReduce<LPR>::run(none, m, sh, turn);
        if (!live) continue;
        const float d = delta_from_absmax_bits(m, a.qmax), rho = 1.0f / d;
        if (a.delta && threadIdx.x % LPR == 0) a.delta[id] = d;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = c0 + k * LPR * V, left = F - c;
            if (left <= 0) continue;
            const int64_t p = id * 2 * a.F + c;
            gated_grad_out<T, MODE, STREAM>(a, p, dg[k], left, rho);
            gated_grad_out<T, MODE, STREAM>(a, p + a.F, du[k], left, rho);
        }
    }
}

// Longer rows: a workgroup goes over its row twice, the second time out of the L2.
template <typename T, int MODE, int ACT> __global__ void __launch_bounds__(kRowLanes)
gated_grad_long(GatedGradArgs a)
{
    constexpr int V = Vec<T>::V;
    __shared__ typename RowReduce<kRowLanes>::Shared sh;
    const int64_t total = a.batch * a.rows;
    int turn = 0;
    for (int64_t id = blockIdx.x; id < total; id += gridDim.x, turn ^= 1) {
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const T* dh = static_cast<const T*>(a.dh) + b * a.dh_batch + i * a.dh_row;
        const T* g = static_cast<const T*>(a.gu) + b * a.gu_batch + i * a.gu_row;
        float dg[V], du[V], none = 0.0f;
        uint32_t m = 0;
        if (a.codes) {
            for (int64_t c = (int64_t)threadIdx.x * V; c < a.F; c += kRowLanes * V) {
                gated_grad<T, ACT>(load_row<T>(dh, (int)c, (int)a.F), load_row<T>(g, (int)c, (int)a.F), load_row<T>(g + a.F, (int)c, (int)a.F), dg, du);
#pragma unroll
                for (int e = 0; e < V; ++e) m = max(m, max(mag_bits(dg[e]), mag_bits(du[e])));
            }
            RowReduce<kRowLanes>::run(none, m, sh, turn);
        }
        const float d = delta_from_absmax_bits(m, a.qmax), rho = 1.0f / d;
        if (threadIdx.x == 0 && a.delta) a.delta[id] = d;
        for (int64_t c = (int64_t)threadIdx.x * V; c < a.F; c += kRowLanes * V) {
            const int left = (int)min((int64_t)V, a.F - c);
            gated_grad<T, ACT>(load_row<T>(dh, (int)c, (int)a.F), load_row<T>(g, (int)c, (int)a.F), load_row<T>(g + a.F, (int)c, (int)a.F), dg, du);
            const int64_t p = id * 2 * a.F + c;
            gated_grad_out<T, MODE, false>(a, p, dg, left, rho);
            gated_grad_out<T, MODE, false>(a, p + a.F, du, left, rho);
        }
    }
}

template <typename T, int MODE, int ACT> qmm_status launch_gated_grad(const GatedGradArgs& a, bool stream, hipStream_t s)
{
    const int64_t total = a.batch * a.rows;
    if (a.F > kRowElements) gated_grad_long<T, MODE, ACT><<<row_blocks(total, 1), kRowLanes, 0, s>>>(a);
    else for_row_size<T>(a.F, [&](auto lpr, auto nv) {
        constexpr int threads = lpr.value > 256 ? lpr.value : 256;
        if constexpr (lpr.value >= kWave) {
            if (stream) { gated_grad_rows<T, MODE, ACT, lpr.value, nv.value, true><<<row_blocks(total, threads / lpr.value), threads, 0, s>>>(a); return; }
        }
        gated_grad_rows<T, MODE, ACT, lpr.value, nv.value, false><<<row_blocks(total, threads / lpr.value), threads, 0, s>>>(a);
    });
    return launch_status();
}
template <typename T, int MODE> qmm_status launch_gated_act(const GatedGradArgs& a, qmm_activation act, bool stream, hipStream_t s)
{
    return act == QMM_ACT_SILU ? launch_gated_grad<T, MODE, QMM_ACT_SILU>(a, stream, s) : launch_gated_grad<T, MODE, QMM_ACT_GELU>(a, stream, s);
}

}  // namespace
}  // namespace qmm

using namespace qmm;

extern "C" qmm_status qmm_gated_backward(const qmm_tensor* dh, const qmm_tensor* gu, qmm_activation act, qmm_format fmt, qmm_round mode,
                                         uint64_t seed, uint64_t offset, void* dgu_out, float* delta_out, uint8_t* codes_out, void* stream)
{
    if (!dh || !gu) return QMM_ERR_NULL;
    qmm_status st = check_rows(dh);
    if (st != QMM_OK) return st;
    st = check_rows(gu);
    if (st != QMM_OK) return st;
    if (gu->batch != dh->batch || gu->rows != dh->rows || gu->cols != 2 * dh->cols) return QMM_ERR_SHAPE;
    if (gu->dtype != dh->dtype) return QMM_ERR_UNSUPPORTED;
    if (act != QMM_ACT_SILU && act != QMM_ACT_GELU) return QMM_ERR_ENUM;
    if (fmt != QMM_FMT_INT8 && fmt != QMM_FMT_E4M3 && fmt != QMM_FMT_E5M2) return QMM_ERR_ENUM;
    if (mode != QMM_ROUND_RTNE && mode != QMM_ROUND_STOCHASTIC) return QMM_ERR_ENUM;
    if (dh->batch * dh->rows == 0 || (dh->cols == 0 && !delta_out)) return QMM_OK;
    if (dh->cols > 0) {
        if ((codes_out != nullptr) != (delta_out != nullptr)) return QMM_ERR_NULL;
        if (!dh->data || !gu->data || (!codes_out && !dgu_out)) return QMM_ERR_NULL;
    }
    if (!element_aligned(dh->data, dh->dtype) || !element_aligned(gu->data, gu->dtype) || !element_aligned(dgu_out, dh->dtype) ||
        !element_aligned(delta_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    if (dgu_out && dgu_out == dh->data) return QMM_ERR_SHAPE;
    if (dgu_out && dgu_out == gu->data && !dense(gu)) return QMM_ERR_SHAPE;

    GatedGradArgs a{};
    a.dh = dh->data; a.dh_batch = dh->batch_stride; a.dh_row = dh->row_stride;
    a.gu = gu->data; a.gu_batch = gu->batch_stride; a.gu_row = gu->row_stride;
    a.dgu = dgu_out; a.delta = delta_out; a.codes = codes_out;
    a.batch = dh->batch; a.rows = dh->rows; a.F = dh->cols;
    a.seed = seed; a.offset = offset; a.qmax = host_qmax(fmt); a.fmt = fmt;
    // From 64 MB of dh on, i.e. 128 MB of dgu, half of what the memory-side cache holds: bfloat16 16384 x 4096 142 -> 120 us, binary32 4096 x 8192 133 -> 123
    // (the loads alone 140, 134).
    const bool streaming = streams(dh) && streams(gu) && aligned16(dgu_out);
    hipStream_t s = as_stream(stream);
    if (dh->dtype == QMM_DT_BF16)
        return mode == QMM_ROUND_RTNE ? launch_gated_act<uint16_t, QMM_ROUND_RTNE>(a, act, streaming, s) : launch_gated_act<uint16_t, QMM_ROUND_STOCHASTIC>(a, act, streaming, s);
    return mode == QMM_ROUND_RTNE ? launch_gated_act<float, QMM_ROUND_RTNE>(a, act, streaming, s) : launch_gated_act<float, QMM_ROUND_STOCHASTIC>(a, act, streaming, s);
}
