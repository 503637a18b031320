// qmm_quantize_blocks: step sizes and FP8 codes (Eq. 1) with a scale group of its own for every block of 128 elements along the contracting axis and one
// row, or 128 rows, along the other one.  A block is small enough to stay in registers between its maximum and its codes, so x is read once whatever the
// axis, and once for both axes (a gradient is contracted over its columns by the data gradient's product and over its rows by the weight gradient's).
// Bound by memory traffic: 16384 x 4096 bfloat16 is read once and leaves as codes along both axes in 56 us (4.8 TB/s), along one in 35 to 38 (5.3 to 5.8),
// 8192 x 4096 binary32 in 45 and 30 to 31.
#include "qmm_blocks.h"

namespace qmm {
namespace {

struct BlockArgs {
    const void* x;
    int64_t batch, rows, cols, batch_stride, row_stride;
    // contracting over columns: delta [batch][ceil(cols / 128)][row blocks], codes [batch][rows][cols]; over rows: the same of the transposed matrix
    float* delta; uint8_t* codes;
    float* delta_t; uint8_t* codes_t;
    uint64_t seed, offset;
    float qmax;
};

template <typename T> constexpr int kTileThreads = kBlock * kBlock / 4 / Vec<T>::V;              // four vectors each

// Maxima per position over the lanes that lie a multiple of CG apart.
template <int CG, typename T> QMM_DEV void over_quads(VecMax<T>& most)
{
    static_assert(CG == 16 || CG == 32, "rows of lanes");
    uint32_t m[4], other[4];
    if constexpr (CG == 16) {
        most.words(m);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const auto p = __builtin_amdgcn_permlane16_swap(m[j], m[j], false, false);
            const uint32_t first = p[0], second = p[1];
            m[j] = first; other[j] = second;
        }
        most.fold_words(m);
        most.fold_words(other);
    }
    most.words(m);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto p = __builtin_amdgcn_permlane32_swap(m[j], m[j], false, false);
        const uint32_t first = p[0], second = p[1];
        m[j] = first; other[j] = second;
    }
    most.fold_words(m);
    most.fold_words(other);
}

// One step size per row and 128 columns, contracting over columns: eight lanes hold a block, sixteen elements each.
template <typename T, int FMT, int MODE> __global__ void __launch_bounds__(kThreads)
block_rows(BlockArgs a)
{
    constexpr int V = Vec<T>::V, NV = 16 / V;
    const int64_t blocks = (a.cols + kBlock - 1) / kBlock, units = blocks * 8, total = a.batch * a.rows * units;
    const int64_t whole = (total + kWave - 1) / kWave * kWave;               // (all lanes of a wavefront go through the exchange)
    for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v < whole; v += (int64_t)gridDim.x * kThreads) {
        const bool live = v < total;
        const int64_t id = !live ? 0 : total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)v / (uint32_t)units) : v / units;
        const int unit = live ? (int)(v - id * units) : 0;
        const int64_t b = a.batch > 1 ? id / a.rows : 0, i = id - b * a.rows;
        const int cols = live ? (int)a.cols : 0, c = unit * 16;
        const T* x = static_cast<const T*>(a.x) + b * a.batch_stride + i * a.row_stride;
        u32x4 w[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) w[k] = fetch_row<T>(x, c + k * V, cols);
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            w[k] = settle_row<T>(w[k], c + k * V, cols);
            m = max(m, Vec<T>::max_bits(w[k]));
        }
#pragma unroll
        for (int off = 4; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, kWave));
        if (c >= cols) continue;
        const float d = delta_from_absmax_bits(m, a.qmax), rho = 1.0f / d;
        if ((unit & 7) == 0) a.delta[(b * blocks + (unit >> 3)) * a.rows + i] = d;
        const int64_t p = id * a.cols + c;
        float t[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) t[e] = Vec<T>::at(w[e / V], e % V) * rho;
        const uint64_t g = (uint64_t)p + a.offset;
        uint32_t q[4];
        encode_quads<FMT, MODE, 4>(t, g, a.seed, MODE == QMM_ROUND_STOCHASTIC && !__any((g & 3u) != 0u), q);
        const u32x4 codes = {q[0], q[1], q[2], q[3]};
        if (c + 16 <= cols) *reinterpret_cast<u32x4_byte*>(a.codes + p) = codes;
        else store_bytes<16>(a.codes + p, codes, cols - c);
    }
}

// Tiles of 128 x 128 in registers: step sizes per row, per column or of the whole tile (SQUARE), codes contracting over columns (ROWS), over rows (COLS), or
// both.  A thread holds four neighbouring rows of a vector of columns: their codes are a dword of each column's codes, which are put together in LDS.  The
// maxima go through LDS as well, so that one thread makes a step size and its reciprocal (some twenty instructions each) for all.  (By 256 threads that held
// eight rows, each with every step size it needed made by itself and every quotient clamped, 16384 x 4096 bfloat16 took 94 us along both axes: 231 registers, two
// wavefronts a SIMD.  Capped at 64 registers this kernel spills and takes 94 as well.)  A wavefront reads four rows' 256 bytes at a time; neighbouring
// tiles of a row run together, since those below each other, whose lines lie rows apart, are slower (56 -> 60, binary32 45 -> 60).
template <typename T, int FMT, int MODE, bool SQUARE, bool ROWS, bool COLS> __global__ void __launch_bounds__(kTileThreads<T>)
block_tiles(BlockArgs a, uint32_t tiles_c, uint32_t tiles_r, int64_t tiles)
{
    constexpr int V = Vec<T>::V, CG = kBlock / V, THREADS = kTileThreads<T>, WAVES = THREADS / kWave, GROUPS = SQUARE ? 1 : (ROWS ? kBlock : 0) + (COLS ? kBlock : 0);
    __shared__ __attribute__((aligned(16))) uint8_t tile[COLS ? kBlock * kBlock : 16];
    __shared__ __attribute__((aligned(16))) u32x4 s_cols[COLS && !SQUARE ? WAVES * CG : 1];          // each wavefront's maxima of the columns
    __shared__ uint32_t s_rows[SQUARE ? WAVES : kBlock];                                             // the rows' maxima, or each wavefront's
    __shared__ __attribute__((aligned(16))) float s_rho[GROUPS];                                     // of the columns, then of the rows
    const int tid = (int)threadIdx.x, cg = tid % CG, r = tid / CG * 4, wave = tid / kWave, lane = tid % kWave, c = cg * V;
    // 16-byte chunk c of column n's codes lies at chunk position c ^ (n / 8): the dword stores of a wavefront meet in pairs at most
    auto place = [](int n, int k) { return n * kBlock + ((((k >> 4) ^ (n >> 3)) & 7) << 4) + (k & 15); };
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t q = t / tiles_c, b = q / tiles_r;
        const int tc = (int)(t - q * tiles_c), tr = (int)(q - b * tiles_r);
        const int64_t r0 = (int64_t)tr * kBlock, c0 = (int64_t)tc * kBlock;
        const int rows = (int)min((int64_t)kBlock, a.rows - r0), cols = (int)min((int64_t)kBlock, a.cols - c0);       // of the tile, inside the matrix
        const int left = cols - c;
        const T* base = static_cast<const T*>(a.x) + b * a.batch_stride + (r0 + r) * a.row_stride + c0 + c;
        u32x4 w[4];
        if (rows == kBlock && cols == kBlock) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const u32x4_any*>(base + i * a.row_stride);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = u32x4{0u, 0u, 0u, 0u};
                if (r + i < rows) w[i] = load_columns<T, V>(base + i * a.row_stride, min(left, V));
            }
        }
        if constexpr (SQUARE) {
            VecMax<T> most;
#pragma unroll
            for (int i = 0; i < 4; ++i) most.fold(w[i]);
            const uint32_t m = over_lanes<kWave>(most.finish(), Most{});
            if (lane == 0) s_rows[wave] = m;
        } else {
            if constexpr (ROWS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t m = over_lanes<CG>(Vec<T>::max_bits(w[i]), Most{});
                    if (cg == 0) s_rows[r + i] = m;
                }
            }
            if constexpr (COLS) {
                VecMax<T> most;
#pragma unroll
                for (int i = 0; i < 4; ++i) most.fold(w[i]);
                over_quads<CG>(most);
                uint32_t m[4];
                most.words(m);
                if (lane < CG) s_cols[wave * CG + cg] = u32x4{m[0], m[1], m[2], m[3]};
            }
        }
        __syncthreads();
        if (tid < GROUPS) {
            const bool col = !SQUARE && COLS && tid < kBlock;
            uint32_t m = 0;
            if constexpr (SQUARE) {
#pragma unroll
                for (int k = 0; k < WAVES; ++k) m = max(m, s_rows[k]);
            } else if (col) {
                const T* p = reinterpret_cast<const T*>(s_cols) + tid;
#pragma unroll
                for (int k = 0; k < WAVES; ++k) m = max(m, mag_bits<T>(p[k * kBlock]));
            } else m = s_rows[tid % kBlock];
            const float d = delta_from_absmax_bits(m, a.qmax);
            s_rho[tid] = 1.0f / d;
            if constexpr (SQUARE) {
                if (ROWS) a.delta[(b * tiles_c + tc) * tiles_r + tr] = d;
                if (COLS) a.delta_t[(b * tiles_r + tr) * tiles_c + tc] = d;
            } else if (col) {
                if (tid < cols) a.delta_t[(b * tiles_r + tr) * a.cols + c0 + tid] = d;
            } else if (tid % kBlock < rows) a.delta[(b * tiles_c + tc) * a.rows + r0 + tid % kBlock] = d;
        }
        __syncthreads();
        // A step size from infinity or NaN has a reciprocal that is not above zero; all others have one that is.
        if constexpr (ROWS) {
            float rho[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) rho[i] = SQUARE ? s_rho[0] : s_rho[(COLS ? kBlock : 0) + r + i];
            const bool known = MODE == QMM_ROUND_RTNE && __all(rho[0] > 0.0f && rho[1] > 0.0f && rho[2] > 0.0f && rho[3] > 0.0f);
            const int64_t at0 = (b * a.rows + r0 + r) * a.cols + c0 + c;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t at = at0 + i * a.cols;
                u32x2 codes;
                if (known) {
                    codes = u32x2{0u, 0u};
#pragma unroll
                    for (int e = 0; e < V; e += 4)
                        codes[e / 4] = encode_finite<FMT>(Vec<T>::at(w[i], e) * rho[i], Vec<T>::at(w[i], e + 1) * rho[i], Vec<T>::at(w[i], e + 2) * rho[i], Vec<T>::at(w[i], e + 3) * rho[i]);
                } else codes = encode_vec<T, FMT, MODE>(w[i], rho[i], (uint64_t)at + a.offset, a.seed);
                if (r + i < rows && left > 0) store_row_codes<T>(a.codes + at, codes, left);
            }
        }
        if constexpr (COLS) {
            float rho[V];
            bool known = MODE == QMM_ROUND_RTNE;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                rho[e] = s_rho[SQUARE ? 0 : c + e];
                known = known && rho[e] > 0.0f;
            }
            known = __all(known);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v[4] = {Vec<T>::at(w[0], e) * rho[e], Vec<T>::at(w[1], e) * rho[e], Vec<T>::at(w[2], e) * rho[e], Vec<T>::at(w[3], e) * rho[e]};
                uint32_t code[1];
                if (known) code[0] = encode_finite<FMT>(v[0], v[1], v[2], v[3]);
                else {
                    const uint64_t g = (uint64_t)((b * a.cols + c0 + c + e) * a.rows + r0 + r) + a.offset;
                    encode_quads<FMT, MODE, 1>(v, g, a.seed, MODE == QMM_ROUND_STOCHASTIC && !__any((g & 3u) != 0u), code);
                }
                *reinterpret_cast<uint32_t*>(tile + place(c + e, r)) = code[0];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kBlock * 8 / THREADS; ++k) {                 // eight lanes a column, 16 bytes each
                const int n = tid / 8 + k * (THREADS / 8), from = tid % 8 * 16;
                if (n < cols && from < rows) {
                    const u32x4 codes = *reinterpret_cast<const u32x4*>(tile + place(n, from));
                    uint8_t* out = a.codes_t + (b * a.cols + c0 + n) * a.rows + r0 + from;
                    if (from + 16 <= rows) *reinterpret_cast<u32x4_byte*>(out) = codes;
                    else store_bytes<16>(out, codes, rows - from);
                }
            }
        }
        // (No barrier here: what the next tile writes first was read in front of the second barrier, the reciprocals and codes it writes behind its own.)
    }
}

template <typename T, int FMT, int MODE> qmm_status launch_blocks(const BlockArgs& a, bool square, hipStream_t s)
{
    const int64_t tiles_c = (a.cols + kBlock - 1) / kBlock, tiles_r = (a.rows + kBlock - 1) / kBlock, tiles = tiles_c * tiles_r * a.batch;
    const unsigned grid = (unsigned)std::min<int64_t>(tiles, ((int64_t)1 << 31) / kTileThreads<T>);       // (a launch takes less than 2^32 threads; the others follow in turn)
#define QMM_TILES(SQ, R, C) block_tiles<T, FMT, MODE, SQ, R, C><<<grid, kTileThreads<T>, 0, s>>>(a, (uint32_t)tiles_c, (uint32_t)tiles_r, tiles)
    if (square) {
        if (a.codes && a.codes_t) QMM_TILES(true, true, true);
        else if (a.codes) QMM_TILES(true, true, false);
        else QMM_TILES(true, false, true);
    } else if (a.codes_t) {
        if (a.codes) QMM_TILES(false, true, true);
        else QMM_TILES(false, false, true);
    } else {
        // Step sizes per row, codes along the columns alone: by tiles where these fill the card, since a tile's step sizes are neighbours in memory
        // (16384 x 4096 bfloat16 35 us against 40 by rows, 8192 x 4096 binary32 30 / 36, 16384 x 1024 11.4 / 12.3); fewer by rows, which have no barrier.
        if (a.rows >= kBlock && a.batch * a.rows * tiles_c >= 512 * kBlock) { QMM_TILES(false, true, false); return launch_status(); }
        const int64_t units = a.batch * a.rows * tiles_c * 8;
        block_rows<T, FMT, MODE><<<(unsigned)std::min<int64_t>((units + kThreads - 1) / kThreads, 1 << 22), kThreads, 0, s>>>(a);
    }
#undef QMM_TILES
    return launch_status();
}
template <typename T> qmm_status launch_blocks_form(const BlockArgs& a, bool square, int fmt, qmm_round mode, hipStream_t s)
{
    if (fmt == QMM_FMT_E4M3) return mode == QMM_ROUND_RTNE ? launch_blocks<T, QMM_FMT_E4M3, QMM_ROUND_RTNE>(a, square, s) : launch_blocks<T, QMM_FMT_E4M3, QMM_ROUND_STOCHASTIC>(a, square, s);
    return mode == QMM_ROUND_RTNE ? launch_blocks<T, QMM_FMT_E5M2, QMM_ROUND_RTNE>(a, square, s) : launch_blocks<T, QMM_FMT_E5M2, QMM_ROUND_STOCHASTIC>(a, square, s);
}

}  // namespace
}  // namespace qmm

using namespace qmm;

extern "C" int64_t qmm_num_block_scales(int64_t batch, int64_t rows, int64_t K, int32_t block_rows)
{
    if (batch < 0 || rows < 0 || K < 0 || (block_rows != 1 && block_rows != kBlock)) return -1;
    return batch * ((K + kBlock - 1) / kBlock) * ((rows + block_rows - 1) / block_rows);
}

extern "C" qmm_status qmm_quantize_blocks(const qmm_tensor* x, qmm_format fmt, int32_t block_rows, qmm_round mode, uint64_t seed, uint64_t offset,
                                          float* delta_out, uint8_t* codes_out, float* delta_t_out, uint8_t* codes_t_out, void* stream)
{
    if (!x) return QMM_ERR_NULL;
    if (x->dtype != QMM_DT_BF16 && x->dtype != QMM_DT_F32) return QMM_ERR_ENUM;
    if (x->contract_axis != 0 && x->contract_axis != 1) return QMM_ERR_ENUM;
    if (x->batch < 0 || x->rows < 0 || x->cols < 0 || x->row_stride < x->cols) return QMM_ERR_SHAPE;
    if (x->batch > 1 && x->rows > 0 && x->batch_stride < (x->rows - 1) * x->row_stride + x->cols) return QMM_ERR_SHAPE;
    if (fmt == QMM_FMT_INT8) return QMM_ERR_UNSUPPORTED;
    if (fmt != QMM_FMT_E4M3 && fmt != QMM_FMT_E5M2) return QMM_ERR_ENUM;
    if (block_rows != 1 && block_rows != kBlock) return QMM_ERR_ENUM;
    if (mode != QMM_ROUND_RTNE && mode != QMM_ROUND_STOCHASTIC) return QMM_ERR_ENUM;
    if (!delta_t_out != !codes_t_out) return QMM_ERR_NULL;
    if (x->batch > 65535 || x->rows > 0x7FFFFFFF - kBlock || x->cols > 0x7FFFFFFF - kBlock) return QMM_ERR_UNSUPPORTED;
    if (x->batch == 0 || x->rows == 0 || x->cols == 0) return QMM_OK;
    if (!x->data || !delta_out || !codes_out) return QMM_ERR_NULL;
    if (!element_aligned(x->data, x->dtype) || !element_aligned(delta_out, QMM_DT_F32) || !element_aligned(delta_t_out, QMM_DT_F32)) return QMM_ERR_ALIGN;
    BlockArgs a{};
    a.x = x->data; a.batch = x->batch; a.rows = x->rows; a.cols = x->cols;
    a.batch_stride = x->batch_stride; a.row_stride = x->row_stride;
    const bool along = x->contract_axis == 1;
    a.delta = along ? delta_out : delta_t_out; a.codes = along ? codes_out : codes_t_out;
    a.delta_t = along ? delta_t_out : delta_out; a.codes_t = along ? codes_t_out : codes_out;
    a.seed = seed; a.offset = offset; a.qmax = host_qmax(fmt);
    hipStream_t s = as_stream(stream);
    return x->dtype == QMM_DT_BF16 ? launch_blocks_form<uint16_t>(a, block_rows == kBlock, fmt, mode, s) : launch_blocks_form<float>(a, block_rows == kBlock, fmt, mode, s);
}
