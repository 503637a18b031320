// qmm_gemm_blocks: product of two FP8 operands with a step size for every block of 128 elements along the contraction and one or 128 rows.
//
//   y_ij = sum over blocks t of  (sum_{k in t} a_ik b_jk) da[t][i] db[t][j]
//
// One matrix instruction (v_mfma_f32_16x16x128_f8f6f4) contracts a whole block, so its result, started from zero, is what the step sizes multiply: four
// multiply-adds of a lane an instruction, into accumulators in vector registers, beside matrix instructions of the SIMD's other wavefront.
// The second operand (the weights) feeds the instruction's first input: a lane then holds four of its rows and one row of the first operand (a token), so
// where the weights' step sizes are per 128 rows, a wavefront has one of them and a lane one factor da db per token; with a step size per row of
// both, a product more an element.
// Operands are [rows][K] with K contiguous; a slab of 128 bytes a row is staged in LDS by copies that need no registers, 16-byte chunk c of LDS row p at
// position c ^ ((p >> 1) & 7), its step sizes beside it.  K bytes [16 q, +16) and [64 + 16 q, +16) of a slab belong to lanes 16 q .. 16 q + 15, as in the plain
// product, so that a block's sum is that product's, bit for bit.
#include <algorithm>
#include <atomic>
#include <type_traits>
#include <utility>
#include "qmm_block_plan.h"
#include "qmm_encode.h"

namespace qmm {
namespace {

constexpr int kNumXcd = 8;
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));

struct BlockGemmArgs {
    const uint8_t* a; const uint8_t* b;        // codes [batch][M][K], [batch][N][K]
    const float* da; const float* db;          // step sizes [batch][K blocks][row blocks]
    int a_shift, b_shift;                      // row >> shift: its row block
    int64_t a_blocks, b_blocks;                // row blocks
    int64_t M, N, K, batch;
    void* y; int y_bf16;
    float* partial;                            // [splits][batch][M][N] where K is split
    int splits;
    int tiles_m, tiles_n;
};

// 16 (4) bytes per lane from global memory into LDS, source a wavefront-uniform base and a 32-bit byte offset per lane, target a wavefront-uniform LDS address.
QMM_DEV void copy16(const void* base, uint32_t lane_offset, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_addr), "v"(lane_offset), "s"(base) : "memory", "m0");
}
QMM_DEV void copy4(const void* base, uint32_t lane_offset, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(lds_addr), "v"(lane_offset), "s"(base) : "memory", "m0");
}
template <int N> QMM_DEV void wait_copies()
{
    static_assert(N >= 0 && N <= 63, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}
QMM_DEV uint32_t pack_bf16(float a, float b)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, bf2));
}
// One block's sums of 16 rows of the weights (format FB) and 16 tokens (format FA).
template <int FA, int FB> QMM_DEV v4f block_sums(const v8i& weights, const v8i& tokens)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(weights, tokens, v4f{0.0f, 0.0f, 0.0f, 0.0f}, FB == QMM_FMT_E5M2 ? 1 : 0,
                                                            FA == QMM_FMT_E5M2 ? 1 : 0, 0, 0, 0, 0);
}
// f(0), f(1), .. as constants: sequences of instructions that are too long for the compiler to unroll a loop.
template <typename F, int... N> QMM_DEV void in_order(F&& f, std::integer_sequence<int, N...>) { (f(std::integral_constant<int, N>{}), ...); }
// Up to eight neighbouring outputs of a row.
QMM_DEV void store8(void* out, bool bf16, int64_t at, const float (&v)[8], int64_t left)
{
    if (bf16) {
        uint16_t* p = static_cast<uint16_t*>(out) + at;
        const u32x4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if (left >= 8) *reinterpret_cast<u32x4_any*>(p) = w;
        else store_bytes<16>(reinterpret_cast<uint8_t*>(p), w, (int)left * 2);
    } else {
        float* p = static_cast<float*>(out) + at;
        const u32x4 w0 = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        const u32x4 w1 = {__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        if (left >= 4) *reinterpret_cast<u32x4_any*>(p) = w0;
        else store_bytes<16>(reinterpret_cast<uint8_t*>(p), w0, (int)left * 4);
        if (left >= 8) *reinterpret_cast<u32x4_any*>(p + 4) = w1;
        else if (left > 4) store_bytes<16>(reinterpret_cast<uint8_t*>(p + 4), w1, (int)(left - 4) * 4);
    }
}

// WN x WM wavefronts of 16 TN rows of the weights x 16 TM tokens; SLOTS slabs in LDS, all but one on their way.  PER_ROW: the weights have a step size per row.
// (Two wavefronts a SIMD as the bound: with one the compiler has the matrix results in accumulation registers, out of which each is read behind a wait for it, and
// 2048 x 2048 x 2048 takes 24.4 us instead of 17.4.)
template <int FA, int FB, int WN, int WM, int TN, int TM, int SLOTS, bool PER_ROW>
__global__ void __launch_bounds__(64 * WN * WM, 2)
block_gemm(BlockGemmArgs g)
{
    constexpr int BN = 16 * WN * TN, BM = 16 * WM * TM, ROWS = BN + BM, WAVES = WN * WM;
    constexpr int UNITS = ROWS / 8 / WAVES;                    // copies of 8 LDS rows a wavefront and slab
    constexpr int SLOT = ROWS * kBlock + ROWS * 4;             // a slab's rows (weights, then tokens), then their step sizes
    constexpr int STEPS = (ROWS / 64 + WAVES - 1) / WAVES;     // copies of 64 step sizes a wavefront and slab (some twice, so that every wavefront counts alike)
    constexpr int COPIES = UNITS + STEPS;
    static_assert(ROWS % (8 * WAVES) == 0 && TN % 2 == 0 && kBlock % (16 * TN) == 0 && (SLOTS - 1) * COPIES <= 63, "tile");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];

    const int lane = threadIdx.x & 63, q = lane >> 4, j16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wm = wave / WN;
    // Workgroups go to the XCDs in turn: each XCD gets a run of tiles, bands of eight tiles of tokens, so that its L2 holds what they share.
    const uint32_t per_matrix = (uint32_t)g.tiles_m * (uint32_t)g.tiles_n, per_split = per_matrix * (uint32_t)g.batch;
    const uint32_t total = per_split * (uint32_t)g.splits, xcd = blockIdx.x % kNumXcd, even = total / kNumXcd, odd = total % kNumXcd;
    uint32_t t = xcd * even + min(xcd, odd) + blockIdx.x / kNumXcd;
    const int split = __builtin_amdgcn_readfirstlane((int)(t / per_split));
    t -= (uint32_t)split * per_split;
    const int64_t bidx = __builtin_amdgcn_readfirstlane((int)(t / per_matrix));
    t -= (uint32_t)bidx * per_matrix;
    constexpr uint32_t BAND = 8;
    const uint32_t band = t / (BAND * (uint32_t)g.tiles_n), in_band = t - band * BAND * (uint32_t)g.tiles_n;
    const uint32_t height = min(BAND, (uint32_t)g.tiles_m - band * BAND);
    const int64_t m0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(band * BAND + in_band % height)) * BM;
    const int64_t n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(in_band / height)) * BN;
    const int rowbytes = (int)g.K, slabs = (rowbytes + kBlock - 1) / kBlock;
    const int begin = (int)((int64_t)slabs * split / g.splits), end = (int)((int64_t)slabs * (split + 1) / g.splits);
    const uint8_t* a_tile = g.a + (bidx * g.M + m0) * g.K;
    const uint8_t* b_tile = g.b + (bidx * g.N + n0) * g.K;
    const float* da = g.da + bidx * slabs * g.a_blocks + (m0 >> g.a_shift);
    const float* db = g.db + bidx * slabs * g.b_blocks + (n0 >> g.b_shift);

    // LDS row p of the weights is their row weight_row(p): register v of tile i, lanes 16 q ..: columns 32 (i / 2) + 8 q + 4 (i % 2) + v of the wavefront's, so that
    // two tiles make eight neighbouring outputs of a lane.
    auto weight_row = [](int p) {
        const int w = p / (16 * TN), i = p % (16 * TN) / 16, r = p % 16;
        return w * 16 * TN + (i / 2) * 32 + (r / 4) * 8 + (i % 2) * 4 + r % 4;
    };
    // rows past the last are the last one again: their outputs are not stored
    auto a_row = [&](int p) { return (int)min((int64_t)p, g.M - 1 - m0); };
    auto b_row = [&](int p) { return (int)min((int64_t)weight_row(p), g.N - 1 - n0); };
    uint32_t src[UNITS];
    auto chunk = [&](int unit) { return ((lane & 7) ^ ((unit & 1) * 4 + (lane >> 4))) * 16; };      // p >> 1 of rows p = 8 unit + lane / 8
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int p = (wave * UNITS + u) * 8 + (lane >> 3);
        src[u] = (uint32_t)(p < BN ? b_row(p) : a_row(p - BN)) * (uint32_t)rowbytes + (uint32_t)chunk(wave * UNITS + u);
    }
    uint32_t step_src[STEPS];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
        const int p = ((wave + u * WAVES) % (ROWS / 64)) * 64 + lane;
        step_src[u] = 4u * (uint32_t)(p < BN ? ((n0 + b_row(p)) >> g.b_shift) - (n0 >> g.b_shift) : ((m0 + a_row(p - BN)) >> g.a_shift) - (m0 >> g.a_shift));
    }
    typedef __attribute__((address_space(3))) uint8_t* lds_ptr_t;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    auto copy_slab = [&](int slab, int slot) {
        const int k0 = slab * kBlock;
        auto base_of = [&](int unit) { return (unit * 8 < BN ? b_tile : a_tile) + k0; };         // (a unit is of one operand: BN is a multiple of 8)
        const uint32_t to = (uint32_t)(slot * SLOT + wave * (UNITS * 1024));
        if (k0 + kBlock <= rowbytes) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) copy16(base_of(wave * UNITS + u), src[u], lds_at + to + u * 1024);
        } else {
            asm volatile("; rows that end within the slab");   // (keeps the compiler from asking at every copy)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                // (a chunk past the end of the rows: zeros; the first one never is, so every slab counts the same number of copies)
                const bool there = k0 + chunk(wave * UNITS + u) < rowbytes;
                if (there) copy16(base_of(wave * UNITS + u), src[u], lds_at + to + u * 1024);
                else *reinterpret_cast<u32x4*>(lds + to + u * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
            }
        }
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int group = (wave + u * WAVES) % (ROWS / 64);
            const float* base = group * 64 < BN ? db + (int64_t)slab * g.b_blocks : da + (int64_t)slab * g.a_blocks;
            copy4(base, step_src[u], lds_at + (uint32_t)(slot * SLOT + ROWS * kBlock + group * 256));
        }
    };

    v4f acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    const int coff = (q ^ ((j16 >> 1) & 7)) * 16;
    auto fragment = [&](const uint8_t* row) -> v8i {
        const v4i p0 = *reinterpret_cast<const v4i*>(row + coff), p1 = *reinterpret_cast<const v4i*>(row + (coff ^ 64));
        return v8i{p0[0], p0[1], p0[2], p0[3], p1[0], p1[1], p1[2], p1[3]};
    };
    const uint8_t* const weights = lds + (wn * 16 * TN + j16) * kBlock;        // of slot 0, as are the following
    const uint8_t* const tokens = lds + (BN + wm * 16 * TM + j16) * kBlock;
    const uint8_t* const token_steps = lds + ROWS * kBlock + (BN + wm * 16 * TM + j16) * 4;
    const uint8_t* const row_steps = lds + ROWS * kBlock + wn * 16 * TN * 4;

    // Matrix instruction number n of a slab is of tile n / TM of the weights and n % TM of the tokens; behind it stand the multiply-adds of the one LAG before it, whose
    // result has arrived.  The order is pinned group by group: left to itself the compiler puts the multiply-adds right behind their instruction and waits for
    // it, each time.  Likewise a tile's fragment is read a row of instructions ahead.
    constexpr int LAG = 2, RING = 4, COUNT = TN * TM;
    static_assert(TM >= LAG && COUNT % RING == 0, "results of one slab's end and the next one's start stay apart");
    v4f ring[RING], sb[2];
    v8i fw[2], ft[TM];
    float sa[TM], sa_last[LAG], sa_next[TM];
    auto add = [&](int i, int j, const v4f& sum, float a) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = fmaf(PER_ROW ? sum[v] * sb[i & 1][v] : sum[v], a, acc[i][j][v]);
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(acc[i][j]));                    // here, and not behind the barrier, with the results kept until then
#endif
    };
    // a slab's factors: the tokens' step sizes, times the weights' where the wavefront's rows share one
    auto read_token_step = [&](int off, int j) { sa_next[j] = *reinterpret_cast<const float*>(token_steps + off + j * 64); };
    auto read_row_steps = [&](int off, int i) { if constexpr (PER_ROW) sb[i & 1] = *reinterpret_cast<const v4f*>(row_steps + off + i * 64 + q * 16); };
    auto settle_steps = [&](int off) {
        float one = 1.0f;
        if constexpr (!PER_ROW) one = *reinterpret_cast<const float*>(row_steps + off);
#pragma unroll
        for (int k = 0; k < LAG; ++k) sa_last[k] = sa[TM - LAG + k];
#pragma unroll
        for (int j = 0; j < TM; ++j) sa[j] = PER_ROW ? sa_next[j] : sa_next[j] * one;
    };
    auto wait_for = [&](int newer) {                           // all copies but those of the `newer` newest slabs (at most SLOTS - 2) have landed
        if (SLOTS > 2 && newer >= SLOTS - 2) wait_copies<(SLOTS > 2 ? SLOTS - 2 : 0) * COPIES>();
        else if (SLOTS > 3 && newer == 1) wait_copies<(SLOTS > 3 ? COPIES : 0)>();
        else wait_copies<0>();
    };

    if (begin < end) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (begin + s < end) copy_slab(begin + s, s);
        if (SLOTS > 3 && end - begin >= 4) wait_copies<(SLOTS > 3 ? 3 : 0) * COPIES>();
        else if (SLOTS > 2 && end - begin >= 3) wait_copies<(SLOTS > 2 ? 2 : 0) * COPIES>();
        else if (end - begin >= 2) wait_copies<COPIES>();
        else wait_copies<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            ft[j] = fragment(tokens + j * 16 * kBlock);
            read_token_step(0, j);
            sa[j] = 0.0f;                                      // (what is added for the slab before the first: nothing)
        }
        fw[0] = fragment(weights);
        sb[1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        read_row_steps(0, 0);
        settle_steps(0);
#pragma unroll
        for (int k = 0; k < RING; ++k) ring[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        int slot = 0;
        for (int kt = begin; kt < end; ++kt) {
            const int next_slot = slot == SLOTS - 1 ? 0 : slot + 1, at = slot * SLOT, next = next_slot * SLOT;
#pragma unroll
            for (int n = 0; n < COUNT; ++n) {
                const int i = n / TM, j = n % TM;
                ring[n % RING] = block_sums<FA, FB>(fw[i & 1], ft[j]);
                if (j == 0 && i < TN - 1) fw[(i + 1) & 1] = fragment(weights + at + (i + 1) * 16 * kBlock);
                if (i == TN - 1) {                             // (behind the barrier: of the next slab, or, behind the last one, of what is there)
                    ft[j] = fragment(tokens + next + j * 16 * kBlock);
                    if (j == 0) fw[0] = fragment(weights + next);
                    read_token_step(next, j);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (n >= LAG) add((n - LAG) / TM, (n - LAG) % TM, ring[(n - LAG) % RING], sa[(n - LAG) % TM]);
                else add(TN - 1, TM - LAG + n, ring[(COUNT - LAG + n) % RING], sa_last[n]);      // of the slab before
                if (j == LAG - 1) {                            // (the tile before has had its multiply-adds)
                    if (i < TN - 1) read_row_steps(at, i + 1);
                    else read_row_steps(next, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (n == COUNT - TM - 1) {
                    // This wavefront has read all of the slab and its copies of the next one have landed; behind the barrier that holds for every wavefront, so the
                    // next slab may be read and another one take this one's place.
                    wait_for(end - 2 - kt);
                    __builtin_amdgcn_s_barrier();
                    if (kt + SLOTS < end) copy_slab(kt + SLOTS, slot);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            settle_steps(next);
            slot = next_slot;
        }
#pragma unroll
        for (int k = 0; k < LAG; ++k) add(TN - 1, TM - LAG + k, ring[(COUNT - LAG + k) % RING], sa_last[k]);
    }

    void* out = g.splits > 1 ? static_cast<void*>(g.partial + (int64_t)split * g.batch * g.M * g.N) : g.y;
    const bool bf16 = g.splits == 1 && g.y_bf16;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t m = m0 + wm * 16 * TM + 16 * j + j16;
        if (m >= g.M) continue;
#pragma unroll
        for (int i = 0; i < TN; i += 2) {
            const int64_t n = n0 + wn * 16 * TN + 16 * i + 8 * q;
            if (n >= g.N) continue;
            const float v[8] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], acc[i + 1][j][0], acc[i + 1][j][1], acc[i + 1][j][2], acc[i + 1][j][3]};
            store8(out, bf16, (bidx * g.M + m) * g.N + n, v, g.N - n);
        }
    }
}

// The large tile: 256 rows of the weights x 256 tokens, eight wavefronts of 128 x 64, two slabs in LDS.  A workgroup stays on its CU and the slabs of all of its tiles are one
// stream: the copies of a tile's first slabs and its first fragments are requested in the last steps of the tile before, whose outputs leave beside
// them.  A step is 32 matrix instructions of a wavefront, the multiply-adds of each one instruction behind it (two behind: 500 us where this takes 490).  LDS is
// what limits it next to the matrix units (192 KB of fragments a step and CU), so nothing comes in bursts: a row's fragment is read while the row before runs, the
// slab's last row runs behind the barrier, so that a token's fragment of the next slab takes the register of the one just used, and the copies go out one every second
// instruction.
// 8192 x 8192 x 8192 490 us (2.25 PFLOP/s; qmm_gemm's one scale group 380): of 2048 cycles of matrix work a step, LDS gives out fragments in 1536 and takes the copies in 512; with matrix
// instructions and multiply-adds alone, on what LDS happens to hold, it is 298.  16384 x 4096 x 1024 81 to 87 us (qmm_gemm 66; without its stores 66): all CUs finish their tiles together, 33 MB at
// once, and memory operations end in order, so that the second slab of the next tile waits for them.  Slots for more slabs, or registers for outputs that leave later, there are none;
// workgroups that start at different times lose at the end what they gain.
template <int FA, int FB, bool PER_ROW>
__global__ void __launch_bounds__(512, 1)
block_gemm_large(BlockGemmArgs g)
{
    constexpr int WN = 2, TN = 8, TM = 4, BN = 256, BM = 256, ROWS = BN + BM, UNITS = 8, COPIES = UNITS + 1;
    constexpr int SLOT = ROWS * kBlock + ROWS * 4, COUNT = TN * TM, FIRST = COUNT - TM;       // FIRST: the instruction that starts the last row
    constexpr int LAG = 1, RING = 2, APART = 2, EARLY = UNITS - (TM + APART - 1) / APART;      // EARLY: copies of a slab that go out in the step behind the one that frees its place
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];

    const int lane = threadIdx.x & 63, q = lane >> 4, j16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, wm = wave / WN;
    const bool of_a = wave >= 4;                               // the operand whose rows this wavefront copies (64 of them a slab)
    const uint32_t per_matrix = (uint32_t)g.tiles_m * (uint32_t)g.tiles_n, per_split = per_matrix * (uint32_t)g.batch;
    const uint32_t total = per_split * (uint32_t)g.splits, xcd = blockIdx.x % kNumXcd, even = total / kNumXcd, odd = total % kNumXcd;
    const uint32_t stride = (gridDim.x - xcd + kNumXcd - 1) / kNumXcd;         // workgroups of this XCD, which share a run of tiles
    const uint32_t run_end = xcd * even + min(xcd, odd) + even + (xcd < odd ? 1u : 0u);
    const int slabs = (int)((g.K + kBlock - 1) / kBlock);
    struct Tile { int split; int64_t bidx, m0, n0; int begin, end; };
    auto tile_at = [&](uint32_t t) {
        Tile r;
        r.split = __builtin_amdgcn_readfirstlane((int)(t / per_split));
        t -= (uint32_t)r.split * per_split;
        const uint32_t b = t / per_matrix;
        r.bidx = __builtin_amdgcn_readfirstlane((int)b);
        t -= b * per_matrix;
        constexpr uint32_t BAND = 8;                           // bands of eight tiles of tokens: an XCD's run is compact
        const uint32_t band = t / (BAND * (uint32_t)g.tiles_n), in_band = t - band * BAND * (uint32_t)g.tiles_n;
        const uint32_t height = min(BAND, (uint32_t)g.tiles_m - band * BAND);
        r.m0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(band * BAND + in_band % height)) * BM;
        r.n0 = (int64_t)__builtin_amdgcn_readfirstlane((int)(in_band / height)) * BN;
        const uint32_t part = (uint32_t)slabs / (uint32_t)g.splits, more_by = (uint32_t)slabs % (uint32_t)g.splits, at = (uint32_t)r.split;
        r.begin = (int)(at * part + min(at, more_by));
        r.end = r.begin + (int)(part + (at < more_by ? 1u : 0u));
        return r;
    };
    uint32_t t_now = xcd * even + min(xcd, odd) + blockIdx.x / kNumXcd;
    if (t_now >= run_end) return;

    // What a lane derives from its number at the end of a tile is derived there: kept through the steps, which have no register left, it went to scratch memory, and
    // each wait for that one waited for every copy and store before it (16384 x 4096 x 1024 92 -> 84 us).
    auto lane_here = [&]() {
        int l = lane;
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(l));
#endif
        return l;
    };

    // ---- copies.  LDS row p of the weights is their row 32 (p / 32) + 8 (p % 16 / 4) + 4 (p % 32 / 16) + p % 4 (see block_gemm).  A wavefront copies 64 rows of one operand, a
    // unit of 8 rows a copy: of unit u, lane l, that row is a number of u plus one of l / 8.
    auto chunk = [&](int u, int l) { return ((l & 7) ^ ((u & 1) * 4 + (l >> 4))) * 16; };
    const int first = (of_a ? wave - 4 : wave) * 64;           // the wavefront's first LDS row, within the operand
    const uint32_t rowbytes = (uint32_t)g.K, ragged = rowbytes % kBlock;
    const int shift = of_a ? g.a_shift : g.b_shift;
    typedef __attribute__((address_space(3))) uint8_t* lds_ptr_t;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    const uint32_t unit_lds = lds_at + (uint32_t)wave * (UNITS * 1024), step_lds = lds_at + (uint32_t)(ROWS * kBlock + wave * 256);
    // the slab that is copied next
    uint32_t t_copy = t_now;
    int k_copy, k_end;
    const uint8_t* copy_rows; const float* copy_steps;         // of this wavefront's operand: the tile's rows from that slab on, the slab's step sizes
    uint32_t src[UNITS], step_src;                             // a lane's places there
    uint64_t lanes = ~0ull;                                    // none once the stream has ended: its last steps copy nothing
    auto start_copies = [&]() {
        const Tile t = tile_at(t_copy);
        const int64_t blocks = of_a ? g.a_blocks : g.b_blocks, r0 = of_a ? t.m0 : t.n0, rows = of_a ? g.M : g.N;
        k_copy = t.begin; k_end = t.end;
        copy_rows = (of_a ? g.a : g.b) + (t.bidx * rows + r0) * g.K + (int64_t)t.begin * kBlock;
        copy_steps = (of_a ? g.da : g.db) + (t.bidx * slabs + t.begin) * blocks + (r0 >> shift);
        const int last = (int)min(rows - r0, (int64_t)256) - 1;               // rows past the last are the last one again: their outputs are not stored
        const int l = lane_here(), p = l >> 3, row = first + (of_a ? p : (p >> 2) * 8 + (p & 3));
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            src[u] = (uint32_t)min(row + (of_a ? 8 * u : (u >> 2) * 32 + (u & 1) * 16 + (u >> 1 & 1) * 4), last) * rowbytes;
#if defined(__HIP_DEVICE_COMPILE__)
            asm volatile("" : "+v"(src[u]));                   // (a product of its own: as a 64-bit multiply-add it held two registers)
#endif
            src[u] += (uint32_t)chunk(u, l);
        }
        step_src = 4u * (uint32_t)(min(first + (of_a ? l : (l >> 5) * 32 + (l >> 2 & 3) * 8 + (l >> 4 & 1) * 4 + (l & 3)), last) >> shift);
    };
    // The last bytes of rows that end within a slab: chunks behind the end are copied from the row's slab's first one, and overwritten by zeros when they have landed.
    bool ragged_copies = false;
    auto before_copies = [&]() {
        ragged_copies = ragged != 0 && k_copy == slabs - 1 && lanes;
        if (ragged_copies) {
            const int l = lane_here();
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
                if ((uint32_t)chunk(u, l) >= ragged) src[u] -= (uint32_t)chunk(u, l);
        }
    };
    auto clear_ragged = [&](int slot) {
        const int l = lane_here();
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if ((uint32_t)chunk(u, l) >= ragged) *reinterpret_cast<u32x4*>(lds + slot * SLOT + wave * (UNITS * 1024) + u * 1024 + l * 16) = u32x4{0u, 0u, 0u, 0u};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto copy_unit = [&](auto unit, int slot, uint64_t active) __attribute__((always_inline)) {
        constexpr int U = decltype(unit)::value;
        const uint32_t to = unit_lds + (uint32_t)(slot * SLOT), from = src[U];
        const uint8_t* base = copy_rows;
        asm volatile("s_add_u32 m0, %0, %1\n\ts_mov_b64 exec, %2\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b64 exec, -1"
                     :: "s"(to), "n"(U * 1024), "s"(active), "v"(from), "s"(base) : "memory", "m0", "scc");
    };
    auto copy_step = [&](int slot, uint64_t active) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %1\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b64 exec, -1"
                     :: "s"(step_lds + (uint32_t)(slot * SLOT)), "s"(active), "v"(step_src), "s"(copy_steps) : "memory", "m0");
    };
    auto after_copies = [&]() {
        if (!lanes) return;
        ++k_copy;
        copy_rows += kBlock;
        copy_steps += of_a ? g.a_blocks : g.b_blocks;
        if (k_copy == k_end) {
            t_copy += stride;
            if (t_copy < run_end) start_copies();
            else lanes = 0;
        }
    };

    // ---- fragments
    v4f acc[TN][TM];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    };
    clear();
    const int coff = (q ^ ((j16 >> 1) & 7)) * 16;
    const uint8_t* const weights = lds + (wn * 16 * TN + j16) * kBlock + coff;          // of slot 0, as are the following; the other half of a lane's bytes is at ^ 64
    const uint8_t* const weights_h = lds + (wn * 16 * TN + j16) * kBlock + (coff ^ 64);
    const uint8_t* const tokens = lds + (BN + wm * 16 * TM + j16) * kBlock + coff;
    const uint8_t* const tokens_h = lds + (BN + wm * 16 * TM + j16) * kBlock + (coff ^ 64);
    const uint8_t* const token_steps = lds + ROWS * kBlock + (BN + wm * 16 * TM + j16) * 4;
    const uint8_t* const row_steps = lds + ROWS * kBlock + wn * 16 * TN * 4 + (PER_ROW ? q * 16 : 0);
    auto fragment = [&](const uint8_t* p, const uint8_t* h) -> v8i {
        const v4i p0 = *reinterpret_cast<const v4i*>(p), p1 = *reinterpret_cast<const v4i*>(h);
        return v8i{p0[0], p0[1], p0[2], p0[3], p1[0], p1[1], p1[2], p1[3]};
    };
    auto weight_tile = [&](int off, int i) { return fragment(weights + off + i * 16 * kBlock, weights_h + off + i * 16 * kBlock); };
    auto token_tile = [&](int off, int j) { return fragment(tokens + off + j * 16 * kBlock, tokens_h + off + j * 16 * kBlock); };
    v4f ring[RING], sb[PER_ROW ? 2 : 1];                       // step sizes of tile i's rows: i % 2
    v8i fw[2], ft[TM];
    float sa[TM], sa_last[LAG], sa_next[TM], one = 1.0f;
    auto add = [&](int i, int j, const v4f& sum, float a) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = fmaf(PER_ROW ? sum[v] * sb[PER_ROW ? i % 2 : 0][v] : sum[v], a, acc[i][j][v]);
#if defined(__HIP_DEVICE_COMPILE__)
        asm volatile("" : "+v"(acc[i][j]));                    // here, and not behind the barrier, with the results kept until then
#endif
    };
    auto read_token_steps = [&](int off) {
#pragma unroll
        for (int j = 0; j < TM; ++j) sa_next[j] = *reinterpret_cast<const float*>(token_steps + off + j * 64);
    };
    auto read_row_step = [&](int off, int i, int to) {
        if constexpr (PER_ROW) sb[to] = *reinterpret_cast<const v4f*>(row_steps + off + i * 64);
        else one = *reinterpret_cast<const float*>(row_steps + off);
    };

    // ---- the stream
    start_copies();
    bool second = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        second = lanes != 0;
        before_copies();
        in_order([&](auto unit) __attribute__((always_inline)) { copy_unit(unit, s, lanes); }, std::make_integer_sequence<int, UNITS>{});
        copy_step(s, lanes);
        after_copies();
        if (s == 0 && ragged_copies) {                         // (a contraction of one slab)
            wait_copies<0>();
            clear_ragged(0);
        }
    }
    if (second) wait_copies<COPIES>();
    else wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fw[0] = weight_tile(0, 0);
#pragma unroll
    for (int j = 0; j < TM; ++j) ft[j] = token_tile(0, j);
    read_token_steps(0);
    read_row_step(0, 0, 0);
#pragma unroll
    for (int k = 0; k < LAG; ++k) sa[TM - LAG + k] = 0.0f;
    if constexpr (PER_ROW) sb[1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < RING; ++k) ring[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    uint64_t late = 0;                                         // lanes of those copies: none in a tile's first step, they have gone out already
    int slot = 0, kt, k_last, stores = 0;                      // stores: of the tile before, which may be outstanding when this slab's copies are waited for
    {
        const Tile t = tile_at(t_now);
        kt = t.begin; k_last = t.end - 1;
    }
    for (;;) {
        const int at = slot * SLOT, next = SLOT - at;
#pragma unroll
        for (int k = 0; k < LAG; ++k) sa_last[k] = sa[TM - LAG + k];
#pragma unroll
        for (int j = 0; j < TM; ++j) sa[j] = PER_ROW ? sa_next[j] : sa_next[j] * one;
        in_order([&](auto number) __attribute__((always_inline)) {
            constexpr int n = number.value, i = n / TM, j = n % TM;
            ring[n % RING] = block_sums<FA, FB>(fw[i & 1], ft[j]);
            if constexpr (i < TN - 1) {
                if constexpr (j == 0) fw[(i + 1) & 1] = weight_tile(at, i + 1);
            } else {                                           // behind the barrier: of the next slab, or, behind the last one, of what is there
                ft[j] = token_tile(next, j);
                if constexpr (j == 0) fw[0] = weight_tile(next, 0);
                if constexpr (j == 1) read_token_steps(next);
                if constexpr (j % APART == 0) copy_unit(std::integral_constant<int, j / APART>{}, slot, lanes);
            }
            if constexpr (n % APART == 1 && n < APART * EARLY) copy_unit(std::integral_constant<int, UNITS - EARLY + n / APART>{}, slot ^ 1, late);
            if constexpr (n == APART * EARLY + 1) {
                copy_step(slot ^ 1, late);
                if (late) after_copies();
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (n >= LAG) add((n - LAG) / TM, (n - LAG) % TM, ring[(n - LAG) % RING], sa[(n - LAG) % TM]);
            else add(TN - 1, TM - LAG + n, ring[(COUNT - LAG + n) % RING], sa_last[n]);        // of the slab before
            if constexpr (j == LAG - 1) {                      // (the tile before has had its multiply-adds)
                if constexpr (i < TN - 1) { if constexpr (PER_ROW) read_row_step(at, i + 1, (i + 1) % 2); }
                else read_row_step(next, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (n == FIRST - 1) {
                // This wavefront has read all of the slab's fragments and its copies of the next one have landed; behind the barrier that holds for every wavefront, so
                // the next slab may be read and another one take this one's place.
                if (stores == 16) wait_copies<16>();
                else if (stores == 32) wait_copies<32>();
                else wait_copies<0>();
                stores = 0;
                if (ragged_copies) clear_ragged(slot ^ 1);
                before_copies();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
        }, std::make_integer_sequence<int, COUNT>{});
        slot ^= 1;
        late = lanes;
        if (kt < k_last) { ++kt; continue; }

        // ---- the end of a tile
#pragma unroll
        for (int k = 0; k < LAG; ++k) {
            add(TN - 1, TM - LAG + k, ring[(COUNT - LAG + k) % RING], sa[TM - LAG + k]);
            ring[(COUNT - LAG + k) % RING] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int k = 0; k < LAG; ++k) sa[TM - LAG + k] = 0.0f;                // (what the next slab adds for this one: nothing, whatever the step sizes were)
        if constexpr (PER_ROW) sb[1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        // the copies that are still to go out do so in front of the stores: memory operations end in order, so the next barrier need not wait for the stores
        in_order([&](auto unit) __attribute__((always_inline)) { copy_unit(std::integral_constant<int, decltype(unit)::value + UNITS - EARLY>{}, slot ^ 1, lanes); }, std::make_integer_sequence<int, EARLY>{});
        copy_step(slot ^ 1, lanes);
        after_copies();
        late = 0;
        const Tile t = tile_at(t_now);
        void* out = g.splits > 1 ? static_cast<void*>(g.partial + (int64_t)t.split * g.batch * g.M * g.N) : g.y;
        const bool bf16 = g.splits == 1 && g.y_bf16;
        const int64_t n_first = t.n0 + wn * 16 * TN, m_first = t.m0 + wm * 16 * TM;
        const int l = lane_here(), q = l >> 4, j16 = l & 15;
        if (g.M - t.m0 >= BM && g.N - t.n0 >= BN) {
            // Whole tiles leave in whole 128-byte lines: of two units of 16 bytes that a lane has of a line, it trades one with the lane of the next token, so that a store of the
            // wavefront holds eight lines.
            const bool second = l & 1;
            auto put = [&](u32x4 u0, u32x4 u1, int64_t at, int64_t apart) {        // at: of the even token, this lane's unit; apart: from one token to the next
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t given = second ? u0[e] : u1[e], taken = (uint32_t)__builtin_amdgcn_mov_dpp((int)given, 0xB1, 0xF, 0xF, true);      // quad_perm 1, 0, 3, 2
                    u0[e] = second ? taken : u0[e];
                    u1[e] = second ? u1[e] : taken;
                }
                uint8_t* p = static_cast<uint8_t*>(out) + at;
                *reinterpret_cast<u32x4_any*>(p) = u0;
                *reinterpret_cast<u32x4_any*>(p + apart) = u1;
            };
            stores = bf16 ? 16 : 32;
            const int64_t size = bf16 ? 2 : 4, apart = g.N * size;
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int64_t row = ((t.bidx * g.M + m_first + 16 * j + (j16 & ~1)) * g.N + n_first) * size;
                if (bf16) {
#pragma unroll
                    for (int i = 0; i < TN; i += 4) {
                        u32x4 u[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const v4f &x = acc[i + 2 * k][j], &y = acc[i + 2 * k + 1][j];
                            u[k] = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
                        }
                        put(u[0], u[1], row + (16 * i + (second ? 32 : 0) + 8 * q) * 2, apart);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < TN; i += 2)
                        put(__builtin_bit_cast(u32x4, acc[i][j]), __builtin_bit_cast(u32x4, acc[i + 1][j]), row + (16 * i + 8 * q + (second ? 4 : 0)) * 4, apart);
                }
            }
        } else {
            stores = 0;
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int i = 0; i < TN; i += 2) {
                    const int64_t m = m_first + 16 * j + j16, n = n_first + 16 * i + 8 * q;
                    if (m >= g.M || n >= g.N) continue;
                    const float v[8] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3], acc[i + 1][j][0], acc[i + 1][j][1], acc[i + 1][j][2], acc[i + 1][j][3]};
                    store8(out, bf16, (t.bidx * g.M + m) * g.N + n, v, g.N - n);
                }
        }
        t_now += stride;
        if (t_now >= run_end) break;
        clear();
        const Tile u = tile_at(t_now);
        kt = u.begin; k_last = u.end - 1;
    }
}

// Few tokens (at most 16 TB): the time is the weights' on their way from memory.  A workgroup of W wavefronts takes 16 rows of the weights, the wavefronts share the
// contraction slab by slab in turn, fragments go straight into registers up to AHEAD slabs ahead, and the wavefronts' sums are added in their order in LDS.
template <int FA, int FB, int TB, int W, bool PER_ROW>
__global__ void __launch_bounds__(64 * W)
block_few(BlockGemmArgs g)
{
    constexpr int AHEAD = TB == 1 ? 4 : TB == 2 ? 3 : 2;
    __shared__ v4f sums[W][TB][64];
    const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t groups = (uint32_t)g.tiles_n;
    const int64_t bidx = __builtin_amdgcn_readfirstlane((int)(blockIdx.x / groups));
    const int64_t n0 = 16 * (int64_t)(blockIdx.x - (uint32_t)bidx * groups);
    const int rowbytes = (int)g.K, slabs = (rowbytes + kBlock - 1) / kBlock;
    const float* da = g.da + bidx * slabs * g.a_blocks;
    const float* db = g.db + bidx * slabs * g.b_blocks;
    const uint8_t* rows[1 + TB];
    int64_t a_block[TB], b_block[4];
    rows[0] = g.b + (bidx * g.N + min(n0 + j, g.N - 1)) * g.K + 16 * q;
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        const int64_t m = min((int64_t)(16 * t + j), g.M - 1);
        rows[1 + t] = g.a + (bidx * g.M + m) * g.K + 16 * q;
        a_block[t] = m >> g.a_shift;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) b_block[v] = min(n0 + (PER_ROW ? 4 * q + v : 0), g.N - 1) >> g.b_shift;
    v4f acc[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    struct Slab { v4i f[1 + TB][2]; float sa[TB], sb[PER_ROW ? 4 : 1]; };
    Slab ahead[AHEAD];
    auto load = [&](int slab, Slab& s) {
        const int k0 = slab * kBlock;
#pragma unroll
        for (int r = 0; r < 1 + TB; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {                      // (bytes past the end of the rows: zeros)
                s.f[r][h] = v4i{0, 0, 0, 0};
                if (k0 + 64 * h + 16 * q < rowbytes) s.f[r][h] = *reinterpret_cast<const v4i*>(rows[r] + k0 + 64 * h);
            }
#pragma unroll
        for (int t = 0; t < TB; ++t) s.sa[t] = da[slab * g.a_blocks + a_block[t]];
#pragma unroll
        for (int v = 0; v < (PER_ROW ? 4 : 1); ++v) s.sb[v] = db[slab * g.b_blocks + b_block[v]];
    };
    auto multiply = [&](const Slab& s) {
        const v8i fw = {s.f[0][0][0], s.f[0][0][1], s.f[0][0][2], s.f[0][0][3], s.f[0][1][0], s.f[0][1][1], s.f[0][1][2], s.f[0][1][3]};
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            const v4i &x0 = s.f[1 + t][0], &x1 = s.f[1 + t][1];
            const v4f sum = block_sums<FA, FB>(fw, v8i{x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]});
            const float sa = PER_ROW ? s.sa[t] : s.sa[t] * s.sb[0];
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[t][v] = fmaf(PER_ROW ? sum[v] * s.sb[PER_ROW ? v : 0] : sum[v], sa, acc[t][v]);
        }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * W < slabs) load(wave + i * W, ahead[i]);
    for (int k = wave; k < slabs; k += AHEAD * W) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k + i * W < slabs) {
                multiply(ahead[i]);
                if (k + (i + AHEAD) * W < slabs) load(k + (i + AHEAD) * W, ahead[i]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < TB; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < TB; t += W) {
        const int64_t m = 16 * t + j;
        v4f sum = sums[0][t][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) sum += sums[w][t][lane];
        if (m >= g.M) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int64_t n = n0 + 4 * q + v, at = (bidx * g.M + m) * g.N + n;
            if (n >= g.N) continue;
            if (g.y_bf16) static_cast<__bf16*>(g.y)[at] = (__bf16)sum[v];
            else static_cast<float*>(g.y)[at] = sum[v];
        }
    }
}

// Sums of the parts of a split contraction, in ascending order: four neighbouring outputs a thread, four parts on their way at a time.
__global__ void __launch_bounds__(256) block_reduce(BlockGemmArgs g)
{
    const int64_t total = g.batch * g.M * g.N, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= total) return;
    const int left = (int)min((int64_t)4, total - at);
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < g.splits; p += 4) {
        u32x4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            w[k] = u32x4{0u, 0u, 0u, 0u};
            if (p + k < g.splits) {
                const float* part = g.partial + (p + k) * total + at;
                w[k] = left == 4 ? *reinterpret_cast<const u32x4_any*>(part) : Vec<float>::partial_load(part, left);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (p + k < g.splits) s = p + k == 0 ? __builtin_bit_cast(v4f, w[k]) : s + __builtin_bit_cast(v4f, w[k]);
    }
    if (g.y_bf16) {
        const u32x4 w = {pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3]), 0u, 0u};
        uint16_t* p = static_cast<uint16_t*>(g.y) + at;
        if (left == 4) *reinterpret_cast<u32x2_byte*>(p) = u32x2{w[0], w[1]};
        else store_bytes<8>(reinterpret_cast<uint8_t*>(p), w, left * 2);
    } else {
        float* p = static_cast<float*>(g.y) + at;
        if (left == 4) *reinterpret_cast<u32x4_any*>(p) = __builtin_bit_cast(u32x4, s);
        else store_bytes<16>(reinterpret_cast<uint8_t*>(p), __builtin_bit_cast(u32x4, s), left * 4);
    }
}

// ---- host
inline bool ensure_lds(std::atomic<uint64_t>& done, const void* kern, int bytes)      // once per kernel and device
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0;
    if (bit && (done.load(std::memory_order_acquire) & bit)) return true;
    if (hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return false;
    if (bit) done.fetch_or(bit, std::memory_order_release);
    return true;
}
qmm_status launch_reduce(const BlockGemmArgs& g, hipStream_t s)
{
    if (hipGetLastError() != hipSuccess) return QMM_ERR_LAUNCH;
    block_reduce<<<(unsigned)((g.batch * g.M * g.N + 1023) / 1024), 256, 0, s>>>(g);
    return launch_status();
}
template <int FA, int FB, int WN, int WM, int TN, int TM, int SLOTS, bool PER_ROW> qmm_status launch_tiles(BlockGemmArgs& g, hipStream_t s)
{
    constexpr int BN = 16 * WN * TN, BM = 16 * WM * TM, LDS_BYTES = SLOTS * (BN + BM) * (kBlock + 4);
    static_assert(LDS_BYTES <= 160 * 1024 && 64 * WN * WM == kTileThreads, "LDS of a CU, threads of a workgroup");
    const int64_t tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
    if (!launches((double)tm * tn * g.batch * g.splits, kTileThreads)) return QMM_ERR_UNSUPPORTED;      // (no contraction: every other plan fits)
    g.tiles_m = (int)tm; g.tiles_n = (int)tn;
    auto kern = block_gemm<FA, FB, WN, WM, TN, TM, SLOTS, PER_ROW>;
    static std::atomic<uint64_t> done{0};
    if (!ensure_lds(done, reinterpret_cast<const void*>(kern), LDS_BYTES)) return QMM_ERR_LAUNCH;
    kern<<<(unsigned)(tm * tn * g.batch * g.splits), 64 * WN * WM, LDS_BYTES, s>>>(g);
    return g.splits > 1 ? launch_reduce(g, s) : launch_status();
}
constexpr int kLargeGrid = 256;                // one workgroup of the large tile a CU
template <int FA, int FB, bool PER_ROW> qmm_status launch_large(BlockGemmArgs& g, hipStream_t s)
{
    constexpr int LDS_BYTES = 2 * 512 * (kBlock + 4);
    const int64_t tm = (g.M + 255) / 256, tn = (g.N + 255) / 256;
    if ((double)tm * tn * g.batch * g.splits > 0x7FFFFFFF) return QMM_ERR_UNSUPPORTED;      // (in binary64: the product may pass 64 bits)
    g.tiles_m = (int)tm; g.tiles_n = (int)tn;
    auto kern = block_gemm_large<FA, FB, PER_ROW>;
    static std::atomic<uint64_t> done{0};
    if (!ensure_lds(done, reinterpret_cast<const void*>(kern), LDS_BYTES)) return QMM_ERR_LAUNCH;
    kern<<<(unsigned)std::min<int64_t>(tm * tn * g.batch * g.splits, kLargeGrid), 512, LDS_BYTES, s>>>(g);
    return g.splits > 1 ? launch_reduce(g, s) : launch_status();
}
template <int FA, int FB, bool PER_ROW> qmm_status launch_form(BlockGemmArgs& g, int tile, hipStream_t s)
{
    if (tile == 256) return launch_large<FA, FB, PER_ROW>(g, s);
    if (tile == 128) return launch_tiles<FA, FB, 2, 2, 4, 4, 2, PER_ROW>(g, s);
    if (tile == 64) return launch_tiles<FA, FB, 2, 2, 2, 2, 4, PER_ROW>(g, s);
    const int64_t tn = (g.N + 15) / 16;
    if (!launches((double)tn * g.batch, kFewThreads)) return QMM_ERR_UNSUPPORTED;
    g.tiles_n = (int)tn;
    const unsigned grid = (unsigned)(tn * g.batch);
    if (g.M <= 16) block_few<FA, FB, 1, kFewThreads / 64, PER_ROW><<<grid, kFewThreads, 0, s>>>(g);
    else if (g.M <= 32) block_few<FA, FB, 2, kFewThreads / 64, PER_ROW><<<grid, kFewThreads, 0, s>>>(g);
    else block_few<FA, FB, 4, kFewThreads / 64, PER_ROW><<<grid, kFewThreads, 0, s>>>(g);
    return launch_status();
}
template <int FA, int FB> qmm_status launch_formats(BlockGemmArgs& g, bool per_row, int tile, hipStream_t s)
{
    return per_row ? launch_form<FA, FB, true>(g, tile, s) : launch_form<FA, FB, false>(g, tile, s);
}

// (the kernels keep 32-bit byte offsets within a tile's rows)
bool beyond(int64_t M, int64_t N, int64_t K) { return K > (int64_t(1) << 22) || M > 0x7FFFFFFF || N > 0x7FFFFFFF; }
qmm_status check_block_operand(const qmm_block_operand* o)
{
    if (!o) return QMM_ERR_NULL;
    if (o->format == QMM_FMT_INT8 || o->format == QMM_FMT_BF16) return QMM_ERR_UNSUPPORTED;
    if (o->format != QMM_FMT_E4M3 && o->format != QMM_FMT_E5M2) return QMM_ERR_ENUM;
    if (o->block_rows != 1 && o->block_rows != kBlock) return QMM_ERR_ENUM;
    return QMM_OK;
}

}  // namespace
}  // namespace qmm

using namespace qmm;

extern "C" size_t qmm_gemm_blocks_workspace_size(int64_t batch, int64_t M, int64_t N, int64_t K)
{
    if (batch <= 0 || M <= 0 || N <= 0 || K <= 0 || beyond(M, N, K)) return 0;
    const int splits = plan_of(M, N, K, batch).splits;
    return splits > 1 ? (size_t)splits * (size_t)batch * (size_t)M * (size_t)N * 4u : 0;
}

extern "C" qmm_status qmm_gemm_blocks(const qmm_block_operand* a, const qmm_block_operand* b, int64_t batch, int64_t M, int64_t N, int64_t K,
                                      void* y, qmm_dtype y_dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    qmm_status st = check_block_operand(a);
    if (st != QMM_OK) return st;
    st = check_block_operand(b);
    if (st != QMM_OK) return st;
    if (y_dtype != QMM_DT_BF16 && y_dtype != QMM_DT_F32) return QMM_ERR_ENUM;
    if (batch < 0 || M < 0 || N < 0 || K < 0) return QMM_ERR_SHAPE;
    if (K % 16 != 0) return QMM_ERR_ALIGN;
    if (beyond(M, N, K)) return QMM_ERR_UNSUPPORTED;
    if (batch == 0 || M == 0 || N == 0) return QMM_OK;
    if (!y || (K > 0 && (!a->data || !b->data || !a->delta || !b->delta))) return QMM_ERR_NULL;
    if (!aligned16(a->data) || !aligned16(b->data) || !aligned16(y)) return QMM_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(a->delta) | reinterpret_cast<uintptr_t>(b->delta)) & 3u) return QMM_ERR_ALIGN;
    BlockGemmArgs g{};
    g.a = static_cast<const uint8_t*>(a->data); g.b = static_cast<const uint8_t*>(b->data);
    g.da = a->delta; g.db = b->delta;
    g.a_shift = a->block_rows == 1 ? 0 : 7; g.b_shift = b->block_rows == 1 ? 0 : 7;
    g.a_blocks = (M + a->block_rows - 1) / a->block_rows; g.b_blocks = (N + b->block_rows - 1) / b->block_rows;
    g.M = M; g.N = N; g.K = K; g.batch = batch; g.y = y; g.y_bf16 = y_dtype == QMM_DT_BF16;
    const Plan plan = plan_of(M, N, K, batch);
    g.splits = plan.splits;
    if (g.splits > 1) {
        if (!workspace || workspace_bytes < qmm_gemm_blocks_workspace_size(batch, M, N, K)) return QMM_ERR_WORKSPACE;
        if (!aligned16(workspace)) return QMM_ERR_ALIGN;
        g.partial = static_cast<float*>(workspace);
    }
    hipStream_t s = as_stream(stream);
    const bool per_row = g.b_shift == 0;
    if (a->format == QMM_FMT_E4M3) return b->format == QMM_FMT_E4M3 ? launch_formats<QMM_FMT_E4M3, QMM_FMT_E4M3>(g, per_row, plan.tile, s) : launch_formats<QMM_FMT_E4M3, QMM_FMT_E5M2>(g, per_row, plan.tile, s);
    return b->format == QMM_FMT_E4M3 ? launch_formats<QMM_FMT_E5M2, QMM_FMT_E4M3>(g, per_row, plan.tile, s) : launch_formats<QMM_FMT_E5M2, QMM_FMT_E5M2>(g, per_row, plan.tile, s);
}
