// Which kernel a product with step sizes per block of 128 takes.  Host code without the HIP headers, so that a test can compile it and hold the sizes that
// are meant for one of the kernels to it.
#pragma once
#include <stdint.h>
#include <initializer_list>

namespace qmm {
namespace {

constexpr int kBlock = 128;                    // elements along the contraction that share a step size

// Which kernel, and in how many parts of K: the least of what the forms are reckoned to take, in microseconds.  A tile's step (a slab of 128) takes, with one / two workgroups a CU, 1.4 / -
// (1.97 where all CUs work), 0.76 / 1.09 and 0.33 / 0.48 for edges of 256, 128 and 64, and a tile or a launch what is added below; with few tokens a wavefront's slab takes 1.3 + 0.5 for each 16
// tokens and workgroup a CU; a split's second pass takes 3 and its memory traffic at 8.9 TB/s (much of it is still in the memory-side cache).  Fitted to 32 sizes, each by all forms and splits: the form
// taken is 0.1 % slower than the fastest in the mean.  (E4M3, us by 256 / 128 / 64, unsplit, and the best split: 4096 x 4096 x 1024 23 / 27 / -; 2048 x 4096 x 1024 19 / 16 / 25; 128 x 4096 x 4096
// 49 / 25 / 14, 13 by 64 in two; 5120 x 4096 x 2048 58 / 53; 1024 x 1024 x 16384 220 / 94 / 50, 36 by 128 in eight; 4096 x 1024 x 16384 229 / 116 / 130, 94 by 256 in four, 95 by 128 in two; few
// tokens, 16 x 8192 x 4096 11.5, by 64 in two 12, 64 of them 24 / 12.6.)
constexpr int kFewTokens = 64;
// A form that gives each tile a workgroup is offered where a launch takes as many: less than 2^32 threads.  (The 256 x 256 form's workgroups go from tile to tile.)
constexpr int kFewThreads = 512, kTileThreads = 256;
inline bool launches(double groups, int threads) { return groups * threads < 4294967296.0; }
struct Plan { int tile; int splits; };         // tile: 0 few tokens, else its edge
Plan plan_of(int64_t M, int64_t N, int64_t K, int64_t batch)
{
    if (K == 0) return Plan{64, 1};
    const double slabs = (double)((K + kBlock - 1) / kBlock), out = 4.0 * (double)M * (double)N * (double)batch;
    auto up = [](double x) { return (double)(int64_t)(x + 0.999999); };
    Plan best{256, 1};
    double least = 1e300;
    auto offer = [&](int tile, int splits, double us) {
        if (us < least) { least = us; best = Plan{tile, splits}; }
    };
    if (M <= kFewTokens) {
        const double groups = (double)((N + 15) / 16) * (double)batch, blocks = M <= 16 ? 1.0 : M <= 32 ? 2.0 : 4.0;
        if (launches(groups, kFewThreads)) offer(0, 1, 1.4 + up(groups / 512.0) * up(slabs / 8.0) * (1.3 + 0.5 * blocks * (groups > 256.0 ? 2.0 : 1.0)));
    }
    for (int tile : {256, 128, 64}) {
        const double tiles = (double)((M + tile - 1) / tile) * (double)((N + tile - 1) / tile) * (double)batch;
        for (int splits : {1, 2, 4, 8, 16}) {
            if (splits > 1 && (slabs < 4.0 * splits || out * splits > 268435456.0)) break;
            const double groups = tiles * splits, steps = up(slabs / splits);
            if (tile != 256 && !launches(groups, kTileThreads)) break;
            double us;
            if (tile == 256) us = 2.7 + up(groups / 256.0) * (steps * (groups >= 192.0 ? 1.97 : 1.4) + 3.8);
            else if (tile == 128) us = 5.1 + (groups <= 256.0 ? steps * 0.76 : up(groups / 512.0) * (steps * 1.09 + 2.4));
            else us = 3.6 + (groups <= 256.0 ? steps * 0.33 : up(groups / 512.0) * (steps * 0.48 + 0.9));
            if (splits > 1) us += 3.0 + out * (2.0 * splits + 1.0) / 8.9e6;
            offer(tile, splits, us);
        }
    }
    return best;
}

}  // namespace
}  // namespace qmm
