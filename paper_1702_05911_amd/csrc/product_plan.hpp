// Which kernel multiplies matrices in 8-bit blocks, by the sizes and the kind of result (block_product.hip; host code only).
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace pqt {
namespace {

constexpr int kFewRows = 16;               // of A: the kernel that has no tiles
struct Plan {
    int tile;                              // 256, 128, 64, or 16: few
    int tiles_m, tiles_n, splits, per_split;
};
constexpr int64_t kMaxTiles = 0xffffff;    // (256 threads each, fewer than 2^32 in all)
constexpr int kUnits = 256;                // compute units
constexpr int64_t kManyColumns = 32768;    // of a result of few rows: two workgroups a compute unit with 64 columns each

// The time of a product by one of the kernels, as their steps measure: a step of a workgroup that has its compute unit to itself, what one
// more workgroup on it adds, how many fit, and what a call costs before and after (us).
//   wide   2.9 PFLOP/s where there are many tiles; one tile alone takes 14 us before and after its steps
//   bf16 results   128: 8191 x 960 x 2000 27.7 (64: 38.9, wide 31.2), 2048^3 18.2 (21.9, 28.9);  64: 1000^3 6.2 (128: 10.2), 10000 x 128 x 1000 7.8 (10.4)
//   fp32 results (and f16, by the same instructions)   128: 8191 x 960 x 2000 39.6 (64: 50.9);  64: 1000^3 7.9 (13.4)
//   shared out     960 x 2000 x 8191 by four 35.4 (57.5 whole, 64: 40.8), fp32 48.0 (83.8, 59.2);  512 x 512 x 8192 on 64 by eight 14.3 (30.6)
struct Cost { double step, more, fit, around; };
double time_of(const Cost& c, double tiles, int steps, int splits, double results) {
    const double on_one = std::max(1.0, std::ceil(tiles * splits / kUnits));
    const double step = on_one <= c.fit ? c.step + (on_one - 1) * c.more : (c.step + (c.fit - 1) * c.more) * on_one / c.fit;
    return steps * step + c.around + (splits > 1 ? 3.0 + splits * results * 1e-6 : 0.0);
}

Plan plan_of(int64_t m, int64_t n, int kb, bool exact) {
    Plan p{};
    p.splits = 1;
    p.per_split = kb;
    if (m <= kFewRows) {
        p.tile = 16;
        return p;
    }
    double best = 0.0;
    for (int tile : {64, 128, 256}) {
        if (tile == 256 && exact) continue;
        const Cost c = tile == 256 ? Cost{1.25, 0.0, 1.0, 13.0} : tile == 128 ? (exact ? Cost{1.4, 0.45, 2.0, 5.0} : Cost{0.95, 0.27, 2.0, 5.0})
                                                                              : (exact ? Cost{0.5, 0.3, 4.0, 3.0} : Cost{0.36, 0.25, 4.0, 3.0});
        const int64_t tm = (m + tile - 1) / tile, tn = (n + tile - 1) / tile;
        for (int splits = 1; splits <= 16 && (splits == 1 || (tile < 256 && kb >= 4 * splits)); splits *= 2) {
            const int per = splits == 1 ? kb : ((kb + splits - 1) / splits + 1) / 2 * 2, real = (kb + per - 1) / per;
            const double t = time_of(c, (double)tm * (double)tn, per, real, (double)m * (double)n);
            if (p.tile == 0 || t < best) {
                best = t;
                p.tile = tile;
                p.tiles_m = (int)std::min(tm, kMaxTiles);
                p.tiles_n = (int)std::min(tn, kMaxTiles);
                p.splits = real;
                p.per_split = per;
            }
        }
    }
    return p;
}

}  // namespace
}  // namespace pqt
