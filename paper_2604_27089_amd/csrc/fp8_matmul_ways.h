// Which of its kernels a block-scaled product goes to: a host rule on the extents.
//
// Each way's time is estimated from its extents, and the least is taken.  A pipe workgroup takes `fixed` us, and per tile `tile` us and
// `step` us for each block; one of the few-row kernel the same with its rounds over b's rows in place of the tiles, and with `rows` us
// more for each block as far as its rows of a are there to be copied.  All run one workgroup per compute unit.  No estimate is below the
// time of the bytes at 5.6 TB/s and 2.5 us (fitted; single shapes come a little under it: 1 x 57344 x 8192 82 us for 86); where that takes longest
// the first way does, which copies least at a time.
// The constants are fitted to the times of every way over 665 shapes of 1 to 16384 rows with the layer widths of Llama models (b from
// memory, in a graph, random bytes); what the rule takes is 0.8 % slower than the best way in the mean.  Measured then, us, tiles of 256 x 256
// / 256 x 128 / 128 x 128 / few rows with 64 x 32 at a time: 16384 x 28672 x 4096 1336 / 1597 / 2070 / -, 4096 x 6144 x 4096 97 / 89 / 115 / -, 1024 x
// 4096 x 4096 46 / 29 / 22 / 50, 128 x 4096 x 4096 46 / 25 / 21 / 12; one row, N = 4096, K = 14336: 128 x 128 57, few rows 14.  Few rows 16 x
// 16 / 16 x 32 / 32 x 32 / 64 x 32 / 64 x 48 / 64 x 64 at a time: 16 x 4096 x 14336 14.7 / 18.3 / 22 / 29 / - / -, 16 x 57344 x 8192 93 / 90 / 92
// / 101 / - / -, 128 x 6144 x 4096 - / - / - / 18 / 14 / 16, 128 x 8192 x 28672 - / - / - / 101 / 108 / 79.
#pragma once
#include <stdint.h>

namespace sp {
namespace ways {

struct Cost {
    double fixed, step, rows, tile;
};
constexpr int kFew = 6;  // ways
constexpr Cost kFewCost[kFew] = {{3.8, 0.534, 0.402, 0.475}, {4.47, 0.939, 0.559, 0.}, {2.3, 0.8, 0., 1.24}, {1.77, 0.867, 0.083, 3.44},
                                 {1.33, 1.114, 0., 5.08}, {1.88, 1.387, 0., 4.64}};
constexpr int kFewMB[kFew] = {1, 1, 2, 4, 4, 4}, kFewNB[kFew] = {1, 2, 2, 2, 3, 4}, kFewWaves[kFew] = {8, 8, 4, 4, 4, 4}, kFewStages[kFew] = {3, 2, 3, 2, 2, 2};
constexpr Cost kPipeCost[3] = {{2.11, 0.714, 0., 3.06}, {5.24, 0.951, 0., 2.55}, {5.39, 1.581, 0., 4.17}};
constexpr int kPipeGM[3] = {1, 2, 2}, kPipeGN[3] = {1, 1, 2}, kPipeStages[3] = {4, 3, 2};
constexpr Cost kF32Cost = {0.8, 1.63, 0., 5.6};  // per 512 tiles of 128 x 128
constexpr double kAddFixed = 4.5, kAddRate = 5e6, kAddGain = 0.915;  // us; bytes a us, written and read; not for less than this gain
constexpr int64_t kUnits = 256;  // compute units

inline int64_t parts(int64_t n, int64_t of) { return (n + of - 1) / of; }

struct FewGrid {
    int64_t x, y, groups;
};
inline FewGrid few_grid(int way, int64_t M, int64_t N) {
    const int64_t x = parts(M, 16 * kFewMB[way]), all = parts(N, 16), room = kUnits / x > 1 ? kUnits / x : 1;
    const int64_t most = parts(all, kFewNB[way]), groups = parts(all, most < room ? most : room);
    return FewGrid{x, parts(all, groups), groups};
}

// 0 .. 5: few rows, 6 .. 8: pipe, 9: fp32 tiles
inline int which_way(int64_t M, int64_t N, int64_t K, bool f32, double* estimate = nullptr) {
    if (K == 0) return 0;  // the only kernel that has nothing to copy then
    const double blocks = (double)(K / 128), read = (double)(M * K + N * K + M * N * (f32 ? 4 : 2)) / 5.6e6 + 2.5;
    int best = 0;
    double least = 0.;
    auto consider = [&](int way, const Cost& c, double tiles, double steps, double there) {
        const double us = c.fixed + tiles * ((c.step + c.rows * there) * steps + c.tile), time = us > read ? us : read;
        if (way == 0 || time < least) { best = way; least = time; }
    };
    for (int w = 0; w < kFew; ++w) {
        const FewGrid g = few_grid(w, M, N);
        consider(w, kFewCost[w], (double)(parts(g.x * g.y, kUnits) * parts(g.groups, kFewNB[w])), (double)parts(K / 128, kFewWaves[w]),
                 M < 16 * kFewMB[w] ? (double)M / (16 * kFewMB[w]) : 1.);
    }
    if (f32) {
        const double rounds = (double)(parts(M, 128) * parts(N, 128)) / (2. * kUnits);
        consider(kFew + 3, kF32Cost, rounds > 1. ? rounds : 1., blocks, 0.);
    } else {
        for (int w = 0; w < 3; ++w)
            consider(kFew + w, kPipeCost[w], (double)parts(parts(M, 128 * kPipeGM[w]) * parts(N, 128 * kPipeGN[w]), kUnits), 2. * (double)parts(K / 128, 2), 0.);
    }
    if (estimate) *estimate = least;
    return best;
}

// For results in bf16: the contraction of tiles of 128 x 128 shared out among `splits` workgroups, `per` blocks each, and a second
// launch that adds their sums; splits 1: not worth it.  Whole / shared out, us: 48 x 8192 x 28672 64 / 52, 128 x 8192 x 28672 85 / 64, 128 x
// 4096 x 14336 29 / 24, 256 x 4096 x 14336 40 / 31, 256 x 8192 x 28672 144 / 93, 384 x 4096 x 14336 69 / 44; 48 x 2048 x 8192 12 / 14.
struct Split {
    int64_t splits, per;
};
inline Split which_split(int64_t M, int64_t N, int64_t K) {
    Split best{1, K / 128};
    if (M == 0 || N == 0 || K < 1024) return best;
    double least;
    which_way(M, N, K, false, &least);
    least *= kAddGain;
    const int64_t tiles = parts(M, 128) * parts(N, 128), blocks = K / 128;
    if (tiles > kUnits) return best;
    for (int64_t want = 2; want <= 16; ++want) {
        const int64_t per = parts(blocks, want), splits = parts(blocks, per);
        const double us = kPipeCost[0].fixed + (double)parts(tiles * splits, kUnits) * (kPipeCost[0].step * 2. * (double)parts(per, 2) + kPipeCost[0].tile) +
                          kAddFixed + (double)(splits * M * N) * 8. / kAddRate;
        if (us < least) { best = Split{splits, per}; least = us; }
    }
    return best;
}

}  // namespace ways
}  // namespace sp
