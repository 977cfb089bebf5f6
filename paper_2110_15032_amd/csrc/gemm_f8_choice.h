// Which kernel a product of 8-bit tensors runs on.  Host only, and a function of its arguments alone.
#pragma once
#include <algorithm>
#include <cmath>

#include "sbp_internal.h"

namespace sbp {

struct F8Choice {
    int mb, nb;     // 16s of rows and columns: up to 4 tiles of waves, 8 and 16 the tiles through LDS
    bool aligned;   // rows of both operands by 16 bytes, of their scales by 4
};

// The variant whose time the sizes give as the least.  Every one is its rounds over the compute units (`cu`) times a workgroup's time, which goes with the
// blocks of 128 of the reduction and, for tiles of waves, with the operand rows that they bring: 16 (MB + NB) of 128 bytes a block.  The coefficients are
// fits, us, to what the variants measured; where memory or the launch is the bound they are too low for all of them alike.
// us, M x K x N (devices), bf16 results, (MB, NB) of waves | tiles of 128 | of 256:
//   32 x 4096 x 16384 (8):  (2,2) 12.8  (2,4) 13.1  (4,4) 14.2 | 27.2 | 47.6       1024 cubed:  (2,2) 7.6   (4,4) 6.8  | 10.3 | 18.6
//   100 x 16384 x 1000:     (2,1) 12.7  (2,2) 16.0  (4,4) 34.9 | 92.0 | 173        2048 cubed:  (2,2) 33.2  (4,4) 29.9 | 17.3 | 29.9
//   500 x 8192 x 1000 (2):  (2,4) 13.8  (2,2) 16.2  (4,4) 20.1 | 48.9 | 91.0       4096 cubed:  (4,4) 173              | 72.8 | 58.7
//   256 x 4096 x 4096:      (2,4) 15.7  (2,2) 16.4  (4,4) 13.0 | 27.0 | 49.9       64 x 2048 x 65536:  (4,4) 43.9      | 32.2 | 39.3
//   fp32 results, 1024 cubed: (2,2) 8.6  (4,4) 7.5 | 16.2; 2048 cubed: (2,2) 37.7  (4,4) 34.9 | 28.2 | 60.8; 4096 cubed 140 | 112
// and with rows at odd pitches, through registers:
//   300 x 8191 x 513: (2,2) 66.1  (4,4) 129 | 105; 1001 cubed: (2,2) 22.0  (4,4) 13.0 | 20.9; 1111 x 1531 x 1777: (2,4) 57.2  (4,4) 39.3 | 28.8
inline F8Choice choose_f8_tile(const GemmF8Plan& plan, int64_t cu) {
    const bool f32 = plan.out_dtype == SBP_F32;
    int max_m = 0, max_n = 0, max_k = 0;
    bool aligned = true, empty = false;   // empty: a shard without anything to sum: its results are zeros that the tiles of waves write
    for (int g = 0; g < plan.groups; ++g) {
        const GemmF8Shard& s = plan.s[g];
        max_m = std::max(max_m, s.m);
        max_n = std::max(max_n, s.n);
        max_k = std::max(max_k, s.kk);
        empty = empty || s.kk == 0;
        if (s.lda % 16 || s.ldb % 16 || s.ldas % 4 || s.ldbs % 4) aligned = false;
    }
    const int64_t blocks = tiles_along(max_k, F8_BLOCK);
    auto tiles = [&](int rows, int columns) { return (int64_t)tiles_along(max_m, rows) * tiles_along(max_n, columns) * plan.groups; };
    auto rounds = [](int64_t of, int64_t at_once) { return (double)((of + at_once - 1) / at_once); };
    F8Choice best{1, 1, aligned};
    double least = INFINITY;
    auto offer = [&](int mb, int nb, double us) {
        if (us < least) best = F8Choice{mb, nb, aligned}, least = us;
    };
    const double of_rows = !aligned ? 0.2 : f32 ? 0.043 : 0.035;
    for (int mb = 1; mb <= 4; mb *= 2)
        for (int nb = 1; nb <= 4; nb *= 2) offer(mb, nb, rounds(tiles(16 * mb, 16 * nb), cu) * ((mb + nb) * blocks * of_rows + 3.0));
    if (empty) return best;
    const int64_t n128 = tiles(128, 128);   // two share a compute unit where there are more than units
    if (n128 <= cu) offer(8, 8, blocks * (!aligned ? 1.9 : f32 ? 1.4 : 0.72) + 3.0);
    else offer(8, 8, rounds(n128, 2 * cu) * blocks * (!aligned ? 2.2 : f32 ? 1.95 : 1.1) + 3.0);
    if (aligned) offer(16, 16, rounds(tiles(256, 256), cu) * blocks * (f32 ? 3.3 : 1.75) + 3.0);
    return best;
}

}  // namespace sbp
