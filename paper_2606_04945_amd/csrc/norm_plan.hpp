// Launch plan of the norms, without HIP: waves that share a row, and vectors of 8
// entries that a lane holds.
//
// Rows of up to 512 entries are one wave's (no exchange between waves).  Wider ones: few
// rows want the shortest chain, a vector a lane; many want the fewest exchanges and waves, two
// vectors a lane.  Measured (us; a: stream and y in, stream and row out; q: 4-bit codes in place of the row), one
// vector a lane against two:
//   K = 4096: 1 row a 2.27 / 2.47, 16 rows q 3.51 / 4.04, 256 rows q 4.63 / 5.25; K = 3584: 1024 rows q 9.7 / 9.2,
//             2048 rows q 15.2 / 14.2; 16384 x 4096 a 94 / 92, q 93 / 81
//   K = 2048: 1 row q 2.83 / 3.37; 16384 rows a 46.8 / 46.8, q 47 / 44
//   Borders: K = 2048, 700 rows q 5.50 / 5.85, 1024 6.56 / 6.46, 2048 10.9 / 9.8; K = 4096, 512 rows q 6.61 / 6.70,
//             700 8.48 / 7.88 (w, see below: 1024 x 2048 11.4 / 10.7, 512 x 4096 10.7 / 10.5)
//   16384 x 512: a wave a row a 14.9, two 16.4, four 25; 16384 x 1024: two waves, one vector a 22.0, q 24.0; one
//             wave, two vectors 21.7, 24.2; four vectors 22.6, 26.1
// Wider rows (w: stream in fp32, every option, 8-bit codes), waves x vectors:
//   K = 5120, 8 x 2 / 16 x 1 / 4 x 4: 1 row a 2.61 / 2.77 / 2.89; 64 rows w 7.5 / 8.2 / 10.7; 1000 rows q 13.1 / 15.6 /
//             13.3; 4000 rows q 30.7 / 44.3 / 28.0, w 80 / 114 / 74
//   K = 8192, the same: 1 row a 2.77 / 2.98 / 3.01; 1000 rows w 29.8 / 39.1 / 37.2; 4000 rows a 48.3 / 49.9 / 48.0,
//             q 43 / 55 / 44
//   K = 12288, 16 x 2 / 8 x 4: 1 row a 3.66 / 3.48; 64 rows w 11.2 / 13.4; 1000 rows q 24.5 / 21.7, w 55 / 58; 4000
//             rows q 77 / 61, w 186 / 187.  K = 16384: 64 rows w 12.1 / 14.7; 1000 rows q 27.4 / 25.6, w 62 / 69;
//             4000 rows q 88 / 79, w 209 / 222
//   K = 18944 and 32768 fit 16 x 4 alone: 1 row a 5.06, 5.28; 4000 rows a 123, 183 (floors 118, 205), q 138, 189,
//             w 397, 497
// So 16 x 2 is the better form of few rows and of rows with every option, and not of many rows straight into codes.
#pragma once
#include <stdint.h>

namespace sq {

constexpr int kNormMaxK = 32768;

struct NormPlan {
    int waves;             // a row's; 1: four rows a workgroup, each its own wave's
    int nv;                // vectors a lane
};

inline NormPlan norm_plan(int M, int K) {
    const int vecs = (K + 7) / 8;
    if (vecs <= 64) return {1, 1};
    if (vecs <= 128) return {2, 1};
    if (vecs <= 256) return M <= 1024 ? NormPlan{4, 1} : NormPlan{2, 2};
    if (vecs <= 512) return M <= 512 ? NormPlan{8, 1} : NormPlan{4, 2};
    if (vecs <= 1024) return {8, 2};
    if (vecs <= 2048) return {16, 2};
    return {16, 4};
}

}  // namespace sq
