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
//   16384 x 512: a wave a row a 14.9, two 16.4, four 25; 16384 x 1024: two waves, one vector a 22.0, q 24.0; one
//             wave, two vectors 21.7, 24.2; four vectors 22.6, 26.1
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
