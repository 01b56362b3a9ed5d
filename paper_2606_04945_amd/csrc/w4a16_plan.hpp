// Launch plan of the weight-only products, without HIP.
//
// A workgroup multiplies NG groups of 16 outputs; the waves split K.  More groups read
// the rows of X fewer times, fewer make more workgroups.  The estimate, in units of one
// group's codes: rounds of 256 workgroups times (NG + what the rows cost), the rows of a
// full tile as much as a group.  Measured (us) at NG = 1 ... 5:
//   16 x 37888 x 3584: 41.9 25.2 23.6 21.5 19.6, estimate 20 15 16 15 12
//   1 x 24576 x 4096:  13.9 12.6 12.6 14.2 18.6, estimate 7.8 6.9 6.6 8.6 10.6
//   1 x 4096 x 4096:   4.6 5.3 6.4 7.2 9.9,      estimate 1.3 2.3 3.3 4.3 5.3
// Eight waves where workgroups are few (5 x 3584 x 18944 20.6 -> 15.1), four otherwise
// (2 x 12288 x 4096, NG = 1: 9.5 -> 8.5; 32 x 12288 x 4096, NG = 2: 19.0 -> 16.3).  Above
// 16 rows the registers hold at most two groups, and above 32 those of four waves.
// (These figures are of rows read in the operands' order, which now only up to four rows are;
// in whole lines and through LDS, us at 4, 8 and 16 rows: 4096 x 12288 12.9 14.3 17.1 ->
// 12.0 12.0 12.8, 4096 x 4096 5.6 6.1 7.3 -> 5.9 6.0 6.1.)
#pragma once
#include <stdint.h>

namespace sq {

struct W4a16Plan {
    int tm, ng, waves;     // row tiles of 16, groups of 16 outputs, waves
    bool lines;            // X read in whole lines and reordered through LDS
};

inline W4a16Plan w4a16_plan(int M, int N) {
    W4a16Plan p{M <= 16 ? 1 : M <= 32 ? 2 : 4, 1, 4, M > 4};
    const int64_t groups = ((int64_t)N + 15) / 16, row_tiles = ((int64_t)M + 16 * p.tm - 1) / (16 * p.tm);
    const int64_t rows = 4 + 12 * (M < 16 * p.tm ? M : 16 * p.tm) / 16;      // in sixteenths of a group
    int64_t best = INT64_MAX;
    for (int ng = 1; ng <= (p.tm == 1 ? 5 : 2); ++ng) {
        const int64_t wgs = (groups + ng - 1) / ng * row_tiles, cost = (wgs + 255) / 256 * (16 * ng + rows);
        if (cost < best) {
            best = cost;
            p.ng = ng;
            p.waves = ng <= 3 && p.tm < 4 && wgs <= (p.tm == 1 ? 512 : 256) ? 8 : 4;
        }
    }
    return p;
}

}  // namespace sq
