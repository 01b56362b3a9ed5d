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
// (These figures are of rows read in the operands' order.)
//
// Rows in whole lines pass through LDS at each step, which costs a wave of few steps more than the lines save, and
// more the less there are of rows.  us, operands / lines, groups of 128 unless given:
//   4096 x 12288:  5 rows 10.4 / 11.2, 7 11.2 / 11.2, 8 11.7 / 11.3, 16 15.7 / 12.0
//   1024 x 8192:   5 rows 7.1 / 7.6, 6 7.5 / 7.6, 8 8.4 / 7.6, 16 11.0 / 7.7
//   4096 x 4096:   5 rows 5.4 / 5.8, 7 5.8 / 5.9, 8 6.0 / 5.9, 16 7.2 / 6.0
//   8192 x 4096:   5 rows 6.8 / 7.3, 8 7.0 / 7.3, 12 7.4 / 7.4, 16 7.9 / 7.4
//   2048 x 2048:   5 rows 3.7 / 4.0, 8 4.1 / 4.0, 16 4.8 / 4.0;   8192 x 2048: 8 5.2 / 5.6, 16 5.8 / 5.7
//   4096 x 1024:   5 rows 3.1 / 3.4, 8 3.2 / 3.4, 16 3.6 / 3.4
// In groups of 32, whose scales take registers, the more so with two groups of outputs or three: 8192 x 4096 8 rows
// 7.8 / 8.3, 12 8.1 / 8.3, 16 8.9 / 8.7; 12288 x 4096 5 10.2 / 11.2, 12 10.8 / 11.3, 16 11.5 / 11.4.  Three groups of
// outputs with larger groups, whose workgroups are two a CU, and four or five, whose four waves have twice the steps,
// gain or lose little from the first rows on: 12288 x 4096 5 rows 9.3 / 9.0, 24576 x 4096 of 64 15.4 / 14.8, of 128
// 13.9 / 14.0, 16384 x 4096 14.4 / 11.0, 37888 x 3584 15.7 / 16.7, of 32 22.5 / 20.3.
#pragma once
#include <stdint.h>

namespace sq {

struct W4a16Plan {
    int tm, ng, waves;     // row tiles of 16, groups of 16 outputs, waves
    bool lines;            // X read in whole lines and reordered through LDS
};

inline bool w4a16_lines(int M, int ng, int K, int group) {
    if (M <= 4 || M > 16) return M > 4;
    if ((ng >= 4 && K >= 2048) || (ng == 3 && group > 32 && K >= 4096)) return true;
    return (int64_t)(M - 4) * K > (group == 32 && ng > 1 ? 40960 : 12288);
}

// (without K and group: those of a deep product)
inline W4a16Plan w4a16_plan(int M, int N, int K = 1 << 17, int group = 128) {
    W4a16Plan p{M <= 16 ? 1 : M <= 32 ? 2 : 4, 1, 4, false};
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
    p.lines = w4a16_lines(M, p.ng, K, group);
    return p;
}

}  // namespace sq
