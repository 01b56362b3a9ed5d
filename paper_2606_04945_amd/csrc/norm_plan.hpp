// Launch plan of the norms, without HIP: waves that share a row, and vectors of 8
// entries that a lane holds.
#pragma once
#include <stdint.h>

namespace sq {

constexpr int kNormMaxK = 32768;

struct NormPlan {
    int waves;             // a row's; 1: four rows a workgroup, each its own wave's
    int nv;                // vectors a lane: 1, 2, 4 or 8
};

inline NormPlan norm_plan(int M, int K) {
    const int vecs = (K + 7) / 8;
    (void)M;
    NormPlan p{1, 1};
    while (64 * p.waves < vecs && p.waves < 4) p.waves *= 2;
    while (64 * p.waves * p.nv < vecs && p.nv < 4) p.nv *= 2;
    while (64 * p.waves * p.nv < vecs) p.waves *= 2;
    return p;
}

}  // namespace sq
