// Sequences of a ragged batch and the blocks of a paged cache they touch: index
// arithmetic shared by the kernels and by host code without a GPU compiler.
//
// Sequence b's new tokens are rows cu[b] .. cu[b + 1] - 1 of the batch and are the
// last of its len[b] cache positions.  Both arrays live on the device, where a
// call cannot check them, so every reader clamps: rows to [0, T], lengths to what
// the page table can hold.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define SQ_HD __host__ __device__ __forceinline__
#else
#define SQ_HD inline
#endif

namespace sq {

struct Seq {
    int t0, n;     // first row and number of new tokens
    int len;       // positions in the cache, the new tokens' among them
    int off;       // position of the first new token; negative: those before 0 have none
};

SQ_HD Seq make_seq(int c0, int c1, int len, int T, int max_len) {
    Seq s;
    s.t0 = c0 < 0 ? 0 : c0 > T ? T : c0;
    const int t1 = c1 < s.t0 ? s.t0 : c1 > T ? T : c1;
    s.n = t1 - s.t0;
    s.len = len < 0 ? 0 : len > max_len ? max_len : len;
    s.off = s.len - s.n;
    return s;
}

// Where a work list has room for ceil-like counts of every sequence without
// knowing them: sequence b's part starts at floor(cu[b] per / size) + extra b and
// has at least ceil(n per / size) + extra - 1 places.  Non-decreasing in b.  T per is
// below 2^31.
SQ_HD int64_t list_start(int c0, int b, int per, int size, int extra) {
    return c0 * per / size + (int64_t)extra * b;
}

// Page-sized blocks of the cache that sequence s writes: [first, first + count).
// At most floor(n / page) + 2.
SQ_HD int touched_first(const Seq& s, int page) { return (s.off > 0 ? s.off : 0) / page; }
SQ_HD int touched_count(const Seq& s, int page) {
    if (s.len <= 0 || s.n <= 0) return 0;
    return (s.len - 1) / page - touched_first(s, page) + 1;
}
inline int64_t touched_slots(int T, int B, int page) { return (int64_t)T / page + 2 * (int64_t)B; }

}  // namespace sq
