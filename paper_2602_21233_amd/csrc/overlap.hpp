// Whether arrays of a call lie on each other, found on the host from addresses and strides.
#pragma once
#include <stdint.h>

namespace spa {

typedef __int128 wide;               // strides may be any 64-bit values

// n[0] x n[1] rows of `len` bytes, step[0] and step[1] (>= 0) bytes apart; none where len is 0
struct Rows {
    wide at, step[2];
    int64_t n[2], len;
};
inline Rows rows_of(const void* p, int64_t n0, wide step0, int64_t n1, wide step1, int64_t len) {
    return {(wide)(uintptr_t)p, {n0 > 1 ? step0 : 0, n1 > 1 ? step1 : 0}, {n0, n1}, p != nullptr && n0 > 0 && n1 > 0 ? len : 0};
}
inline Rows row_of(const void* p, int64_t bytes) { return rows_of(p, 1, 0, 1, 0, bytes); }

inline wide end_of(const Rows& r) { return r.at + (r.n[0] - 1) * r.step[0] + (r.n[1] - 1) * r.step[1] + r.len; }
inline wide floor_div(wide a, wide b) { return a >= 0 ? a / b : -((-a + b - 1) / b); }
// whether lo < base + u * step < hi for a u of u0 .. u1
inline bool reaches(wide base, wide step, wide u0, wide u1, wide lo, wide hi) {
    if (step == 0) return u0 <= u1 && lo < base && base < hi;
    const wide least = floor_div(lo - base, step) + 1;          // first u past lo
    const wide u = least > u0 ? least : u0;
    return u <= u1 && base + u * step < hi;
}

// Exact where the steps of both agree, which slices of one tensor have, and where one of the two is a single row.  Others are taken to lie
// on each other as soon as their extents do.
inline bool overlap(const Rows& a, const Rows& b) {
    if (a.len == 0 || b.len == 0 || end_of(a) <= b.at || end_of(b) <= a.at) return false;
    wide step[2];
    for (int x = 0; x < 2; ++x) {
        if (a.n[x] > 1 && b.n[x] > 1 && a.step[x] != b.step[x]) return true;
        step[x] = a.n[x] > 1 ? a.step[x] : b.step[x];
    }
    // rows i of a and k of b are base + (i0 - k0) step[0] + (i1 - k1) step[1] apart
    const wide base = a.at - b.at;
    for (int64_t v = 1 - b.n[1]; v < a.n[1]; ++v)
        if (reaches(base + v * step[1], step[0], 1 - (wide)b.n[0], (wide)a.n[0] - 1, -(wide)a.len, b.len)) return true;
    return false;
}
// whether rows of one array lie on each other
inline bool overlaps_itself(const Rows& a) {
    const wide s0 = a.step[0], s1 = a.step[1], n0 = a.n[0], n1 = a.n[1];
    if ((n0 > 1 && s0 < a.len) || (n1 > 1 && s1 < a.len)) return true;
    if (n0 == 1 || n1 == 1 || s0 >= (n1 - 1) * s1 + a.len || s1 >= (n0 - 1) * s0 + a.len) return false;
    for (wide v = 1; v < n1; ++v)
        if (reaches(v * s1, s0, 1 - n0, n0 - 1, -(wide)a.len, a.len)) return true;
    return false;
}

}  // namespace spa
