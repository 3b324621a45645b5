// Decisions of the training operators' host code that need no device, free of
// HIP so that they can be checked without one: sizes, extents and overlaps of
// strided tensors.
#pragma once

#include <cstdint>

namespace sdpops {

// A strided tensor of up to three outer dimensions around `inner` contiguous
// elements; strides count elements.
struct Layout {
    int64_t ext[3];
    int64_t stride[3];
    int64_t inner;
};

// a / b rounded up, for all a >= 0 that an int32_t holds (a + b - 1 may not).
constexpr int32_t parts_of(int32_t a, int32_t b) { return a / b + (a % b != 0 ? 1 : 0); }

// a b c of three sizes, or -1 where that does not fit 60 bits.
inline int64_t product(int64_t a, int64_t b, int64_t c) {
    if (a == 0 || b == 0 || c == 0) return 0;
    const int64_t most = (int64_t)1 << 60;
    return b <= most / a && c <= most / (a * b) ? a * b * c : -1;
}

inline bool no_elements(const Layout &l) { return l.inner == 0 || l.ext[0] == 0 || l.ext[1] == 0 || l.ext[2] == 0; }

// Elements from the first to the last one, or -1 where that does not fit 60
// bits or a stride is negative.
inline int64_t span(const Layout &l) {
    if (no_elements(l)) return 0;
    __int128 s = l.inner;
    for (int k = 0; k < 3; ++k) {
        if (l.stride[k] < 0) return -1;
        s += (__int128)(l.ext[k] - 1) * l.stride[k];
    }
    return s < ((__int128)1 << 60) ? (int64_t)s : -1;
}

// Whether no two index tuples name the same element, by the sufficient test
// that each dimension steps past all that the smaller ones cover.
inline bool injective(const Layout &l) {
    if (no_elements(l)) return true;
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (l.stride[order[j]] < l.stride[order[i]]) {
                const int t = order[i];
                order[i] = order[j];
                order[j] = t;
            }
    __int128 covered = l.inner;
    for (int k : order) {
        if (l.ext[k] == 1) continue;
        if ((__int128)l.stride[k] < covered) return false;
        covered += (__int128)(l.ext[k] - 1) * l.stride[k];
    }
    return true;
}

// Whether the strides agree wherever both tensors step, so that equal
// addresses mean the same tensor.
inline bool same_strides(const Layout &a, const Layout &b) {
    for (int k = 0; k < 3; ++k)
        if (a.ext[k] > 1 && b.ext[k] > 1 && a.stride[k] != b.stride[k]) return false;
    return true;
}

inline bool same_tensor(const char *pa, const Layout &a, const char *pb, const Layout &b) {
    if (pa != pb || a.inner != b.inner) return false;
    for (int k = 0; k < 3; ++k)
        if (a.ext[k] != b.ext[k] || (a.ext[k] > 1 && a.stride[k] != b.stride[k])) return false;
    return true;
}

// The outer dimensions (0 and 1) of two tensors that step alike there, around `inner`
// elements of each step: of a buffer that holds both.
inline Layout around(const Layout &a, const Layout &b, int64_t inner) {
    Layout all{{1, 1, 1}, {0, 0, 0}, inner};
    for (int k = 0; k < 2; ++k) {
        all.ext[k] = a.ext[k] > b.ext[k] ? a.ext[k] : b.ext[k];
        all.stride[k] = a.ext[k] > 1 ? a.stride[k] : b.stride[k];
    }
    return all;
}

// Whether `hi`, which starts `apart` elements past `lo`, lies in other columns of the
// same rows: past all that lo has of a row, and before its next one.
inline bool other_columns(const Layout &lo, const Layout &hi, int64_t apart) {
    for (int k = 0; k < 2; ++k)
        if (lo.ext[k] > 1 && hi.ext[k] > 1 && lo.stride[k] != hi.stride[k]) return false;
    const int64_t lo_width = (lo.ext[2] - 1) * lo.stride[2] + lo.inner, hi_width = (hi.ext[2] - 1) * hi.stride[2] + hi.inner;
    return apart >= lo_width && injective(around(lo, hi, apart + hi_width));
}

// Whether two tensors of elements of `size` bytes share no element: their
// byte ranges are apart, or they are columns of the same rows, or runs of heads
// (dimension 2) of one fused tensor, whose runs do not meet.  Where none can be
// shown, false.
inline bool disjoint(const char *pa, const Layout &a, const char *pb, const Layout &b, int64_t size) {
    if (no_elements(a) || no_elements(b)) return true;
    const int64_t sa = span(a) * size, sb = span(b) * size;
    if (pa + sa <= pb || pb + sb <= pa) return true;
    const bool a_first = pa <= pb;
    const Layout &lo = a_first ? a : b, &hi = a_first ? b : a;
    const int64_t apart = a_first ? pb - pa : pa - pb;
    if (apart % size == 0 && other_columns(lo, hi, apart / size)) return true;
    if (a.inner != b.inner || !same_strides(a, b)) return false;
    const int64_t hs = lo.ext[2] > 1 ? lo.stride[2] : hi.ext[2] > 1 ? hi.stride[2] : lo.inner;
    if (hs < lo.inner || apart % (hs * size) != 0) return false;
    const int64_t first = apart / (hs * size);
    if (first < lo.ext[2]) return false;
    Layout all = around(lo, hi, lo.inner);
    all.stride[2] = hs;
    all.ext[2] = first + hi.ext[2];
    return injective(all);
}

}  // namespace sdpops
