// Where strided arrays lie, on the host: whether two of them share an entry, or one of them an entry with itself.
#pragma once
#include <cstdint>
#include <initializer_list>
#include <utility>

namespace ckks {

// Bytes [lo, hi) that an array of rows touches: `n` counts and strides (in elements), outermost first.
struct Extent {
    uintptr_t lo, hi;
};
inline Extent extent(const void *p, uint32_t elem_bytes, std::initializer_list<std::pair<uint64_t, int64_t>> dims) {
    int64_t lo = 0, hi = 0;
    for (const auto &d : dims) {
        if (!d.first) return {0, 0};
        const int64_t span = (int64_t)(d.first - 1) * d.second;
        (span < 0 ? lo : hi) += span;
    }
    return {(uintptr_t)p + (uintptr_t)(lo * elem_bytes), (uintptr_t)p + (uintptr_t)((hi + 1) * elem_bytes)};
}
inline bool overlap(const Extent &a, const Extent &b) { return a.lo < b.hi && b.lo < a.hi && a.lo != a.hi && b.lo != b.hi; }

// An array of runs of `run` bytes, one for each index: counts and strides (in bytes), outermost first.
struct Runs {
    const void *at;
    int64_t run;
    int dims;
    struct {
        int64_t n, stride;
    } dim[3];
};

// Whether some whole numbers d_k of [lo_k, hi_k] bring at + sum d_k stride_k strictly between -run and run.  The widest stride goes
// first: the others reach past it a little at most where arrays are nested, so few of its d_k are looked at.  With `tries` used up the
// answer is yes.
struct Step {
    int64_t lo, hi, stride;
};
inline bool reaches(int64_t at, int64_t run, const Step *s, int n, int &tries) {
    if (!n) return at > -run && at < run;
    if (--tries < 0) return true;
    int64_t low = 0, high = 0;  // of the other steps
    for (int k = 1; k < n; ++k) {
        low += s[k].lo * s[k].stride;
        high += s[k].hi * s[k].stride;
    }
    // d * stride has to lie in (-run - high - at, run - low - at)
    const int64_t from = 1 - run - high - at, to = run - 1 - low - at, w = s[0].stride;
    if (!w) return from <= 0 && to >= 0 && reaches(at, run, s + 1, n - 1, tries);
    const auto floor_div = [](int64_t a, int64_t b) { return a / b - (a % b < 0); };
    int64_t d = -floor_div(-from, w), end = floor_div(to, w);
    if (d < s[0].lo) d = s[0].lo;
    if (end > s[0].hi) end = s[0].hi;
    for (; d <= end; ++d)
        if (reaches(at + d * w, run, s + 1, n - 1, tries)) return true;
    return false;
}
// Strides made positive, widest first.
inline bool reaches(int64_t at, int64_t run, Step *s, int n) {
    for (int k = 0; k < n; ++k) {
        if (s[k].lo > s[k].hi) return false;
        if (s[k].stride < 0) s[k] = {-s[k].hi, -s[k].lo, -s[k].stride};
        for (int j = k; j && s[j].stride > s[j - 1].stride; --j) std::swap(s[j], s[j - 1]);
    }
    int tries = 1 << 16;
    return reaches(at, run, (const Step *)s, n, tries);
}

// Two arrays of as many dimensions and runs of the same length share a byte.
inline bool share(const Runs &a, const Runs &b) {
    Step s[6];
    int n = 0;
    for (int k = 0; k < a.dims; ++k) {
        const auto &x = a.dim[k], &y = b.dim[k];
        if (!x.n || !y.n) return false;
        if (x.stride == y.stride) {
            s[n++] = {1 - y.n, x.n - 1, x.stride};
            continue;
        }
        if (x.n > 1) s[n++] = {0, x.n - 1, x.stride};
        if (y.n > 1) s[n++] = {1 - y.n, 0, y.stride};
    }
    return reaches((int64_t)((uintptr_t)a.at - (uintptr_t)b.at), a.run, s, n);
}

// Two runs of one array share a byte.
inline bool share_within(const Runs &a) {
    Step s[3];
    // nested arrays, and those are nearly all, have each stride at least as wide as all that lies within it
    int n = 0;
    for (int k = 0; k < a.dims; ++k) {
        if (!a.dim[k].n) return false;
        if (a.dim[k].n == 1) continue;
        s[n++] = {0, a.dim[k].n - 1, a.dim[k].stride < 0 ? -a.dim[k].stride : a.dim[k].stride};
        for (int j = n - 1; j && s[j].stride < s[j - 1].stride; --j) std::swap(s[j], s[j - 1]);
    }
    int64_t span = a.run;
    bool nested = true;
    Step all[3];
    for (int k = 0; k < n; ++k) {
        nested &= s[k].stride >= span;
        span += s[k].hi * s[k].stride;
        all[k] = s[k];
    }
    if (nested) return false;
    // the first index in which the two runs differ, the others either way
    const int dims = n;
    for (int lead = 0; lead < dims; ++lead) {
        n = 0;
        s[n++] = {1, all[lead].hi, all[lead].stride};
        for (int k = lead + 1; k < dims; ++k) s[n++] = {-all[k].hi, all[k].hi, all[k].stride};
        if (reaches(0, a.run, s, n)) return true;
    }
    return false;
}

}  // namespace ckks
