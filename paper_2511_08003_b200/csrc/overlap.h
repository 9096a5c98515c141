// Whether arrays with strides share bytes (host).  Ranges of addresses do not tell: the queries and keys of a fused projection
// interleave, and so do codes and scales that lie layer by layer.
#pragma once

#include <stdint.h>

namespace sharpv {

// Runs of `bytes` bytes at base + sum of i_k * stride[k], 0 <= i_k < count[k]; strides are not negative.
struct Runs {
    static constexpr int kMaxDims = 4;
    uintptr_t base;
    int64_t bytes;
    int dims;
    int64_t stride[kMaxDims], count[kMaxDims];
    uintptr_t end() const {
        uintptr_t e = base + (uintptr_t)bytes;
        for (int k = 0; k < dims; ++k) e += (uintptr_t)((count[k] - 1) * stride[k]);
        return e;
    }
    bool empty() const {
        for (int k = 0; k < dims; ++k)
            if (count[k] < 1) return true;
        return bytes < 1;
    }
};

enum class Share { no, yes, unsettled };

// Looks for whole x_k in [lo_k, hi_k] with -before < c + sum of x_k * stride_k < behind, the largest stride first: of each x_k only
// those are tried that leave the rest in reach, one to three where the layouts are nested as layouts are.
class ShareSearch {
public:
    ShareSearch(int64_t before, int64_t behind) : before_(before), behind_(behind) {}
    // `merge`: equal strides are one
    void add(int64_t stride, int64_t lo, int64_t hi, bool merge) {
        if (lo == hi && lo == 0) return;
        if (merge && stride == 0) return;
        int at = 0;
        while (at < n_ && d_[at].stride > stride) ++at;
        if (merge && at < n_ && d_[at].stride == stride) {
            d_[at].lo += lo;
            d_[at].hi += hi;
            return;
        }
        for (int k = n_++; k > at; --k) d_[k] = d_[k - 1];
        d_[at] = Dim{stride, lo, hi, 0, 0};
    }
    // `moves`: not all x_k are 0
    Share find(__int128 c, bool moves) {
        __int128 least = 0, most = 0;
        for (int k = n_ - 1; k >= 0; --k) {
            d_[k].rest_least = least;
            d_[k].rest_most = most;
            least += (__int128)d_[k].lo * d_[k].stride;
            most += (__int128)d_[k].hi * d_[k].stride;
        }
        return step(0, c, !moves);
    }

private:
    struct Dim { int64_t stride, lo, hi; __int128 rest_least, rest_most; };
    static __int128 floor_div(__int128 a, __int128 b) { return a >= 0 ? a / b : -((b - 1 - a) / b); }
    Share step(int k, __int128 c, bool moved) {
        if (--left_ < 0) return Share::unsettled;
        if (k == n_) return moved && c > -(__int128)before_ && c < behind_ ? Share::yes : Share::no;
        const Dim& d = d_[k];
        if (d.stride == 0) return step(k + 1, c, true);
        __int128 lo = d.lo, hi = d.hi;
        const __int128 from = floor_div(-(__int128)before_ - c - d.rest_most, d.stride) + 1;
        const __int128 to = -floor_div(-((__int128)behind_ - c - d.rest_least), d.stride) - 1;
        if (from > lo) lo = from;
        if (to < hi) hi = to;
        for (__int128 x = lo; x <= hi; ++x) {
            const Share s = step(k + 1, c + x * d.stride, moved || x != 0);
            if (s != Share::no) return s;
        }
        return Share::no;
    }
    int64_t before_, behind_;
    int n_ = 0, left_ = 1 << 14;
    Dim d_[2 * Runs::kMaxDims];
};

// Whether two arrays share bytes.
inline Share share_bytes(const Runs& a, const Runs& b) {
    if (a.empty() || b.empty() || a.base >= b.end() || b.base >= a.end()) return Share::no;
    ShareSearch s(a.bytes, b.bytes);
    for (int k = 0; k < a.dims; ++k) s.add(a.stride[k], 0, a.count[k] - 1, true);
    for (int k = 0; k < b.dims; ++k) s.add(b.stride[k], 1 - b.count[k], 0, true);
    return s.find((__int128)a.base - (__int128)b.base, false);
}

// Whether two runs of an array share bytes.
inline Share shares_own_bytes(const Runs& a) {
    if (a.empty()) return Share::no;
    ShareSearch s(a.bytes, a.bytes);
    for (int k = 0; k < a.dims; ++k) s.add(a.stride[k], 1 - a.count[k], a.count[k] - 1, false);
    return s.find(0, true);
}

}  // namespace sharpv
