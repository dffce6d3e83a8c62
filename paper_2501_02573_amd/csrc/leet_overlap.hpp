// Whether two strided tensors share memory: host arithmetic on addresses alone.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace leet {

struct Dim {
    long long size, stride;
};

// Rows of `count` items of `item` bytes at an address and at all combinations of up to three strides (in items) behind it.  No
// address or no rows: an empty span, which shares nothing.
struct Span {
    using Wide = __int128;  // bytes: a size times a stride, whatever they are
    struct Step {
        Wide size, stride;
    };
    Wide at = 0, first = 0, last = 0, width = 0;
    Step dims[3];
    int n = 0;

    Span() = default;
    Span(const void* data, long long item, long long count, std::initializer_list<Dim> strides = {}) {
        if (!data || count <= 0) return;
        const Wide bytes = (Wide)item * count;
        at = first = (Wide) reinterpret_cast<uintptr_t>(data);
        last = at + bytes;
        for (const Dim& d : strides) {
            if (d.size <= 0) {
                *this = Span();
                return;
            }
            if (d.size == 1) continue;
            dims[n] = {d.size, (Wide)d.stride * item};
            const Wide reach = (dims[n].size - 1) * dims[n].stride;
            (reach < 0 ? first : last) += reach;
            ++n;
        }
        width = bytes;
    }
    bool operator==(const Span& o) const {
        if (at != o.at || width != o.width || n != o.n) return false;
        for (int i = 0; i < n; ++i)
            if (dims[i].size != o.dims[i].size || dims[i].stride != o.dims[i].stride) return false;
        return true;
    }
};

// Looks for a row of b that begins less than its width before a row of a, or less than a's width behind it: a sum of whole
// multiples of the strides in a range.  The largest stride's multiples are tried first, and of each stride only those that the
// smaller ones can still bring into the range: one or two where the larger strides step over all that the smaller ones reach,
// as those of dense tensors and of parts of one buffer do.
class RowSearch {
    using Wide = Span::Wide;
    struct Term {
        Wide stride, least, most;  // stride > 0
    };
    Term terms_[6];
    int n_ = 0;
    Wide below_[7] = {0}, above_[7] = {0};  // what the terms from i on reach
    Wide low_, high_;
    int looks_ = kLooks;

    void add(Wide stride, Wide least, Wide most) {
        if (stride < 0) {
            const Wide l = least;
            least = -most;
            most = -l;
            stride = -stride;
        }
        if (stride == 0) return;  // rows over one another
        int i = 0;
        while (i < n_ && terms_[i].stride > stride) ++i;
        if (i < n_ && terms_[i].stride == stride) {
            terms_[i].least += least;
            terms_[i].most += most;
            return;
        }
        for (int j = n_++; j > i; --j) terms_[j] = terms_[j - 1];
        terms_[i] = {stride, least, most};
    }
    // the largest whole number not above x / y, y > 0
    static Wide floored(Wide x, Wide y) { return x / y - (x % y < 0); }

    bool from(int i, Wide at) {
        if (i == n_) return at >= low_ && at <= high_;
        const Term& t = terms_[i];
        Wide c = -floored(-(low_ - at - above_[i + 1]), t.stride), end = floored(high_ - at - below_[i + 1], t.stride);
        if (c < t.least) c = t.least;
        if (end > t.most) end = t.most;
        for (; c <= end; ++c) {
            if (looks_ == 0) return false;
            --looks_;
            if (from(i + 1, at + c * t.stride)) return true;
        }
        return false;
    }

public:
    static constexpr int kLooks = 256;

    bool found(const Span& a, const Span& b) {
        low_ = 1 - b.width;
        high_ = a.width - 1;
        for (int i = 0; i < a.n; ++i) add(-a.dims[i].stride, 0, a.dims[i].size - 1);
        for (int i = 0; i < b.n; ++i) add(b.dims[i].stride, 0, b.dims[i].size - 1);
        for (int i = n_ - 1; i >= 0; --i) {
            below_[i] = below_[i + 1] + terms_[i].stride * terms_[i].least;
            above_[i] = above_[i + 1] + terms_[i].stride * terms_[i].most;
        }
        return from(0, b.at - a.at);
    }
};

// True: they share a byte.  False: they share none, or their strides leave so many possibilities that kLooks did not find one.
inline bool overlap(const Span& a, const Span& b) {
    if (a.width == 0 || b.width == 0 || a.last <= b.first || b.last <= a.first) return false;
    return RowSearch().found(a, b);
}

}  // namespace leet
