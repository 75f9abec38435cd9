// tas_step_overlap.h - whether two strided tensors share memory (host only).
#pragma once
#include <stdint.h>

#include <algorithm>

namespace tas_step_impl {

// Rows of `row` adjacent units, at base + i0 stride[0] + i1 stride[1] + i2 stride[2] (units)
// for all 0 <= i < n, none of them negative but base, an address of any 64 bits. The unit is the
// caller's, the same on both sides: 16 bytes, two or one.
struct Region {
    int64_t base, row;
    int64_t stride[3], n[3];
};

// a + sum i s + x = b + sum j t + y, with x and y inside the rows, has a solution where
// b - a is a sum of multiples: of every s from 0 to n - 1, of every t from 1 - n to 0, and
// of 1 between the rows' lengths. Tried from the longest stride on; what the shorter ones
// reach leaves a multiple or two of each where tensors are nested as usual. Past kTries
// (strides that no usual tensors have) they count as overlapping, and so do regions of kLongest
// units, more than there are addresses: below it no sum or difference of places overflows.
class Overlap {
    static constexpr int kTries = 1 << 14;
    static constexpr int64_t kLongest = int64_t(1) << 60;
    struct Axis {
        int64_t stride, lo, hi;  // lo to hi times the stride
    };
    Axis axes[7];
    int n = 0, tries = 0;
    int64_t least[8] = {}, most[8] = {};  // that the axes from one on reach

    void add(int64_t stride, int64_t lo, int64_t hi) {
        if (!stride || lo == hi) return;  // no other places
        for (int i = 0; i < n; i++)
            if (axes[i].stride == stride) {
                axes[i].lo += lo;
                axes[i].hi += hi;
                return;
            }
        axes[n++] = {stride, lo, hi};
    }
    // From the first unit of a region to behind the last.
    static int64_t span(const Region &r) {
        int64_t sum = r.row;
        for (int i = 0; i < 3; i++) {
            int64_t x;
            if (sum >= kLongest || __builtin_mul_overflow(r.stride[i], r.n[i] - 1, &x) ||
                x >= kLongest)
                return kLongest;
            sum += x;
        }
        return sum;
    }
    static int64_t floor_div(int64_t x, int64_t y) { return x / y - (x % y < 0); }
    bool reached(int i, int64_t d) {
        if (d < least[i] || d > most[i]) return false;
        if (i == n || ++tries > kTries) return true;
        const Axis &x = axes[i];
        const int64_t lo = std::max(x.lo, -floor_div(most[i + 1] - d, x.stride));
        const int64_t hi = std::min(x.hi, floor_div(d - least[i + 1], x.stride));
        for (int64_t m = lo; m <= hi; m++)
            if (reached(i + 1, d - m * x.stride)) return true;
        return false;
    }

  public:
    bool operator()(const Region &a, const Region &b) {
        n = tries = 0;
        for (int i = 0; i < 3; i++)
            if (!a.n[i] || !b.n[i]) return false;
        const int64_t span_a = span(a), span_b = span(b);
        if (span_a >= kLongest || span_b >= kLongest) return true;
        const uint64_t from_a = (uint64_t)b.base - (uint64_t)a.base, from_b = 0 - from_a;
        if (from_a >= (uint64_t)span_a && from_b >= (uint64_t)span_b) return false;
        for (int i = 0; i < 3; i++) {
            add(a.stride[i], 0, a.n[i] - 1);
            add(b.stride[i], 1 - b.n[i], 0);
        }
        add(1, 1 - b.row, a.row - 1);
        std::sort(axes, axes + n, [](const Axis &x, const Axis &y) { return x.stride > y.stride; });
        least[n] = most[n] = 0;
        for (int i = n - 1; i >= 0; i--) {
            least[i] = least[i + 1] + axes[i].lo * axes[i].stride;
            most[i] = most[i + 1] + axes[i].hi * axes[i].stride;
        }
        return reached(0, (int64_t)from_a);
    }
};

}  // namespace tas_step_impl
