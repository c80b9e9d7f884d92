// Whether two arrays with strides share an element: host code without a device, tested as such.
#pragma once
#include <algorithm>
#include <cstdint>

namespace overlap {

// `run` bytes at p + the sum of i stride[k], 0 <= i < count[k], in bytes; strides are not negative.
struct Array {
    uintptr_t p = 0;
    int64_t run = 0;
    int dims = 0;
    int64_t stride[4] = {}, count[4] = {};
    void dim(int64_t bytes, int64_t n)
    {
        if (n == 0) run = 0;
        if (n <= 1 || bytes == 0) return;
        stride[dims] = bytes;
        count[dims++] = n;
    }
    int64_t extent() const
    {
        int64_t e = run;
        for (int k = 0; k < dims; ++k) e += stride[k] * (count[k] - 1);
        return e;
    }
};

enum Answer { APART, SHARED, UNKNOWN };

struct Search {
    int64_t stride[8], low[8], high[8];         // multiples that are to be found, the largest stride first
    int64_t least[9], most[9];                  // what the strides from here on can make
    int count = 0, steps = 0;
    int64_t run_a = 0, run_b = 0;
    Answer from(int k, int64_t wanted)
    {
        if (++steps > 4096) return UNKNOWN;
        if (k == count) return wanted < run_a && wanted > -run_b ? SHARED : APART;
        // the multiples that leave something the rest can make, runs included
        const int64_t s = stride[k], top = wanted - least[k + 1] + run_b - 1, bottom = wanted - most[k + 1] - run_a + 1;
        const int64_t first = std::max(low[k], bottom > 0 ? (bottom + s - 1) / s : -(-bottom / s)), last = std::min(high[k], top >= 0 ? top / s : -((-top + s - 1) / s));
        Answer so_far = APART;
        for (int64_t x = first; x <= last; ++x) {
            const Answer a = from(k + 1, wanted - x * s);
            if (a != APART) so_far = a;
            if (so_far == SHARED || steps > 4096) return so_far;
        }
        return so_far;
    }
};

// Views of one buffer, whose strides are alike or nested, are settled in some ten steps; UNKNOWN where thousands do not settle it.
inline Answer of(const Array &a, const Array &b)
{
    if (a.run == 0 || b.run == 0) return APART;
    const int64_t there = (int64_t)(b.p - a.p);             // from a's begin to b's
    if (there >= a.extent() || -there >= b.extent()) return APART;
    // a's element at sum i s is b's at there + sum j t: sum i s - sum j t = there, but for the runs
    Search w;
    w.run_a = a.run;
    w.run_b = b.run;
    auto add = [&](int64_t stride, int64_t low, int64_t high) {
        for (int k = 0; k < w.count; ++k)
            if (w.stride[k] == stride) {
                w.low[k] += low;
                w.high[k] += high;
                return;
            }
        int at = w.count++;
        for (; at > 0 && w.stride[at - 1] < stride; --at) {
            w.stride[at] = w.stride[at - 1];
            w.low[at] = w.low[at - 1];
            w.high[at] = w.high[at - 1];
        }
        w.stride[at] = stride;
        w.low[at] = low;
        w.high[at] = high;
    };
    for (int k = 0; k < a.dims; ++k) add(a.stride[k], 0, a.count[k] - 1);
    for (int k = 0; k < b.dims; ++k) add(b.stride[k], 1 - b.count[k], 0);
    w.least[w.count] = w.most[w.count] = 0;
    for (int k = w.count; k-- > 0;) {
        w.least[k] = w.least[k + 1] + w.stride[k] * w.low[k];
        w.most[k] = w.most[k + 1] + w.stride[k] * w.high[k];
    }
    return w.from(0, there);
}

} // namespace overlap
