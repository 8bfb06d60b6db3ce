// Where arrays lie in memory, for the checks that what a call writes overlaps
// nothing else.
#pragma once

#include <cstddef>
#include <cstdint>

namespace tag {

// bytes from b up to e: runs of `run` bytes that repeat every `step` (0: no gaps that are known)
struct Area {
    uintptr_t b, e;
    int64_t step, run;
    bool meets(const Area &o) const {
        if (!(b < e && o.b < o.e && b < o.e && o.b < e)) return false;
        if (step == 0 || step != o.step) return true;
        // columns of wider rows, side by side: from this one's run on to the other's, within a row
        const int64_t d = o.b >= b ? (int64_t)((o.b - b) % (uintptr_t)step)
                                   : (step - (int64_t)((b - o.b) % (uintptr_t)step)) % step;
        return d < run || d + o.run > step;
    }
};

inline Area flat_area(const void *p, size_t bytes) { return Area{(uintptr_t)p, (uintptr_t)p + (p ? bytes : 0), 0, 0}; }

// rows of `row` bytes every `stride`
inline Area rows_area(const void *p, int64_t rows, int64_t stride, int64_t row) {
    return Area{(uintptr_t)p, (uintptr_t)p + (rows - 1) * stride + row, rows > 1 && stride >= row ? stride : 0, row};
}

}  // namespace tag
