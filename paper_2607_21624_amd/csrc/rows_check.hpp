// rows_check.hpp -- argument checks of the entry points on matrices given by a
// pointer and a row stride (host).
#pragma once

#include <cstdint>

#include "../../include/fbl.h"

namespace fbl {

inline int64_t dtype_size(int32_t dt) { return dt == FBL_BF16 ? 2 : dt == FBL_F32 ? 4 : 0; }

// A matrix of `rows` rows of `width` elements of `es` bytes, `ld` elements apart.
struct RowsView {
    const void* p;
    int64_t rows, width, ld, es;
    uintptr_t begin() const { return reinterpret_cast<uintptr_t>(p); }
    int64_t bytes() const { return ((rows - 1) * ld + width) * es; }
    bool addressable() const { return rows <= (int64_t(1) << 46) / ld; }  // bytes() cannot overflow
    bool natural() const { return begin() % (uintptr_t)es == 0; }
    bool aligned16() const { return begin() % 16 == 0 && ld * es % 16 == 0; }
};

// Whether two of them share a byte.  Exact for two column views of the same rows (same
// row stride, one's rows between the other's columns); otherwise the byte ranges
// decide.
inline bool overlap(const RowsView& a, const RowsView& b) {
    if (!a.p || !b.p) return false;
    if (a.begin() >= b.begin() + (uintptr_t)b.bytes() || b.begin() >= a.begin() + (uintptr_t)a.bytes()) return false;
    if (a.ld * a.es != b.ld * b.es || a.rows < 2 || b.rows < 2) return true;
    const int64_t pitch = a.ld * a.es, wa = a.width * a.es, wb = b.width * b.es;
    int64_t d = (int64_t)(b.begin() - a.begin()) % pitch;  // b's columns from a's, within a row
    if (d < 0) d += pitch;
    return d < wa || d + wb > pitch;
}

constexpr int64_t kMaxExtent = INT32_MAX;
inline bool extent(int64_t n) { return n > 0 && n <= kMaxExtent; }

}  // namespace fbl
