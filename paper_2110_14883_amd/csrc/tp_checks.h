// Checks of arguments that the C-ABI host code shares (tp_api.cpp, tp_ops.cpp): blocks, workspaces, ranges of memory.
#pragma once
#include <cstddef>
#include <cstdint>
#include <utility>

#include "tp_linear.h"

namespace tpl {

constexpr int64_t kMaxLd = (int64_t)1 << 21;    // keeps every in-tile byte offset below 2^31

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_cblk(const tp_cblk_t& b, int64_t cols) {
    if (!b.ptr) return TP_ERR_NULL;
    if (!aligned16(b.ptr) || (b.ld & 7) || (cols & 7)) return TP_ERR_ALIGN;
    if (b.ld < cols || b.ld > kMaxLd) return TP_ERR_SHAPE;
    return TP_OK;
}
inline int check_oblk(const tp_oblk_t& b, int64_t cols, bool f32_only) {
    if (!b.ptr) return TP_ERR_NULL;
    if (b.dtype != TP_BF16 && b.dtype != TP_F32) return TP_ERR_DTYPE;
    if (f32_only && b.dtype != TP_F32) return TP_ERR_DTYPE;
    if (!aligned16(b.ptr) || (b.ld & 7) || (cols & 7)) return TP_ERR_ALIGN;
    if (b.ld < cols) return TP_ERR_SHAPE;
    return TP_OK;
}

inline bool ws_ok(size_t need, const void* workspace, size_t bytes) {
    return need == 0 || (workspace && bytes >= need && aligned16(workspace));
}

// Bytes that a block of rows x cols takes up (es bytes an element)
struct Range { uintptr_t lo, hi; };
inline Range span(const void* p, int64_t ld, int64_t rows, int64_t cols, int es) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Range{lo, lo + (uintptr_t)(((rows - 1) * ld + cols) * es)};
}
inline bool overlap(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }
// The same of two blocks of `rows` rows, row by row where their rows lie equally far apart: columns of one matrix may lie between each other's rows.
// (pitch, width: bytes from row to row and of a row.)
inline bool rows_overlap(const void* p, int64_t pitch, int64_t width, const void* q, int64_t pitch_q, int64_t width_q, int64_t rows) {
    if (pitch != pitch_q) return overlap(span(p, pitch, rows, width, 1), span(q, pitch_q, rows, width_q, 1));
    uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    if (b < a) { std::swap(a, b); std::swap(width, width_q); }
    const uint64_t down = (uint64_t)(b - a) / (uint64_t)pitch, right = (uint64_t)(b - a) % (uint64_t)pitch;      // b's first row from a's, and its first byte there
    return (down < (uint64_t)rows && right < (uint64_t)width) || (down + 1 < (uint64_t)rows && right + (uint64_t)width_q > (uint64_t)pitch);
}

}  // namespace tpl
