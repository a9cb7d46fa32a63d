// C ABI of what stands beside the layer's products (see include/tp_linear.h): dropout without a stored mask.  Everything is checked before the
// first launch; nothing is allocated or synchronised here.
#include <cmath>
#include <cstdint>

#include "tp_checks.h"
#include "tp_internal.h"

using namespace tpl;

namespace {

// A mask whose block begins at (row, col) behind the caller's own position
int check_dropout(const tp_dropout_t* d, int64_t row, int64_t col, int64_t rows, int64_t cols, DropArgs* a) {
    if (!(d->p >= 0.0 && d->p <= 1.0)) return TP_ERR_MODE;
    if ((d->col0 & 7) || (col & 7) || (reinterpret_cast<uintptr_t>(d->offset_dev) & 7)) return TP_ERR_ALIGN;
    constexpr int64_t kRows = (int64_t)1 << 32, kCols = (int64_t)1 << 35;      // row and column group are words of the counter
    if (d->row0 < 0 || d->col0 < 0 || d->row0 > kRows || d->col0 > kCols || row > kRows || col > kCols || rows > kRows - d->row0 - row ||
        cols > kCols - d->col0 - col)
        return TP_ERR_SHAPE;
    a->key0 = (uint32_t)d->seed; a->key1 = (uint32_t)(d->seed >> 32);
    a->offset = d->offset; a->offset_dev = d->offset_dev;
    a->threshold = (uint32_t)std::nearbyint(d->p * 65536.0);
    a->factor = a->threshold < 65536 ? (float)(65536.0 / (65536.0 - a->threshold)) : 0.0f;
    a->row0 = (uint32_t)(d->row0 + row); a->group0 = (uint32_t)((d->col0 + col) >> 3);
    return TP_OK;
}

}  // namespace

extern "C" {

int tp_dropout_fwd(const tp_dropout_t* drop, const void* x, int64_t ld_x, int x_dtype, const void* bias, int epi, tp_cblk_t residual, tp_oblk_t y,
                   tp_oblk_t preact, int64_t rows, int64_t cols, void* hip_stream) {
    if (!drop) return TP_ERR_NULL;
    if (rows == 0 || cols == 0) {                // (an empty tensor has no address)
        DropArgs a;
        return check_dropout(drop, 0, 0, rows, cols, &a);
    }
    if (!x || !y.ptr) return TP_ERR_NULL;
    if (epi != TP_EPI_NONE && epi != TP_EPI_BIAS && epi != TP_EPI_BIAS_GELU) return TP_ERR_MODE;
    if (epi != TP_EPI_NONE && !bias) return TP_ERR_NULL;
    if (x_dtype != TP_F32 && x_dtype != TP_BF16) return TP_ERR_DTYPE;
    if (rows < 0 || cols < 0) return TP_ERR_SHAPE;
    if (!aligned16(x) || (bias && !aligned16(bias)) || (ld_x & 7)) return TP_ERR_ALIGN;
    if (ld_x < cols) return TP_ERR_SHAPE;
    if (int e = check_oblk(y, cols, false)) return e;
    if (preact.ptr) {
        if (int e = check_oblk(preact, cols, false)) return e;
        if (preact.dtype != TP_BF16) return TP_ERR_DTYPE;
    }
    if (residual.ptr) {
        if (!aligned16(residual.ptr) || (residual.ld & 7)) return TP_ERR_ALIGN;
        if (residual.ld < cols) return TP_ERR_SHAPE;
    }
    DropArgs a;
    if (int e = check_dropout(drop, 0, 0, rows, cols, &a)) return e;
    if (launch_dropout(a, x, ld_x, x_dtype == TP_F32, epi == TP_EPI_NONE ? nullptr : bias, epi == TP_EPI_BIAS_GELU, residual.ptr, residual.ld, y.ptr, y.ld,
                       y.dtype == TP_F32, preact.ptr, preact.ld, rows, cols, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return TP_ERR_HIP;
    return TP_OK;
}

int tp_dropout_bwd(const tp_dropout_t* drop, const void* dy, int64_t ld_dy, const void* preact, int64_t ld_pre, void* dx, int64_t ld_dx, void* db_f32,
                   int64_t rows, int64_t cols, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!drop || (rows != 0 && cols != 0 && (!dy || !dx))) return TP_ERR_NULL;
    if (rows < 0 || cols < 0 || (db_f32 && cols > INT32_MAX)) return TP_ERR_SHAPE;
    if (!aligned16(dy) || !aligned16(dx) || (cols & 7) || (ld_dy & 7) || (ld_dx & 7)) return TP_ERR_ALIGN;
    if (preact && (!aligned16(preact) || (ld_pre & 7))) return TP_ERR_ALIGN;
    if (db_f32 && !aligned16(db_f32)) return TP_ERR_ALIGN;
    if (ld_dy < cols || ld_dx < cols || (preact && ld_pre < cols)) return TP_ERR_SHAPE;
    DropArgs a;
    if (int e = check_dropout(drop, 0, 0, rows, cols, &a)) return e;
    if (db_f32 && workspace && (!aligned16(workspace) || workspace_bytes < colsum_ws_bytes(rows, cols))) return TP_ERR_WORKSPACE;
    if (cols == 0) return TP_OK;
    if (launch_dropout_bwd(a, dy, ld_dy, preact, ld_pre, dx, ld_dx, rows, cols, static_cast<float*>(db_f32), static_cast<float*>(workspace),
                           static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return TP_ERR_HIP;
    return TP_OK;
}

}  // extern "C"
