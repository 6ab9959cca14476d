// Argument checks that the entry points of the training operators share (host only).
#pragma once

#include <math.h>

#include "../../include/galore.h"

#include "mx.hpp"

namespace galore {

#define GALORE_TRY(expr)                                   \
    do {                                                   \
        hipError_t e_ = (expr);                            \
        if (e_ != hipSuccess) return GALORE_ERR_HIP;       \
    } while (0)

constexpr int64_t kMaxSide = int64_t{1} << 28;   // rows and columns: tile origins and grids stay within 32 bits
constexpr int32_t kMaxBatch = 65535;             // a grid's third dimension
constexpr size_t kAlign = 256;

inline bool dtype_ok(int32_t t) { return t == GALORE_F32 || t == GALORE_BF16; }
inline bool is_aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// rows x cols entries at pitch ld, `batch` of them at `stride` from each other (rows ld
// may pass 64 bits: divided, not multiplied)
inline bool matrix_ok(int64_t rows, int64_t cols, int64_t ld, int64_t stride, int32_t batch) {
    return ld >= cols && (batch == 1 || (rows == 0 ? stride >= 0 : stride / rows >= ld));
}

// `bytes` code bytes a row; GALORE_OK or the error
inline int check_mx(const galore_mx_t* q, int64_t rows, int64_t cols, int64_t block_bytes, int32_t batch) {
    if (q == nullptr) return GALORE_ERR_INVALID_ARG;
    if (rows > 0 && (q->codes == nullptr || q->scales == nullptr)) return GALORE_ERR_INVALID_ARG;
    if (!is_aligned(q->codes, 16) || !is_aligned(q->scales, 4)) return GALORE_ERR_INVALID_ARG;
    if (q->ldq % 16 != 0 || q->lds % 4 != 0) return GALORE_ERR_SHAPE;
    if (!matrix_ok(rows, mx_blocks(cols) * block_bytes, q->ldq, q->stride_q, batch)) return GALORE_ERR_SHAPE;
    if (!matrix_ok(rows, mx_scale_bytes(cols), q->lds, q->stride_s, batch)) return GALORE_ERR_SHAPE;
    if (batch > 1 && (q->stride_q % 16 != 0 || q->stride_s % 4 != 0)) return GALORE_ERR_SHAPE;
    return GALORE_OK;
}
constexpr int64_t kBytes8 = kMxBlock, kBytes4 = kMxBlock / 2;

inline MxMatrix matrix_of(const galore_mx_t* q, int32_t batch) {
    return {static_cast<uint8_t*>(q->codes), q->ldq, batch > 1 ? q->stride_q : 0, q->scales, q->lds,
            batch > 1 ? q->stride_s : 0};
}

inline bool sides_ok(int64_t rows, int64_t cols, int32_t batch) {
    return rows >= 0 && cols >= 1 && rows <= kMaxSide && cols <= kMaxSide && batch >= 1 && batch <= kMaxBatch;
}

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool finite_f(float x) { return isfinite(x); }

}  // namespace galore
