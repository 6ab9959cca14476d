// Host side of the training operators: argument validation and launches. As in
// the rest of the library everything is enqueued on the caller's stream, nothing
// allocates device memory and nothing synchronises.
#include "../../include/galore.h"

#include "host_checks.hpp"
#include "training.hpp"

using namespace galore;

extern "C" {

int64_t galore_mx_scale_bytes(int64_t cols) { return cols < 1 || cols > kMaxSide ? 0 : mx_scale_bytes(cols); }

// ---- 8-bit checkpoints ------------------------------------------------------

int galore_checkpoint_pack(const void* X, int32_t x_dtype, int64_t tokens, int64_t cols, int64_t ldx, int64_t stride_x,
                           const galore_mx_t* out, int32_t batch, hipStream_t stream) {
    if ((X == nullptr && tokens > 0) || !dtype_ok(x_dtype)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, cols, batch) || !matrix_ok(tokens, cols, ldx, stride_x, batch)) return GALORE_ERR_SHAPE;
    const int e = check_mx(out, tokens, cols, kBytes8, batch);
    if (e != GALORE_OK || tokens == 0) return e;
    GALORE_TRY(launch_pack(X, x_dtype == GALORE_BF16, ldx, stride_x, matrix_of(out, batch), tokens, cols, batch, stream));
    return GALORE_OK;
}

int galore_checkpoint_unpack(const galore_mx_t* in, int64_t tokens, int64_t cols, void* X, int32_t x_dtype, int64_t ldx,
                             int64_t stride_x, int32_t batch, hipStream_t stream) {
    if ((X == nullptr && tokens > 0) || !dtype_ok(x_dtype)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, cols, batch) || !matrix_ok(tokens, cols, ldx, stride_x, batch)) return GALORE_ERR_SHAPE;
    const int e = check_mx(in, tokens, cols, kBytes8, batch);
    if (e != GALORE_OK || tokens == 0) return e;
    GALORE_TRY(launch_unpack(matrix_of(in, batch), X, x_dtype == GALORE_BF16, ldx, stride_x, tokens, cols, batch, stream));
    return GALORE_OK;
}

size_t galore_checkpoint_weight_grad_workspace_size(int64_t tokens, int64_t m, int64_t n, int32_t batch) {
    if (!sides_ok(tokens, n, batch) || m < 1 || m > kMaxSide) return 0;
    const int splits = weight_grad_splits(tokens, m, n, batch);
    return splits > 1 ? align_up(sizeof(float) * static_cast<size_t>(m) * n * splits * batch) : 0;
}

int galore_checkpoint_weight_grad(const void* dY, int32_t dy_dtype, int64_t ldy, int64_t stride_y, const galore_mx_t* x,
                                  int64_t tokens, int64_t m, int64_t n, void* G, int32_t g_dtype, int64_t ldg,
                                  int64_t stride_g, int32_t accumulate, int32_t batch, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream) {
    if ((dY == nullptr && tokens > 0) || G == nullptr || !dtype_ok(dy_dtype) || !dtype_ok(g_dtype))
        return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, n, batch) || m < 1 || m > kMaxSide) return GALORE_ERR_SHAPE;
    if (!matrix_ok(tokens, m, ldy, stride_y, batch) || !matrix_ok(m, n, ldg, stride_g, batch)) return GALORE_ERR_SHAPE;
    const int e = check_mx(x, tokens, n, kBytes8, batch);
    if (e != GALORE_OK) return e;
    const size_t need = galore_checkpoint_weight_grad_workspace_size(tokens, m, n, batch);
    if (workspace != nullptr && (!is_aligned(workspace, kAlign) || workspace_bytes < need)) return GALORE_ERR_WORKSPACE;
    WeightGradArgs a{};
    a.dY = dY;
    a.dy_bf16 = dy_dtype == GALORE_BF16;
    a.ldy = ldy;
    a.strideY = stride_y;
    a.X = matrix_of(x, batch);
    a.G = G;
    a.g_bf16 = g_dtype == GALORE_BF16;
    a.ldg = ldg;
    a.strideG = stride_g;
    a.T = tokens;
    a.m = m;
    a.n = n;
    a.accumulate = accumulate != 0;
    a.part = static_cast<float*>(workspace);
    GALORE_TRY(launch_weight_grad(a, batch, stream));
    return GALORE_OK;
}

// ---- microscaled 4-bit floating point ----------------------------------------

int galore_mx4_quantize(const void* X, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ldx, int64_t stride_x,
                        const galore_mx_t* by_rows, const galore_mx_t* by_columns, int32_t batch, hipStream_t stream) {
    if ((X == nullptr && rows > 0) || !dtype_ok(x_dtype)) return GALORE_ERR_INVALID_ARG;
    if (by_rows == nullptr && by_columns == nullptr) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(rows, cols, batch) || !matrix_ok(rows, cols, ldx, stride_x, batch)) return GALORE_ERR_SHAPE;
    if (rows == 0) return GALORE_OK;
    MxMatrix q{}, qt{};
    if (by_rows != nullptr) {
        const int e = check_mx(by_rows, rows, cols, kBytes4, batch);
        if (e != GALORE_OK) return e;
        q = matrix_of(by_rows, batch);
    }
    if (by_columns != nullptr) {
        const int e = check_mx(by_columns, cols, rows, kBytes4, batch);
        if (e != GALORE_OK) return e;
        qt = matrix_of(by_columns, batch);
    }
    GALORE_TRY(launch_mx4_quantize(X, x_dtype == GALORE_BF16, ldx, stride_x, by_rows ? &q : nullptr,
                                   by_columns ? &qt : nullptr, rows, cols, batch, stream));
    return GALORE_OK;
}

int galore_mx4_dequantize(const galore_mx_t* in, int64_t rows, int64_t cols, void* X, int32_t x_dtype, int64_t ldx,
                          int64_t stride_x, int32_t batch, hipStream_t stream) {
    if ((X == nullptr && rows > 0) || !dtype_ok(x_dtype)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(rows, cols, batch) || !matrix_ok(rows, cols, ldx, stride_x, batch)) return GALORE_ERR_SHAPE;
    const int e = check_mx(in, rows, cols, kBytes4, batch);
    if (e != GALORE_OK || rows == 0) return e;
    GALORE_TRY(launch_mx4_dequantize(matrix_of(in, batch), X, x_dtype == GALORE_BF16, ldx, stride_x, rows, cols, batch,
                                     stream));
    return GALORE_OK;
}

int galore_mx4_matmul(const galore_mx_t* a, const galore_mx_t* b, int64_t m, int64_t n, int64_t k, void* C,
                      int32_t c_dtype, int64_t ldc, int64_t stride_c, int32_t batch, hipStream_t stream) {
    if ((C == nullptr && m > 0) || !dtype_ok(c_dtype)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(m, n, batch) || k < 1 || k > kMaxSide) return GALORE_ERR_SHAPE;
    if (!matrix_ok(m, n, ldc, stride_c, batch)) return GALORE_ERR_SHAPE;
    int e = check_mx(a, m, k, kBytes4, batch);
    if (e == GALORE_OK) e = check_mx(b, n, k, kBytes4, batch);
    if (e != GALORE_OK || m == 0) return e;
    GALORE_TRY(launch_mx4_gemm(matrix_of(a, batch), matrix_of(b, batch), C, c_dtype == GALORE_BF16, ldc, stride_c, m, n, k,
                               batch, stream));
    return GALORE_OK;
}

// ---- the norms of a block -----------------------------------------------------

int galore_norm_block(const void* X, int64_t ldx, const void* Y, int64_t ldy, int32_t dtype, const float* w_post,
                      const float* w_pre, const void* gate, int64_t ldgate, int32_t gate_mode, float alpha, float eps,
                      int64_t tokens, int64_t d, void* H, int64_t ldh, void* Z, int64_t ldz, float* rstd,
                      const galore_mx_t* y8, const galore_mx_t* h8, const galore_mx_t* z8, hipStream_t stream) {
    if (tokens > 0 && (X == nullptr || Y == nullptr || H == nullptr || Z == nullptr || rstd == nullptr))
        return GALORE_ERR_INVALID_ARG;
    if (w_post == nullptr || w_pre == nullptr || !dtype_ok(dtype)) return GALORE_ERR_INVALID_ARG;
    if (gate_mode < GALORE_GATE_NONE || gate_mode > GALORE_GATE_TOKENS) return GALORE_ERR_INVALID_ARG;
    if (gate == nullptr && (gate_mode == GALORE_GATE_VECTOR || (gate_mode == GALORE_GATE_TOKENS && tokens > 0)))
        return GALORE_ERR_INVALID_ARG;
    if (!finite_f(alpha) || !finite_f(eps) || eps <= 0.0f) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, 1) || d > kNormMaxWidth) return GALORE_ERR_SHAPE;
    if (ldx < d || ldy < d || ldh < d || ldz < d || (gate_mode == GALORE_GATE_TOKENS && ldgate < d)) return GALORE_ERR_SHAPE;
    NormForwardArgs a{};
    const galore_mx_t* given[3] = {y8, h8, z8};
    MxMatrix* to[3] = {&a.y8, &a.h8, &a.z8};
    for (int i = 0; i < 3; ++i) {
        if (given[i] == nullptr) continue;
        const int e = check_mx(given[i], tokens, d, kBytes8, 1);
        if (e != GALORE_OK) return e;
        *to[i] = matrix_of(given[i], 1);
    }
    a.X = X;
    a.Y = Y;
    a.ldx = ldx;
    a.ldy = ldy;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.gate = gate;
    a.ldgate = ldgate;
    a.gate_mode = gate_mode;
    a.H = H;
    a.Z = Z;
    a.ldh = ldh;
    a.ldz = ldz;
    a.rstd = rstd;
    a.T = tokens;
    a.d = d;
    a.alpha = alpha;
    a.eps = eps;
    GALORE_TRY(launch_norm_forward(a, dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

size_t galore_norm_block_backward_workspace_size(int64_t tokens, int64_t d) {
    if (!sides_ok(tokens, d, 1) || d > kNormMaxWidth) return 0;
    return align_up(sizeof(float) * 2 * static_cast<size_t>(d) * norm_backward_groups(tokens, d));
}

int galore_norm_block_backward(const void* dZ, int64_t lddz, const void* dH, int64_t lddh, int32_t dtype, const void* H,
                               int64_t ldh, const void* Y, int64_t ldy, const galore_mx_t* h8, const galore_mx_t* y8,
                               const float* rstd, const float* w_post, const float* w_pre, const void* gate,
                               int64_t ldgate, int32_t gate_mode, float alpha, int64_t tokens, int64_t d, void* dX,
                               int64_t lddx, void* dY, int64_t lddy, void* dgate, int64_t lddgate, float* dw_post,
                               float* dw_pre, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const bool packed = h8 != nullptr;
    if (packed != (y8 != nullptr) || (packed && (H != nullptr || Y != nullptr))) return GALORE_ERR_INVALID_ARG;
    if (tokens > 0 && (dZ == nullptr || (!packed && (H == nullptr || Y == nullptr)) || rstd == nullptr || dX == nullptr ||
                       dY == nullptr))
        return GALORE_ERR_INVALID_ARG;
    if (w_post == nullptr || w_pre == nullptr || dw_post == nullptr || dw_pre == nullptr || !dtype_ok(dtype))
        return GALORE_ERR_INVALID_ARG;
    if (gate_mode < GALORE_GATE_NONE || gate_mode > GALORE_GATE_TOKENS || !finite_f(alpha)) return GALORE_ERR_INVALID_ARG;
    if ((gate == nullptr || dgate == nullptr) &&
        (gate_mode == GALORE_GATE_VECTOR || (gate_mode == GALORE_GATE_TOKENS && tokens > 0)))
        return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, 1) || d > kNormMaxWidth) return GALORE_ERR_SHAPE;
    if (lddz < d || (dH != nullptr && lddh < d) || (!packed && (ldh < d || ldy < d)) || lddx < d || lddy < d)
        return GALORE_ERR_SHAPE;
    if (gate_mode == GALORE_GATE_TOKENS && (ldgate < d || lddgate < d)) return GALORE_ERR_SHAPE;
    NormBackwardArgs a{};
    if (packed) {
        int e = check_mx(h8, tokens, d, kBytes8, 1);
        if (e == GALORE_OK) e = check_mx(y8, tokens, d, kBytes8, 1);
        if (e != GALORE_OK) return e;
        a.h8 = matrix_of(h8, 1);
        a.y8 = matrix_of(y8, 1);
    }
    const size_t need = galore_norm_block_backward_workspace_size(tokens, d);
    if (need > 0 && (workspace == nullptr || !is_aligned(workspace, kAlign) || workspace_bytes < need))
        return GALORE_ERR_WORKSPACE;
    a.dZ = dZ;
    a.dH = dH;
    a.lddz = lddz;
    a.lddh = lddh;
    a.H = H;
    a.Y = Y;
    a.ldh = ldh;
    a.ldy = ldy;
    a.rstd = rstd;
    a.w_post = w_post;
    a.w_pre = w_pre;
    a.gate = gate;
    a.ldgate = ldgate;
    a.gate_mode = gate_mode;
    a.dX = dX;
    a.dY = dY;
    a.dgate = dgate;
    a.lddx = lddx;
    a.lddy = lddy;
    a.lddgate = lddgate;
    a.dw_post = dw_post;
    a.dw_pre = dw_pre;
    a.part = static_cast<float*>(workspace);
    a.T = tokens;
    a.d = d;
    a.alpha = alpha;
    GALORE_TRY(launch_norm_backward(a, dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

}  // extern "C"
