// Launchers of the training operators (8-bit checkpoints, 4-bit products, the
// norms of a block). All return the hipError_t of the launch; arguments are
// checked by the entry points (training.hip).
#pragma once

#include "mx.hpp"

namespace galore {

// checkpoint.hip
hipError_t launch_pack(const void* X, bool bf16, int64_t ldx, int64_t strideX, const MxMatrix& q, int64_t rows,
                       int64_t cols, int batch, hipStream_t stream);
hipError_t launch_unpack(const MxMatrix& q, void* X, bool bf16, int64_t ldx, int64_t strideX, int64_t rows, int64_t cols,
                         int batch, hipStream_t stream);

// mx4.hip: q (rows of X) or qt (columns of X) may be null, not both
hipError_t launch_mx4_quantize(const void* X, bool bf16, int64_t ldx, int64_t strideX, const MxMatrix* q, const MxMatrix* qt,
                               int64_t rows, int64_t cols, int batch, hipStream_t stream);
hipError_t launch_mx4_dequantize(const MxMatrix& q, void* X, bool bf16, int64_t ldx, int64_t strideX, int64_t rows,
                                 int64_t cols, int batch, hipStream_t stream);

// mx4_gemm.hip: C (M x N) = A (M x K) B^T (N x K)
hipError_t launch_mx4_gemm(const MxMatrix& A, const MxMatrix& B, void* C, bool bf16, int64_t ldc, int64_t strideC, int64_t M,
                           int64_t N, int64_t K, int batch, hipStream_t stream);

// weight_grad.hip: G (m x n) = dY^T X (+ G), dY T x m, X a T x n checkpoint. part: room for the
// partial sums of a split over T (weight_grad_splits of them, where above 1), fp32, m x n each.
struct WeightGradArgs {
    const void* dY;
    bool dy_bf16;
    int64_t ldy, strideY;
    MxMatrix X;
    void* G;
    bool g_bf16;
    int64_t ldg, strideG;
    int64_t T, m, n;
    bool accumulate;
    float* part;                 // null: the tokens are not split
};
int weight_grad_splits(int64_t T, int64_t m, int64_t n, int64_t batch);
hipError_t launch_weight_grad(const WeightGradArgs& a, int batch, hipStream_t stream);

// norm_block.hip
enum GateMode { kGateNone = 0, kGateVector = 1, kGateTokens = 2 };
struct NormForwardArgs {
    const void *X, *Y;
    int64_t ldx, ldy;
    const float *w_post, *w_pre;
    const void* gate;
    int64_t ldgate;
    int gate_mode;
    void *H, *Z;
    int64_t ldh, ldz;
    float* rstd;                 // T x 2
    MxMatrix y8, h8, z8;         // codes null: not written
    int64_t T, d;
    float alpha, eps;
};
struct NormBackwardArgs {
    const void *dZ, *dH;         // dH may be null
    int64_t lddz, lddh;
    const void *H, *Y;           // plain, or null with the checkpoints in h8 and y8
    int64_t ldh, ldy;
    MxMatrix h8, y8;
    const float* rstd;
    const float *w_post, *w_pre;
    const void* gate;
    int64_t ldgate;
    int gate_mode;
    void *dX, *dY, *dgate;       // dgate: fp32 d (vector), T x d (tokens), or null
    int64_t lddx, lddy, lddgate;
    float *dw_post, *dw_pre;
    float* part;                 // norm_backward_groups(T, d) x 2 x d
    int64_t T, d;
    float alpha;
    bool once;                   // set by the launcher: bf16 rows on 16 bytes, moved past the caches
};
constexpr int64_t kNormMaxWidth = 16384;
int64_t norm_backward_groups(int64_t T, int64_t d);
hipError_t launch_norm_forward(const NormForwardArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_norm_backward(const NormBackwardArgs& a, bool bf16, hipStream_t stream);

}  // namespace galore
