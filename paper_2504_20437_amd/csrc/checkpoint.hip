// Activations as 8-bit checkpoints: the forward pass stores a block's input in
// 8.25 bits a value and the backward pass reads it (weight_grad.hip,
// norm_block.hip) or has it decoded here.
//
// Integer codes with a power-of-two scale for each 32 values of a token: for
// values spread like a normal distribution the error is about 0.9% of their
// standard deviation, a third of what eight floating bits (E4M3) leave, and a
// decoded value is exact in bfloat16, so that the weight gradient runs on the
// bf16 matrix cores with no second rounding.
//
// Both kernels are bound by memory: one read and one write of every value, a
// thread's eight values in 16-byte accesses, four lanes to a block, whose
// maximum they exchange by cross-lane moves. 8192 x 4096 bf16: pack 17.5 us (5.8
// TB/s), unpack 16.6 (6.1); rows of 5461, which start on any element: 23.8 (5.7) and
// 23.6 (5.8). A plain copy reaches 6.7.
#include "mx.hpp"
#include "training.hpp"

namespace galore {
namespace {

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* Xb, int64_t ldx, int64_t strideX, MxMatrix q, int64_t rows,
                                                   int64_t cols, int64_t nb, int64_t groups) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x;
    if (g >= groups) return;   // groups is a multiple of 16: a quad leaves whole
    const int64_t b = blockIdx.z;
    for (int64_t row = first_row(); row < rows; row += row_step()) {
        float x[8];
        load8(Xb + b * strideX + row * ldx, 8 * g, cols, x);
        int scale;
        const u32x2 w = mx8_encode_quad(x, scale);
        if (g < 4 * nb) *reinterpret_cast<u32x2*>(q.codes + b * q.stride_q + row * q.ldq + 8 * g) = w;
        if ((g & 3) == 0) q.scales[b * q.stride_s + row * q.lds + (g >> 2)] = static_cast<uint8_t>(g < 4 * nb ? scale : 0);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(MxMatrix q, T* Xb, int64_t ldx, int64_t strideX, int64_t rows,
                                                     int64_t cols, int64_t groups) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x;
    if (g >= groups) return;
    const int64_t b = blockIdx.z;
    for (int64_t row = first_row(); row < rows; row += row_step()) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(q.codes + b * q.stride_q + row * q.ldq + 8 * g);
        float x[8];
        mx8_decode8(w, mx_unit<133>(q.scales[b * q.stride_s + row * q.lds + (g >> 2)]), x);
        store8(Xb + b * strideX + row * ldx + 8 * g, cols - 8 * g, x);
    }
}

}  // namespace

hipError_t launch_pack(const void* X, bool bf16, int64_t ldx, int64_t strideX, const MxMatrix& q, int64_t rows,
                       int64_t cols, int batch, hipStream_t stream) {
    const int64_t nb = mx_blocks(cols), groups = 4 * mx_scale_bytes(cols);
    const RowGrid g = row_grid(rows, groups, batch);
    if (bf16)
        hipLaunchKernelGGL(pack_kernel<bf16_t>, g.grid, g.block, 0, stream, static_cast<const bf16_t*>(X), ldx, strideX, q,
                           rows, cols, nb, groups);
    else
        hipLaunchKernelGGL(pack_kernel<float>, g.grid, g.block, 0, stream, static_cast<const float*>(X), ldx, strideX, q,
                           rows, cols, nb, groups);
    return hipGetLastError();
}

hipError_t launch_unpack(const MxMatrix& q, void* X, bool bf16, int64_t ldx, int64_t strideX, int64_t rows, int64_t cols,
                         int batch, hipStream_t stream) {
    const int64_t groups = (cols + 7) / 8;
    const RowGrid g = row_grid(rows, groups, batch);
    if (bf16)
        hipLaunchKernelGGL(unpack_kernel<bf16_t>, g.grid, g.block, 0, stream, q, static_cast<bf16_t*>(X), ldx, strideX,
                           rows, cols, groups);
    else
        hipLaunchKernelGGL(unpack_kernel<float>, g.grid, g.block, 0, stream, q, static_cast<float*>(X), ldx, strideX, rows,
                           cols, groups);
    return hipGetLastError();
}

}  // namespace galore
