// Dropout whose mask is a function of (seed, index, place) and is never stored: the
// backward pass is the same call on the incoming gradient.
//   Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011): key = seed, counter =
//   (column / 8, row, matrix, index), so that a value's bits depend on neither
//   strides nor tiles. 128 bits a counter, 16 for each of 8 columns: columns 2 i and
//   2 i + 1 have the halves of word i.
// A value is kept where its 16 bits are `cut` or more and scaled by 65536 / (65536 -
// cut), the inverse of the chance that is really taken, so that the mean is exact. A
// dropped value is replaced, not multiplied: what it held (NaN, Inf) does not come
// through.
//
// Bound by memory: a thread has eight values of a row, one counter and 16-byte accesses,
// and the counter's 20 products (32 bits, a quarter of the rate of others) are made while
// the loads are on their way. 16384 x 4096 bf16: 62 us (4.3 TB/s; one round of the ten,
// to see what they cost, 55), with a residual 72 (5.6), with its checkpoint 71 (4.8; 74
// through the caches), with both 83 (5.7). A fixed grid of 2048 or 4096 workgroups with the
// next row loaded ahead: 54 alone, but 75 with a residual and 69 to 75 with the checkpoint.
#include "mx.hpp"
#include "layers.hpp"

namespace galore {
namespace {

__device__ __forceinline__ u32x4 philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ k0;
        c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ k1;
        c1 = static_cast<uint32_t>(p1);
        c3 = static_cast<uint32_t>(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int64_t nb, int64_t groups, bool once) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x;
    if (g >= groups) return;   // groups is a multiple of 16 where codes are written: a quad leaves whole
    const int64_t b = blockIdx.z, e = 8 * g;
    const int d = static_cast<int>(a.cols);
    for (int64_t row = first_row(); row < a.rows; row += row_step()) {
        Eight<T> x, r;
        x.load(static_cast<const T*>(a.X) + b * a.strideX + row * a.ldx, e, d, once);
        if (a.R != nullptr) r.load(static_cast<const T*>(a.R) + b * a.strideR + row * a.ldr, e, d, once);
        const u32x4 bits = philox4x32_10(static_cast<uint32_t>(g), static_cast<uint32_t>(row), static_cast<uint32_t>(b),
                                         a.index, a.key0, a.key1);
        x.settle(e, d);
        if (a.R != nullptr) r.settle(e, d);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma clang fp contract(off)   // a product and a sum, each rounded: the codes are those of fp32 arithmetic as written
            const uint32_t u = i & 1 ? bits[i >> 1] >> 16 : bits[i >> 1] & 0xffffu;
            y[i] = u >= a.cut ? x[i] * a.scale : 0.0f;
            if (a.R != nullptr) y[i] = y[i] + r[i];
        }
        if (e < d) store8(static_cast<T*>(a.Y) + b * a.strideY + row * a.ldy + e, d - e, y, once);
        if (a.y8.codes != nullptr) put_codes(a.y8.from(b), row, g, nb, y);
    }
}

template <typename T>
hipError_t dropout(const DropoutArgs& a, int batch, hipStream_t stream) {
    const int64_t nb = mx_blocks(a.cols), groups = a.y8.codes != nullptr ? 4 * mx_scale_bytes(a.cols) : (a.cols + 7) / 8;
    // past the caches as the backward norms do: bf16 rows on 16 bytes
    const bool once = sizeof(T) == 2 && rows_on_16(static_cast<const T*>(a.X), a.ldx, a.strideX, batch) &&
                      rows_on_16(static_cast<const T*>(a.Y), a.ldy, a.strideY, batch) &&
                      (a.R == nullptr || rows_on_16(static_cast<const T*>(a.R), a.ldr, a.strideR, batch));
    const RowGrid g = row_grid(a.rows, groups, batch);
    hipLaunchKernelGGL(dropout_kernel<T>, g.grid, g.block, 0, stream, a, nb, groups, once);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, bool bf16, int batch, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? dropout<bf16_t>(a, batch, stream) : dropout<float>(a, batch, stream);
}

}  // namespace galore
