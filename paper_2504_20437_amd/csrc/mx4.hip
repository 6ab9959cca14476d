// Microscaled 4-bit floating point: a matrix quantised along its rows, along its
// columns, or both in one read, and read back.
//
// A product contracts over the last axis of both operands (mx4_gemm.hip), and
// the scale of a block belongs to one term of that sum: the forward product of a
// weight takes blocks along its rows, the backward one blocks along its columns,
// stored as the rows of the transpose.
//
// Bound by memory. Along rows a thread encodes eight values, four lanes to a
// block. Along columns a workgroup holds a tile of 128 rows of 256 bytes in LDS and a
// thread takes four bytes of columns of one block of 32 rows. 8192 x 4096 bf16: rows 15.1 us
// (5.6 TB/s), both 20.7 (5.0), read back 14.8 (5.7); 8192 x 5461: 22.5, 27.4, 21.2;
// fp32: 22.2 (6.9), 30.5 (5.6); both of 2048 x 5461 12.5, with 128 columns a tile 16.5.
#include "mx.hpp"
#include "training.hpp"

namespace galore {
namespace {

// eight codes and the block's scale byte, the block being this lane's quad
__device__ __forceinline__ uint32_t encode_quad(const Eight<float>& x, int& scale) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x.v[i]));
    scale = mx4_scale(quad_max(m));
    return scale == kMxNan ? 0u : mx4_encode8(x.v, mx4_unit(scale));
}
__device__ __forceinline__ uint32_t encode_quad(const Eight<bf16_t>& x, int& scale) {
    uint32_t m = 0;   // two values a word
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max_halves(m, x.w[i] & 0x7fff7fffu);
    scale = mx4_scale(quad_max(max(m << 16, m & 0xffff0000u)));
    return scale == kMxNan ? 0u : mx4_encode8(x.w[0], x.w[1], x.w[2], x.w[3], mx4_unit(scale));
}

template <typename T>
__global__ __launch_bounds__(256) void mx4_rows_kernel(const T* Xb, int64_t ldx, int64_t strideX, MxMatrix q, int64_t rows,
                                                       int64_t cols, int64_t nb, int64_t groups) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x;
    if (g >= groups) return;   // groups is a multiple of 16: a quad leaves whole
    const int64_t b = blockIdx.z;
    for (int64_t row = first_row(); row < rows; row += row_step()) {
        Eight<T> x;
        x.load(Xb + b * strideX + row * ldx, 8 * g, cols);
        x.settle(8 * g, cols);
        int scale;
        const uint32_t w = encode_quad(x, scale);
        if (g < 4 * nb) *reinterpret_cast<uint32_t*>(q.codes + b * q.stride_q + row * q.ldq + 4 * g) = w;
        if ((g & 3) == 0) q.scales[b * q.stride_s + row * q.lds + (g >> 2)] = static_cast<uint8_t>(g < 4 * nb ? scale : 0);
    }
}

__device__ __forceinline__ void lds_put(void* p, const Eight<float>& x) {
    static_cast<f32x4*>(p)[0] = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    static_cast<f32x4*>(p)[1] = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
}
__device__ __forceinline__ void lds_put(void* p, const Eight<bf16_t>& x) {
    *static_cast<u32x4*>(p) = x.w;
}

// A block of 32 rows in four bytes of columns, encoded column by column
template <typename T>
struct Columns;
template <>
struct Columns<float> {
    static constexpr int kCols = 1;
    float v[32];
    uint32_t m = 0;             // bits of the largest magnitude
    __device__ __forceinline__ void read(const unsigned char* p, int i) {
        v[i] = *reinterpret_cast<const float*>(p);
        m = max(m, abs_bits(v[i]));
    }
    __device__ __forceinline__ uint32_t largest(int) const { return m; }
    __device__ __forceinline__ uint32_t codes(int, int k, float unit) const {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[8 * k + i];
        return mx4_encode8(x, unit);
    }
};
template <>
struct Columns<bf16_t> {
    static constexpr int kCols = 2;
    uint32_t v[32];             // a row's two columns
    uint32_t m = 0;
    __device__ __forceinline__ void read(const unsigned char* p, int i) {
        v[i] = *reinterpret_cast<const uint32_t*>(p);
        m = max_halves(m, v[i] & 0x7fff7fffu);
    }
    __device__ __forceinline__ uint32_t largest(int j) const { return j ? m & 0xffff0000u : m << 16; }
    __device__ __forceinline__ uint32_t codes(int j, int k, float unit) const {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)   // rows 2 i and 2 i + 1 of column j
            w[i] = __builtin_amdgcn_perm(v[8 * k + 2 * i + 1], v[8 * k + 2 * i], j ? 0x07060302u : 0x05040100u);
        return mx4_encode8(w[0], w[1], w[2], w[3], unit);
    }
};

constexpr int MT = 128;         // rows of a tile
constexpr int kPitch = 256;     // bytes of a tile's row

// One tile: its values to LDS, encoded along the rows on the way if ROWS, then
// along the columns. A block of 32 rows starts 64 bytes further than the pitch
// says, so that the four row blocks that the lanes of a quad read lie on
// different banks. 128 columns of bf16, 64 of fp32: four workgroups to a CU.
template <typename T, bool ROWS>
__global__ __launch_bounds__(256) void mx4_tile_kernel(const T* Xb, int64_t ldx, int64_t strideX, MxMatrix q, MxMatrix qt,
                                                       int64_t rows, int64_t cols, unsigned tiles_c, int once) {
    constexpr int MC = kPitch / sizeof(T), kLanes = MC / 8;   // columns; threads along a row
    __shared__ __attribute__((aligned(16))) unsigned char sm[MT * kPitch + 4 * 64];
    const int64_t b = blockIdx.z;
    const T* X = Xb + b * strideX;
    const unsigned id = static_cast<unsigned>(xcd_logical_id(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x)));
    const int64_t row0 = static_cast<int64_t>(id / tiles_c) * MT, col0 = static_cast<int64_t>(id % tiles_c) * MC;
    const int tid = threadIdx.x;
    const int64_t nb = mx_blocks(cols);
#pragma unroll
    for (int i = 0; i < MT * kLanes / 256; ++i) {
        const int r = 256 / kLanes * i + tid / kLanes, c = 8 * (tid % kLanes);
        const int64_t row = row0 + r, col = col0 + c;
        Eight<T> x;
        x.load(X + row * ldx, row < rows ? col : cols, cols, once != 0);
        x.settle(col, cols);
        lds_put(sm + r * kPitch + (r >> 5) * 64 + c * sizeof(T), x);
        if (ROWS) {
            int scale;
            const uint32_t w = encode_quad(x, scale);
            if (row < rows) {
                const int64_t blk = col / kMxBlock;
                if (blk < nb) *reinterpret_cast<uint32_t*>(q.codes + b * q.stride_q + row * q.ldq + col / 2) = w;
                if ((tid & 3) == 0)
                    q.scales[b * q.stride_s + row * q.lds + blk] = static_cast<uint8_t>(blk < nb ? scale : 0);
            }
        }
    }
    __syncthreads();
    const int rb = tid & 3, c = Columns<T>::kCols * (tid >> 2);
    Columns<T> v;
#pragma unroll
    for (int i = 0; i < 32; ++i) v.read(sm + (32 * rb + i) * kPitch + rb * 64 + c * sizeof(T), i);
    const int64_t blk = row0 / kMxBlock + rb;
    const bool inside = blk < mx_blocks(rows);
#pragma unroll
    for (int j = 0; j < Columns<T>::kCols; ++j) {
        const int64_t col = col0 + c + j;
        if (col >= cols) break;
        const int scale = mx4_scale(v.largest(j));
        u32x4 w = {0u, 0u, 0u, 0u};
        if (scale != kMxNan) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = v.codes(j, k, mx4_unit(scale));
        }
        if (inside) *reinterpret_cast<u32x4*>(qt.codes + b * qt.stride_q + col * qt.ldq + 16 * blk) = w;
        qt.scales[b * qt.stride_s + col * qt.lds + blk] = static_cast<uint8_t>(inside ? scale : 0);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void mx4_decode_kernel(MxMatrix q, T* Xb, int64_t ldx, int64_t strideX, int64_t rows,
                                                         int64_t cols, int64_t groups) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x;
    if (g >= groups) return;
    const int64_t b = blockIdx.z;
    for (int64_t row = first_row(); row < rows; row += row_step()) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(q.codes + b * q.stride_q + row * q.ldq + 4 * g);
        const float unit = mx_unit<127>(q.scales[b * q.stride_s + row * q.lds + (g >> 2)]);
        float x[8];
        const auto put = [&](int i, bf16x2_t v) {   // the code's own value is exact in bf16
            const uint32_t u = __builtin_bit_cast(uint32_t, v);
            x[i] = __uint_as_float(u << 16) * unit;
            x[i + 1] = __uint_as_float(u & 0xffff0000u) * unit;
        };
        put(0, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
        put(2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
        put(4, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
        put(6, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
        store8(Xb + b * strideX + row * ldx + 8 * g, cols - 8 * g, x);
    }
}

template <typename T>
hipError_t quantize(const T* X, int64_t ldx, int64_t strideX, const MxMatrix* q, const MxMatrix* qt, int64_t rows,
                    int64_t cols, int batch, hipStream_t stream) {
    if (qt == nullptr) {
        const int64_t groups = 4 * mx_scale_bytes(cols);
        const RowGrid g = row_grid(rows, groups, batch);
        hipLaunchKernelGGL(mx4_rows_kernel<T>, g.grid, g.block, 0, stream, X, ldx, strideX, *q, rows, cols, mx_blocks(cols),
                           groups);
        return hipGetLastError();
    }
    // whole groups of four blocks along a row, whose scales' padding the last tile writes
    const int64_t tr = (rows + MT - 1) / MT, tc = mx_scale_bytes(cols) * kMxBlock / (kPitch / static_cast<int>(sizeof(T)));
    if (tr * tc >= 1 << 24) return hipErrorInvalidValue;   // work-items along x fit 32 bits
    const dim3 grid(static_cast<unsigned>(tr * tc), 1, static_cast<unsigned>(batch));
    const int once = rows_on_16(X, ldx, strideX, batch) ? 1 : 0;
    if (q != nullptr)
        hipLaunchKernelGGL((mx4_tile_kernel<T, true>), grid, dim3(256), 0, stream, X, ldx, strideX, *q, *qt, rows, cols,
                           static_cast<unsigned>(tc), once);
    else
        hipLaunchKernelGGL((mx4_tile_kernel<T, false>), grid, dim3(256), 0, stream, X, ldx, strideX, MxMatrix{}, *qt, rows,
                           cols, static_cast<unsigned>(tc), once);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_quantize(const void* X, bool bf16, int64_t ldx, int64_t strideX, const MxMatrix* q, const MxMatrix* qt,
                               int64_t rows, int64_t cols, int batch, hipStream_t stream) {
    return bf16 ? quantize(static_cast<const bf16_t*>(X), ldx, strideX, q, qt, rows, cols, batch, stream)
                : quantize(static_cast<const float*>(X), ldx, strideX, q, qt, rows, cols, batch, stream);
}

hipError_t launch_mx4_dequantize(const MxMatrix& q, void* X, bool bf16, int64_t ldx, int64_t strideX, int64_t rows,
                                 int64_t cols, int batch, hipStream_t stream) {
    const int64_t groups = (cols + 7) / 8;
    const RowGrid g = row_grid(rows, groups, batch);
    if (bf16)
        hipLaunchKernelGGL(mx4_decode_kernel<bf16_t>, g.grid, g.block, 0, stream, q, static_cast<bf16_t*>(X), ldx, strideX,
                           rows, cols, groups);
    else
        hipLaunchKernelGGL(mx4_decode_kernel<float>, g.grid, g.block, 0, stream, q, static_cast<float*>(X), ldx, strideX,
                           rows, cols, groups);
    return hipGetLastError();
}

}  // namespace galore
