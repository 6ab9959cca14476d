// The norms after and before a block, with the block's gate and residual scale
// between them, in one pass over the token's row (d values):
//   u = y rstd(y),  h = x + alpha gate u w_post,  z = h rstd(h) w_pre,
//   rstd(v) = (mean v^2 + eps)^(-1/2)
// and the 8-bit checkpoints of y, h and z if they are wanted. Backward, with
// n = h rstd(h) and a = dz w_pre:
//   dx = dh + rstd(h) (a - n mean(a n))          (dx is also the gradient of h)
//   g = alpha dx gate w_post;  dy = rstd(y) (g - u mean(g u))
//   dw_pre = sum_t dz n;  dw_post = sum_t alpha dx gate u;  dgate = alpha dx u w_post
//
// Bound by memory: each activation is read once and stays in registers. A row
// belongs to W waves (one up to d = 1024, so that no barrier is needed, then 4, 8
// or 16), a workgroup walks over rows with the weights in registers, and the sums
// over tokens stay in the registers of the thread that owns the column until the
// end; a second launch adds the workgroups' sums in order. All sums in fp32. Forward
// 8192 x 2736 bf16 34 us (5.3 TB/s), 4096 x 2048 with its three checkpoints 20.3 (4.6),
// one token of 4096 3.9; backward 8192 x 4096 bf16 73 (5.5), on checkpoints 74 (4.5),
// fp32 154 (5.2), 1003 x 1024 fp32 with token gates 10.6 and 4.9 for the sums. Far from
// their bytes: rows past d = 8192 (2048 x 16384 bf16 118 us, 3.4 TB/s: registers spill),
// widths between the shapes (8192 x 2736 71 us, 3.8: a third of the threads' second groups
// hold anything) and odd ones (2731: 96, 2.8: through the caches too).
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "dispatch.hpp"
#include "training.hpp"

namespace galore {
namespace {

// sum over the W waves of a row; `red` alternates between two calls
template <int W>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += red[i];
    }
    return v;
}

template <int W, int NC>
struct RowShape {
    static constexpr int kRows = W >= 4 ? 1 : 4 / W;          // rows of a workgroup
    static constexpr int kThreads = 64 * W * kRows;
    static constexpr int kGroups = 64 * W;                    // groups of 8 values between a thread's own
};

// eight entries of a vector, ones where p is null
__device__ __forceinline__ void load_group(const float* p, int e, int d, float (&v)[8]) {
    if (p != nullptr) {
        load8(p, e, d, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    }
}
// the vectors of a thread's columns
template <int NC, int STEP>
__device__ __forceinline__ void load_vector(const float* p, int64_t d, int g0, float (&v)[NC][8]) {
#pragma unroll
    for (int c = 0; c < NC; ++c) load_group(p, 8 * (g0 + c * STEP), d, v[c]);
}

template <typename T, int W, int NC>
__global__ __launch_bounds__((RowShape<W, NC>::kThreads)) void norm_forward_kernel(NormForwardArgs a) {
    using S = RowShape<W, NC>;
    __shared__ float red[2][W];
    const int wave = (threadIdx.x >> 6) % W;
    const int g0 = threadIdx.x % S::kGroups;
    const int64_t d = a.d, nb = mx_blocks(d);
    const float inv_d = 1.0f / static_cast<float>(d);
    float wo[NC][8], wp[NC][8];
    load_vector<NC, S::kGroups>(a.w_post, d, g0, wo);
    load_vector<NC, S::kGroups>(a.w_pre, d, g0, wp);
    if (a.gate_mode == kGateVector) {
        float gv[NC][8];
        load_vector<NC, S::kGroups>(static_cast<const float*>(a.gate), d, g0, gv);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) wo[c][i] *= gv[c][i];
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * S::kRows;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * S::kRows + threadIdx.x / S::kGroups; row < a.T; row += step) {
        Eight<T> xs[NC], ys[NC];
        float x[NC][8], y[NC][8];
        float sy = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
            ys[c].load(static_cast<const T*>(a.Y) + row * a.ldy, e, d);
            xs[c].load(static_cast<const T*>(a.X) + row * a.ldx, e, d);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
            ys[c].settle(e, d);
            xs[c].settle(e, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[c][i] = ys[c][i];
                x[c][i] = xs[c][i];
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sy += y[c][i] * y[c][i];
        const float ry = 1.0f / sqrtf(row_sum<W>(sy, red[0], wave) * inv_d + a.eps);
        if (a.y8.codes != nullptr) {
#pragma unroll
            for (int c = 0; c < NC; ++c) put_codes(a.y8, row, g0 + c * S::kGroups, nb, y[c]);
        }
        const float s = a.alpha * ry;
        float sh = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
            float gt[8];
            if (a.gate_mode == kGateTokens) load8(static_cast<const T*>(a.gate) + row * a.ldgate, e, d, gt);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = y[c][i] * s * wo[c][i];
                x[c][i] += a.gate_mode == kGateTokens ? u * gt[i] : u;
                sh += x[c][i] * x[c][i];
            }
            store8(static_cast<T*>(a.H) + row * a.ldh + e, d - e, x[c]);
            if (a.h8.codes != nullptr) put_codes(a.h8, row, g0 + c * S::kGroups, nb, x[c]);
        }
        const float rh = 1.0f / sqrtf(row_sum<W>(sh, red[1], wave) * inv_d + a.eps);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[c][i] = x[c][i] * rh * wp[c][i];
            store8(static_cast<T*>(a.Z) + row * a.ldz + e, d - e, x[c]);
            if (a.z8.codes != nullptr) put_codes(a.z8, row, g0 + c * S::kGroups, nb, x[c]);
        }
        if (g0 == 0) {
            a.rstd[2 * row] = ry;
            a.rstd[2 * row + 1] = rh;
        }
    }
}

struct Codes8 {
    u32x2 w;
    int scale;
    __device__ __forceinline__ void load(const MxMatrix& q, int64_t row, int64_t g, bool inside) {
        w = u32x2{0u, 0u};   // past the row: zeros (its last block holds them where it ends inside)
        scale = 0;
        if (inside) {
            w = get_vector<u32x2>(reinterpret_cast<const u32x2*>(q.codes + row * q.ldq + 8 * g), true);
            scale = q.scales[row * q.lds + (g >> 2)];
        }
    }
};

// what a row's backward pass reads, of one thread
template <typename T, int NC, bool PACKED, bool TOKENS>
struct BackwardRow {
    float ry, rh;
    Eight<T> dz[NC], dh[NC];
    Eight<T> h[PACKED ? 1 : NC], y[PACKED ? 1 : NC], gate[TOKENS ? NC : 1];
    Codes8 h8[PACKED ? NC : 1], y8[PACKED ? NC : 1];
    __device__ __forceinline__ void load(const NormBackwardArgs& a, int64_t row, int g0, int step) {
        ry = a.rstd[2 * row];
        rh = a.rstd[2 * row + 1];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t g = g0 + static_cast<int64_t>(c) * step, e = 8 * g;
            dz[c].load(static_cast<const T*>(a.dZ) + row * a.lddz, e, a.d, a.once);
            if (a.dH != nullptr) dh[c].load(static_cast<const T*>(a.dH) + row * a.lddh, e, a.d, a.once);
            else dh[c].clear();
            if constexpr (PACKED) {
                h8[c].load(a.h8, row, g, e < a.d);
                y8[c].load(a.y8, row, g, e < a.d);
            } else {
                h[c].load(static_cast<const T*>(a.H) + row * a.ldh, e, a.d, a.once);
                y[c].load(static_cast<const T*>(a.Y) + row * a.ldy, e, a.d, a.once);
            }
            if constexpr (TOKENS) gate[c].load(static_cast<const T*>(a.gate) + row * a.ldgate, e, a.d, a.once);
        }
    }
    __device__ __forceinline__ void settle(int64_t d, int g0, int step) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * step);
            dz[c].settle(e, d);
            dh[c].settle(e, d);
            if constexpr (!PACKED) {
                h[c].settle(e, d);
                y[c].settle(e, d);
            }
            if constexpr (TOKENS) gate[c].settle(e, d);
        }
    }
};

// The next row's values are loaded while a row is worked on: its two sums over the
// row stand in a chain, and without that the memory would wait for them (8192 x 4096
// bf16, before its accesses went past the caches: 99.8 us without, 83.2 with). Where the
// registers of 1024 or, in fp32 with a gate for each token, of 512 threads do not hold
// that, it is left out, and past d = 8192 the vectors are read again for each row too,
// from the caches: 2048 x 16384 bf16 301 us with all of it held and 118 so; 4096 x 8192
// fp32 with token gates 295 and 214. Past d = 8192 that spills less, not nothing: 1024
// threads have 128 registers each, and 22 (fp32, on checkpoints) to 81 (fp32, token
// gates) more go through scratch.
template <typename T, int W, int NC, bool PACKED, bool TOKENS>
__global__ __launch_bounds__((RowShape<W, NC>::kThreads)) void norm_backward_kernel(NormBackwardArgs a) {
    using S = RowShape<W, NC>;
    constexpr int R = S::kRows;
    constexpr int kCols = 8 * NC * S::kGroups;
    constexpr bool kHold = W < 16;
    constexpr bool kAhead = W < 16 && !(W == 8 && TOKENS && std::is_same<T, float>::value);
    __shared__ float red[2][W];
    __shared__ float join[R > 1 ? R : 1][R > 1 ? kCols : 1];
    const int wave = (threadIdx.x >> 6) % W;
    const int g0 = threadIdx.x % S::kGroups, rg = threadIdx.x / S::kGroups;
    const int64_t d = a.d;
    const float inv_d = 1.0f / static_cast<float>(d);
    float wo[NC][8], wp[NC][8], sum_pre[NC][8], sum_post[NC][8];
    auto pre = [&](int c, float (&w)[8]) { load_group(a.w_pre, 8 * (g0 + c * S::kGroups), d, w); };
    auto post = [&](int c, float (&w)[8]) {
        const int e = 8 * (g0 + c * S::kGroups);
        load_group(a.w_post, e, d, w);
        if (a.gate_mode != kGateVector) return;
        float gv[8];
        load_group(static_cast<const float*>(a.gate), e, d, gv);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] *= gv[i];
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_pre[c][i] = sum_post[c][i] = 0.0f;
        if (kHold) {
            pre(c, wp[c]);
            post(c, wo[c]);
        }
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * R;
    int64_t row = static_cast<int64_t>(blockIdx.x) * R + rg;
    BackwardRow<T, NC, PACKED, TOKENS> next;
    if (kAhead && row < a.T) next.load(a, row, g0, S::kGroups);
    for (; row < a.T; row += step) {
        BackwardRow<T, NC, PACKED, TOKENS> r;
        if (kAhead) r = next;
        else r.load(a, row, g0, S::kGroups);
        r.settle(d, g0, S::kGroups);
        if (kAhead && row + step < a.T) next.load(a, row + step, g0, S::kGroups);
        float p[NC][8], n[NC][8], u[NC][8];
        float s1 = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (PACKED) {
                mx8_decode8(r.h8[c].w, mx_unit<133>(r.h8[c].scale) * r.rh, n[c]);   // a power of two times rstd
                mx8_decode8(r.y8[c].w, mx_unit<133>(r.y8[c].scale) * r.ry, u[c]);
            }
            if (!kHold) pre(c, wp[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (!PACKED) {
                    n[c][i] = r.h[c][i] * r.rh;
                    u[c][i] = r.y[c][i] * r.ry;
                }
                const float z = r.dz[c][i];
                sum_pre[c][i] += z * n[c][i];
                p[c][i] = z * wp[c][i];
                s1 += p[c][i] * n[c][i];
            }
        }
        const float m1 = row_sum<W>(s1, red[0], wave) * inv_d;
        float s2 = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
            float dx[8], dg[8];
            if (!kHold) post(c, wo[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dx[i] = r.dh[c][i] + r.rh * (p[c][i] - n[c][i] * m1);
                const float b = a.alpha * dx[i], bu = b * u[c][i];
                float g = b * wo[c][i];
                if constexpr (TOKENS) {
                    dg[i] = bu * wo[c][i];
                    sum_post[c][i] += bu * r.gate[c][i];
                    g *= r.gate[c][i];
                } else {
                    sum_post[c][i] += bu;
                }
                p[c][i] = g;
                s2 += g * u[c][i];
            }
            store8(static_cast<T*>(a.dX) + row * a.lddx + e, d - e, dx, a.once);
            if constexpr (TOKENS) store8(static_cast<T*>(a.dgate) + row * a.lddgate + e, d - e, dg, a.once);
        }
        const float m2 = row_sum<W>(s2, red[1], wave) * inv_d;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[c][i] = r.ry * (p[c][i] - u[c][i] * m2);
            store8(static_cast<T*>(a.dY) + row * a.lddy + e, d - e, p[c], a.once);
        }
    }
    // this workgroup's sums over its tokens: its rows joined in order, then to memory
    float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * d;
    if constexpr (R == 1) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int64_t e = 8 * (g0 + static_cast<int64_t>(c) * S::kGroups);
            store8(part + e, d - e, sum_pre[c]);
            store8(part + d + e, d - e, sum_post[c]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) join[rg][8 * (g0 + c * S::kGroups) + i] = k ? sum_post[c][i] : sum_pre[c][i];
            __syncthreads();
            for (int64_t e = threadIdx.x; e < d; e += S::kThreads) {
                float s = join[0][e];
#pragma unroll
                for (int r = 1; r < R; ++r) s += join[r][e];
                part[k * d + e] = s;
            }
        }
    }
}

// dw_pre, dw_post and a gate vector's gradient from the workgroups' sums: 32
// columns a workgroup, 32 slices of the groups joined in LDS in order
__global__ __launch_bounds__(1024) void norm_join_kernel(NormBackwardArgs a, int64_t groups) {
    __shared__ float red[32][33];
    const int c = threadIdx.x & 31, sl = threadIdx.x >> 5;
    const int64_t col = static_cast<int64_t>(blockIdx.x) * 32 + c;   // of 2 d: dw_pre, then the sum for dw_post and dgate
    float s = 0.0f;
    if (col < 2 * a.d) {
#pragma unroll 8
        for (int64_t g = sl; g < groups; g += 32) s += a.part[g * 2 * a.d + col];
    }
    red[sl][c] = s;
    __syncthreads();
    if (sl != 0 || col >= 2 * a.d) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) s += red[i][c];
    if (col < a.d) {
        a.dw_pre[col] = s;
        return;
    }
    const int64_t e = col - a.d;
    if (a.gate_mode == kGateVector) {
        a.dw_post[e] = s * static_cast<const float*>(a.gate)[e];
        if (a.dgate != nullptr) static_cast<float*>(a.dgate)[e] = s * a.w_post[e];
    } else {
        a.dw_post[e] = s;
    }
}

// f(waves, groups) for the shape that holds rows of d values
template <typename F>
hipError_t with_shape(int64_t d, F f) {
    if (d <= 512) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    if (d <= 1024) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    if (d <= 2048) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    if (d <= 4096) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    if (d <= 8192) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
}

template <typename T>
hipError_t forward(const NormForwardArgs& a, hipStream_t stream) {
    return with_shape(a.d, [&](auto w, auto nc) {
        using S = RowShape<decltype(w)::value, decltype(nc)::value>;
        const int64_t groups = std::min<int64_t>((a.T + S::kRows - 1) / S::kRows, 256 * 2048 / S::kThreads);
        hipLaunchKernelGGL((norm_forward_kernel<T, decltype(w)::value, decltype(nc)::value>),
                           dim3(static_cast<unsigned>(groups)), dim3(S::kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

template <typename T, bool PACKED, bool TOKENS>
hipError_t backward_rows(const NormBackwardArgs& a, int64_t groups, hipStream_t stream) {
    return with_shape(a.d, [&](auto w, auto nc) {
        using S = RowShape<decltype(w)::value, decltype(nc)::value>;
        hipLaunchKernelGGL((norm_backward_kernel<T, decltype(w)::value, decltype(nc)::value, PACKED, TOKENS>),
                           dim3(static_cast<unsigned>(groups)), dim3(S::kThreads), 0, stream, a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward(NormBackwardArgs a, hipStream_t stream) {
    const auto aligned = [](const void* p, int64_t ld) { return p == nullptr || rows_on_16(static_cast<const T*>(p), ld, 0, 1); };
    const bool tokens_gate = a.gate_mode == kGateTokens;
    a.once = norm_past_caches(sizeof(T), aligned(a.dZ, a.lddz) && aligned(a.dH, a.lddh) && aligned(a.H, a.ldh) &&
                                             aligned(a.Y, a.ldy) && aligned(a.dX, a.lddx) && aligned(a.dY, a.lddy) &&
                                             (!tokens_gate || (aligned(a.gate, a.ldgate) && aligned(a.dgate, a.lddgate))));
    const int64_t groups = norm_backward_groups(a.T, a.d);
    if (groups > 0) {
        const bool packed = a.H == nullptr, tokens = tokens_gate;
        const hipError_t e = packed ? (tokens ? backward_rows<T, true, true>(a, groups, stream)
                                              : backward_rows<T, true, false>(a, groups, stream))
                                    : (tokens ? backward_rows<T, false, true>(a, groups, stream)
                                              : backward_rows<T, false, false>(a, groups, stream));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(norm_join_kernel, dim3(static_cast<unsigned>((2 * a.d + 31) / 32)), dim3(1024), 0, stream, a, groups);
    return hipGetLastError();
}

}  // namespace

// Workgroups of the backward pass: two to a CU (of 256 threads), one past d = 2048,
// where each adds 32 KB and more of sums to the traffic; or as many as there are rows.
// 8192 x 4096 bf16 from checkpoints, other inputs each time: 512 workgroups 78.6 us, 256
// 72.3 (69.5 and 65.7 with the streaming stores and loads); 8192 x 2048: 44.4 and 44.5.
int64_t norm_backward_groups(int64_t T, int64_t d) {
    const int64_t rows = d <= 1024 ? 4 : 1;
    return std::min<int64_t>((T + rows - 1) / rows, d <= 2048 ? 512 : 256);
}

hipError_t launch_norm_forward(const NormForwardArgs& a, bool bf16, hipStream_t stream) {
    if (a.T == 0) return hipSuccess;
    return bf16 ? forward<bf16_t>(a, stream) : forward<float>(a, stream);
}
hipError_t launch_norm_backward(const NormBackwardArgs& a, bool bf16, hipStream_t stream) {
    return bf16 ? backward<bf16_t>(a, stream) : backward<float>(a, stream);
}

}  // namespace galore
