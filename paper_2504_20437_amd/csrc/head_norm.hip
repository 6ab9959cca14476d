// Norms of queries and keys for each head and their rotation by position, in one pass:
//   n = x rstd(x) w,  rstd(x) = (mean x^2 + eps)^(-1/2) over the head's d values
//   (y_i, y_j) = (n_i cos - n_j sin, n_i sin + n_j cos) for the rot / 2 pairs, y = n past them
// and backward, the transposed rotation first:
//   (m_i, m_j) = (dy_i cos + dy_j sin, dy_j cos - dy_i sin)
//   dw = sum over tokens and heads of m x rstd,  p = m w
//   dx = rstd (p - x rstd^2 mean(p x))
// Nothing is kept for the backward pass but x itself, or its 8-bit checkpoint: the
// statistics are summed again from what is read anyway, in the same round of the
// lanes' sums as p x.
//
// Bound by memory. A head belongs to as few lanes as hold eight pairs each: both values
// of a pair lie in one lane, in two vectors of 16 bytes (bf16) that start half the
// rotated width apart, or next to each other where pairs are neighbours. A wave takes
// one token at a time and several heads of it, so that the token's cosines and sines
// stay in registers; backward, queries and keys have workgroups of their own, 384 each,
// which leaves three waves a SIMD. 8192 tokens of 32 + 4 heads of 128 bf16 26.6 us (5.8
// TB/s), one token 4.7; backward 8192 x 64 heads from checkpoints 72 (4.7), from tensors 85
// (4.7), 32 + 4 heads 62 (3.6). Value by value, where the width, the rotated width, a row
// or w is not on 16: 8192 x 32 heads of 80, 40 rotated, 87 (1.0 TB/s) and backward 130.
// Tried backward from checkpoints, when what is read still went through the caches and
// took 81: both kinds' weights and sums in a thread, two waves a SIMD, 91; 256 or 768
// workgroups 94 and 81. A wave that keeps to its heads, with the next token's rows and
// angles loaded ahead, took 87, forward 48.
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "layers.hpp"

namespace galore {
namespace {

// sum over LANES neighbouring lanes, the same bits in each
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (LANES >= 2) v += moved<0xB1>(v);
    if constexpr (LANES >= 4) v += moved<0x4E>(v);
    if constexpr (LANES >= 8) v += moved<0x141>(v);
    if constexpr (LANES >= 16) v += moved<0x140>(v);
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
    if constexpr (LANES >= 64) v += __shfl_xor(v, 32);
    return v;
}

// How a lane's eight pairs lie in a head: kSplit and kNeighbours in two vectors of eight
// values, kAny value by value
enum Pairs { kSplit, kNeighbours, kAny };

// place of the first (k = 0) or second value of pair p of a head; -1 for none. Past the
// rotated values the rest is paired too, first half with second, or as neighbours.
template <int PAIRS>
__device__ __forceinline__ int place(int p, int k, int d, int rot, bool interleaved) {
    if (PAIRS == kNeighbours || (PAIRS == kAny && interleaved)) {
        const int e = 2 * p + k;
        return e < d ? e : -1;
    }
    const int half = rot / 2;
    if (p < half) return p + k * half;
    const int rest = d - rot, first = (rest + 1) / 2, q = p - half;
    if (k == 0) return q < first ? rot + q : -1;
    return first + q < rest ? rot + first + q : -1;
}

// x[i] and x[8 + i]: the pair i of the lane (`once`: past the caches)
template <int PAIRS, typename T>
__device__ __forceinline__ void load_pairs(const T* row, int p0, int d, int rot, bool interleaved, float (&x)[16],
                                           bool once = false) {
    if constexpr (PAIRS == kAny) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = place<PAIRS>(p0 + (i & 7), i >> 3, d, rot, interleaved);
            x[i] = e >= 0 ? to_f32(row[e]) : 0.0f;
        }
    } else {
        float a[8] = {}, b[8] = {};
        if (2 * p0 < d) {
            const int ea = PAIRS == kSplit ? place<PAIRS>(p0, 0, d, rot, false) : 2 * p0;
            const int eb = PAIRS == kSplit ? place<PAIRS>(p0, 1, d, rot, false) : 2 * p0 + 8;
            Eight<T> ra, rb;
            ra.load(row + ea, 0, 8, once);
            rb.load(row + eb, 0, 8, once);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                a[i] = ra[i];
                b[i] = rb[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kSplit) {
                x[i] = a[i];
                x[8 + i] = b[i];
            } else {
                x[i] = i < 4 ? a[2 * i] : b[2 * i - 8];
                x[8 + i] = i < 4 ? a[2 * i + 1] : b[2 * i - 7];
            }
        }
    }
}

template <int PAIRS, typename T>
__device__ __forceinline__ void store_pairs(T* row, int p0, int d, int rot, bool interleaved, const float (&x)[16],
                                            bool once = false) {
    if constexpr (PAIRS == kAny) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = place<PAIRS>(p0 + (i & 7), i >> 3, d, rot, interleaved);
            if (e < 0) continue;
            if constexpr (sizeof(T) == 2) row[e].bits = static_cast<uint16_t>(bf16_pair(x[i], 0.0f));
            else row[e] = x[i];
        }
    } else {
        if (2 * p0 >= d) return;
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kSplit) {
                a[i] = x[i];
                b[i] = x[8 + i];
            } else {
                a[i] = x[(i >> 1) + 8 * (i & 1)];
                b[i] = x[4 + (i >> 1) + 8 * (i & 1)];
            }
        }
        const int ea = PAIRS == kSplit ? place<PAIRS>(p0, 0, d, rot, false) : 2 * p0;
        const int eb = PAIRS == kSplit ? place<PAIRS>(p0, 1, d, rot, false) : 2 * p0 + 8;
        store8(row + ea, 8, a, once);
        store8(row + eb, 8, b, once);
    }
}

// the values of an 8-bit checkpoint whose head begins at value `base` of the token's row
template <int PAIRS>
__device__ __forceinline__ void load_pairs(const MxMatrix& q, int64_t token, int64_t base, int p0, int d, int rot,
                                           bool interleaved, float (&x)[16]) {
    const uint8_t* codes = q.codes + token * q.ldq;
    const uint8_t* scales = q.scales + token * q.lds;
    if constexpr (PAIRS == kAny) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = place<PAIRS>(p0 + (i & 7), i >> 3, d, rot, interleaved);
            x[i] = 0.0f;
            if (e >= 0) x[i] = static_cast<float>(static_cast<int8_t>(codes[base + e])) * mx_unit<133>(scales[(base + e) >> 5]);
        }
    } else {
        float a[8] = {}, b[8] = {};
        if (2 * p0 < d) {
            const int64_t ea = base + (PAIRS == kSplit ? place<PAIRS>(p0, 0, d, rot, false) : 2 * p0);
            const int64_t eb = base + (PAIRS == kSplit ? place<PAIRS>(p0, 1, d, rot, false) : 2 * p0 + 8);
            const u32x2 wa = *reinterpret_cast<const u32x2*>(codes + ea), wb = *reinterpret_cast<const u32x2*>(codes + eb);
            mx8_decode8(wa, mx_unit<133>(scales[ea >> 5]), a);
            mx8_decode8(wb, mx_unit<133>(scales[eb >> 5]), b);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (PAIRS == kSplit) {
                x[i] = a[i];
                x[8 + i] = b[i];
            } else {
                x[i] = i < 4 ? a[2 * i] : b[2 * i - 8];
                x[8 + i] = i < 4 ? a[2 * i + 1] : b[2 * i - 7];
            }
        }
    }
}

// cosines and sines of a lane's pairs at one position: (1, 0) past the rotated ones
__device__ __forceinline__ void load_angles(const float* row, int p0, int rot, float (&c)[8], float (&s)[8]) {
    const int half = rot / 2;
    if (p0 + 8 <= half) {
        load8(row + p0, 0, 8, c);
        load8(row + half + p0, 0, 8, s);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool in = p0 + i < half;
        c[i] = in ? row[p0 + i] : 1.0f;
        s[i] = in ? row[half + p0 + i] : 0.0f;
    }
}

// a token's position: its cosines and sines, or kNone (a negative position: padding), or NaN past the table
enum Where { kInside, kNone, kPast };
__device__ __forceinline__ Where angles_of(const HeadNormArgs& a, int64_t token, int p0, float (&c)[8], float (&s)[8]) {
    const int64_t at = a.positions.p != nullptr ? a.positions.at(token) : token;
    if (at < 0 || at >= a.table_rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = s[i] = at < 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        return at < 0 ? kNone : kPast;
    }
    load_angles(a.table + at * a.ld_table, p0, a.rot, c, s);
    return kInside;
}

// a wave's work: tokens wave, wave + waves ...; of each, `split` waves share the heads
struct WaveSpan {
    int64_t token, step;
    int head, heads;           // first head of the lane's group, heads between its own
};
template <int LANES>
__device__ __forceinline__ WaveSpan wave_span(int64_t waves, int split) {
    const int64_t w = static_cast<int64_t>(blockIdx.x) * (blockDim.x / 64) + (threadIdx.x >> 6);
    constexpr int kRows = 64 / LANES;
    return {w / split, waves / split, static_cast<int>(w % split) * kRows + static_cast<int>(threadIdx.x & 63) / LANES,
            split * kRows};
}

// Past the caches in bf16: forward what is written (8192 x 36 heads of 128, a call: 28 us,
// 32 through them, 33 with what is read too), backward what is read (8192 x 64 heads from
// checkpoints: 73 to 79 and 81, plain 77 to 88 and 89, in several sessions)
template <typename T>
constexpr bool kOnce = sizeof(T) == 2;

template <typename T, int LANES, int PAIRS>
__global__ __launch_bounds__(256) void head_norm_kernel(HeadNormArgs a, int64_t waves, int split) {
    const WaveSpan at = wave_span<LANES>(waves, split);
    const int p0 = 8 * (threadIdx.x % LANES);
    const float inv_d = 1.0f / static_cast<float>(a.d);
    for (int64_t t = at.token; t < a.tokens; t += at.step) {
        float c[8], s[8];
        const Where where = angles_of(a, t, p0, c, s);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float w[16];
            load_pairs<PAIRS>(a.w[k], p0, a.d, a.rot, a.interleaved, w);
            for (int h = at.head; h < a.in[k].n; h += at.heads) {
                float x[16];
                load_pairs<PAIRS>(static_cast<const T*>(a.in[k].p) + t * a.in[k].token + h * a.in[k].head, p0, a.d, a.rot,
                                  a.interleaved, x);
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
                const float r = 1.0f / sqrtf(lanes_sum<LANES>(sum) * inv_d + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float n0 = x[i] * r * w[i], n1 = x[8 + i] * r * w[8 + i];
                    x[i] = n0 * c[i] - n1 * s[i];
                    x[8 + i] = n0 * s[i] + n1 * c[i];
                    if (where == kNone) x[i] = x[8 + i] = 0.0f;
                    if (where == kPast) x[i] = x[8 + i] = c[0];
                }
                store_pairs<PAIRS>(static_cast<T*>(a.out[k].p) + t * a.out[k].token + h * a.out[k].head, p0, a.d, a.rot,
                                   a.interleaved, x, kOnce<T>);
            }
        }
    }
}

// (field by field: a choice between structs goes through memory)
__device__ __forceinline__ Heads pick(const Heads (&h)[2], int k) {
    return {k ? h[1].p : h[0].p, k ? h[1].token : h[0].token, k ? h[1].head : h[0].head, k ? h[1].n : h[0].n};
}
__device__ __forceinline__ MxMatrix pick(const MxMatrix (&q)[2], int k) {
    return {k ? q[1].codes : q[0].codes, k ? q[1].ldq : q[0].ldq, 0, k ? q[1].scales : q[0].scales, k ? q[1].lds : q[0].lds, 0};
}

// Queries and keys in workgroups of their own, so that a thread holds one kind's weights and sums
template <typename T, int LANES, int PAIRS, bool PACKED>
__global__ __launch_bounds__(256) void head_norm_backward_kernel(HeadNormArgs a, int64_t waves, int split) {
    __shared__ float join[4][LANES * 16];
    const WaveSpan at = wave_span<LANES>(waves, split);
    const int lane = threadIdx.x % LANES, p0 = 8 * lane, wave = threadIdx.x >> 6;
    const float inv_d = 1.0f / static_cast<float>(a.d);
    const int k = blockIdx.y;               // queries or keys
    const Heads from = pick(a.in, k), to = pick(a.out, k), saved = pick(a.saved, k);
    const MxMatrix codes = pick(a.codes, k);
    float w[16], dw[16] = {};
    load_pairs<PAIRS>(k ? a.w[1] : a.w[0], p0, a.d, a.rot, a.interleaved, w);
    for (int64_t t = at.token; t < a.tokens; t += at.step) {
        float c[8], s[8];
        const Where where = angles_of(a, t, p0, c, s);
        for (int h = at.head; h < from.n; h += at.heads) {
            float x[16], m[16];
            load_pairs<PAIRS>(static_cast<const T*>(from.p) + t * from.token + h * from.head, p0, a.d, a.rot,
                              a.interleaved, m, kOnce<T>);
            if constexpr (PACKED)
                load_pairs<PAIRS>(codes, t, static_cast<int64_t>(h) * a.d, p0, a.d, a.rot, a.interleaved, x);
            else
                load_pairs<PAIRS>(static_cast<const T*>(saved.p) + t * saved.token + h * saved.head, p0,
                                  a.d, a.rot, a.interleaved, x, kOnce<T>);
            float sx = 0.0f, sp = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float m0 = m[i] * c[i] + m[8 + i] * s[i], m1 = m[8 + i] * c[i] - m[i] * s[i];
                m[i] = m0;
                m[8 + i] = m1;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sx += x[i] * x[i];
                sp += m[i] * w[i] * x[i];
            }
            const float r = 1.0f / sqrtf(lanes_sum<LANES>(sx) * inv_d + a.eps);
            const float mean = lanes_sum<LANES>(sp) * inv_d * r * r;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (where != kNone) dw[i] += m[i] * (x[i] * r);
                x[i] = r * (m[i] * w[i] - x[i] * mean);
                if (where == kNone) x[i] = 0.0f;
                if (where == kPast) x[i] = c[0];
            }
            store_pairs<PAIRS>(static_cast<T*>(to.p) + t * to.token + h * to.head, p0, a.d, a.rot,
                               a.interleaved, x);
        }
    }
    // the sums of a wave's head groups, then of its waves, in order; then to memory
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float v = dw[i];
#pragma unroll
        for (int step = LANES; step < 64; step *= 2) v += __shfl_xor(v, step);
        dw[i] = v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) < LANES) {
#pragma unroll
        for (int i = 0; i < 16; ++i) join[wave][16 * lane + i] = dw[i];
    }
    __syncthreads();
    if (threadIdx.x < LANES) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int e = place<kAny>(p0 + (i & 7), i >> 3, a.d, a.rot, a.interleaved);
            if (e < 0) continue;
            const float* j = &join[0][16 * lane + i];
            a.part[(static_cast<int64_t>(blockIdx.x) * 2 + k) * a.d + e] =
                (j[0] + j[LANES * 16]) + (j[2 * LANES * 16] + j[3 * LANES * 16]);
        }
    }
}

// dw_q and dw_k from the workgroups' sums: 32 columns a workgroup, 32 slices of the
// workgroups joined in LDS in order
__global__ __launch_bounds__(1024) void head_norm_join_kernel(HeadNormArgs a, int64_t groups) {
    __shared__ float red[32][33];
    const int c = threadIdx.x & 31, sl = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + c;      // of 2 d
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
    (col < a.d ? a.dw[0] : a.dw[1])[col < a.d ? col : col - a.d] = s;
}

int pair_count(int d, int rot, bool interleaved) { return interleaved ? (d + 1) / 2 : rot / 2 + (d - rot + 1) / 2; }

// f(lanes) for the lanes that hold a head's pairs
template <typename F>
hipError_t with_lanes(int pairs, F f) {
    if (pairs <= 8) return f(std::integral_constant<int, 1>());
    if (pairs <= 16) return f(std::integral_constant<int, 2>());
    if (pairs <= 32) return f(std::integral_constant<int, 4>());
    if (pairs <= 64) return f(std::integral_constant<int, 8>());
    if (pairs <= 128) return f(std::integral_constant<int, 16>());
    if (pairs <= 256) return f(std::integral_constant<int, 32>());
    return f(std::integral_constant<int, 64>());
}

template <typename T>
Pairs pairs_of(const HeadNormArgs& a, bool backward, bool packed) {
    const auto ok = [](const Heads& h) { return rows_on_16(static_cast<const T*>(h.p), h.token, h.head, 2); };
    for (int k = 0; k < 2; ++k) {
        if (!ok(a.in[k]) || !ok(a.out[k]) || !rows_on_16(a.w[k], 0, 0, 1)) return kAny;
        if (backward && !packed && !ok(a.saved[k])) return kAny;
    }
    if (a.d % 16 != 0 || a.rot % 16 != 0) return kAny;
    return a.interleaved ? kNeighbours : kSplit;
}

// waves of a launch, and how many share a token's heads: enough to fill the chip
struct WavePlan {
    int64_t groups;      // workgroups of four waves
    int split;
};
WavePlan wave_plan(int64_t tokens, int64_t heads, int lanes, int64_t most) {
    const int64_t rows = 64 / lanes, passes = (heads + rows - 1) / rows;
    int split = 1;
    while (split < 4 && split < passes && tokens * split < 8192) split *= 2;
    while (split < passes && tokens * split < 64) split *= 2;
    const int64_t unit = std::max(split / 4, 1);            // workgroups that share a token
    const int64_t want = (tokens * split + 3) / 4;
    int64_t groups = std::min(want, most);
    groups = std::max<int64_t>((groups + unit - 1) / unit * unit, unit);
    return {groups, split};
}

template <typename T, typename F>
hipError_t with_form(const HeadNormArgs& a, Pairs pairs, F f) {
    return with_lanes(pair_count(a.d, a.rot, a.interleaved), [&](auto lanes) {
        if (pairs == kSplit) return f(lanes, std::integral_constant<int, kSplit>());
        if (pairs == kNeighbours) return f(lanes, std::integral_constant<int, kNeighbours>());
        return f(lanes, std::integral_constant<int, kAny>());
    });
}

template <typename T>
hipError_t forward(const HeadNormArgs& a, hipStream_t stream) {
    return with_form<T>(a, pairs_of<T>(a, false, false), [&](auto lanes, auto pairs) {
        const WavePlan plan = wave_plan(a.tokens, std::max(a.in[0].n, a.in[1].n), decltype(lanes)::value, 4096);
        hipLaunchKernelGGL((head_norm_kernel<T, decltype(lanes)::value, decltype(pairs)::value>),
                           dim3(static_cast<unsigned>(plan.groups)), dim3(256), 0, stream, a, 4 * plan.groups, plan.split);
        return hipGetLastError();
    });
}

template <typename T, bool PACKED>
hipError_t backward(const HeadNormArgs& a, int64_t most, hipStream_t stream, int64_t& groups) {
    return with_form<T>(a, pairs_of<T>(a, true, PACKED), [&](auto lanes, auto pairs) {
        const WavePlan plan = wave_plan(a.tokens, std::max(a.in[0].n, a.in[1].n), decltype(lanes)::value, most);
        groups = plan.groups;
        hipLaunchKernelGGL((head_norm_backward_kernel<T, decltype(lanes)::value, decltype(pairs)::value, PACKED>),
                           dim3(static_cast<unsigned>(plan.groups), 2), dim3(256), 0, stream, a, 4 * plan.groups, plan.split);
        return hipGetLastError();
    });
}

constexpr int64_t kBackwardGroups = 384;

}  // namespace

// an upper bound of the backward pass's workgroups, for its partial sums
int64_t head_norm_groups(int64_t tokens) {
    // (a token's heads are shared by up to 64 waves where tokens are few)
    return tokens == 0 ? 0 : std::min<int64_t>(16 * tokens + 16, kBackwardGroups + 16);
}

hipError_t launch_head_norm(const HeadNormArgs& a, bool bf16, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    return bf16 ? forward<bf16_t>(a, stream) : forward<float>(a, stream);
}

hipError_t launch_head_norm_backward(const HeadNormArgs& a, bool bf16, hipStream_t stream) {
    int64_t groups = 0;
    if (a.tokens > 0) {
        const bool packed = a.codes[0].codes != nullptr;
        const hipError_t e = bf16 ? (packed ? backward<bf16_t, true>(a, kBackwardGroups, stream, groups)
                                            : backward<bf16_t, false>(a, kBackwardGroups, stream, groups))
                                  : (packed ? backward<float, true>(a, kBackwardGroups, stream, groups)
                                            : backward<float, false>(a, kBackwardGroups, stream, groups));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(head_norm_join_kernel, dim3(static_cast<unsigned>((2 * a.d + 31) / 32)), dim3(1024), 0, stream, a,
                       groups);
    return hipGetLastError();
}

}  // namespace galore
