// Block formats of the training operators: 32 consecutive values of a row share
// one scale byte E (E8M0: 2^(E - 127), 255 is NaN).
//   8-bit checkpoint: int8 c, value c 2^(E - 133), |c| <= 127
//   4-bit: E2M1 (sign, then 0, .5, 1, 1.5, 2, 3, 4, 6), value times 2^(E - 127)
// E is the smallest with which no value of the block is clipped, so that a value
// moves by at most half a step of its code; at the type's very end, where the
// decoded value would be an Inf, E stays (254 and 252) and the largest code is
// taken. Powers of two make the scaling
// exact: the only rounding is that to a code (half to even), and c 2^(E - 133)
// and the 4-bit values are exact in bfloat16. The lower bounds of E (8 and 3)
// keep every step of a code a normal fp32 number; smaller magnitudes round to
// zero. In a block with a NaN or an Inf, E = 255: every value of it reads as NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace galore {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));   // no more than the element's alignment

constexpr int kMxBlock = 32;
constexpr int kMxNan = 255;
constexpr float kMxMagic = 12582912.0f;   // 1.5 2^23: x + magic holds round-half-even(x) in its low bits, |x| < 2^22

__host__ __device__ inline int64_t mx_blocks(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock; }
// scale bytes of a row: whole dwords, the bytes past the last block zero
__host__ __device__ inline int64_t mx_scale_bytes(int64_t cols) { return (mx_blocks(cols) + 3) / 4 * 4; }

// scale byte of a block whose largest magnitude has the bits `amax` (sign clear)
__device__ __forceinline__ int mx8_scale(uint32_t amax) {
    if (amax >= 0x7f800000u) return kMxNan;
    const int e = static_cast<int>(amax >> 23) + ((amax & 0x7fffffu) > 0x7e0000u ? 1 : 0);   // 127 = 1.984375 2^6
    return min(max(e, 8), 254);
}
__device__ __forceinline__ int mx4_scale(uint32_t amax) {
    if (amax >= 0x7f800000u) return kMxNan;
    const int e = static_cast<int>(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x400000u ? 1 : 0);   // 6 = 1.5 2^2
    return min(max(e, 3), 252);
}
// the inverse of a code's unit, 2^(SHIFT - E) (E as written by mx8_scale / mx4_scale, not NaN)
template <int SHIFT>
__device__ __forceinline__ float mx_inverse(int e) {
    return __uint_as_float(static_cast<uint32_t>(127 + SHIFT - e) << 23);
}
// a code's unit, 2^(E - SHIFT), for any byte
template <int SHIFT>
__device__ __forceinline__ float mx_unit(int e) {
    return e == kMxNan ? __uint_as_float(0x7fc00000u) : ldexpf(1.0f, e - SHIFT);
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// the larger of each half of two words
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return __uint_as_float(static_cast<uint32_t>(
        __builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(v)), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v)), lane)));
}
// sum over the wave, the same bits in every lane: within 16 lanes by cross-lane
// moves (no LDS), then over the four sixteens
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0xB1>(v);    // lanes 1 0 3 2 of a quad
    v += moved<0x4E>(v);    // lanes 2 3 0 1
    v += moved<0x141>(v);   // mirrored within 8
    v += moved<0x140>(v);   // mirrored within 16
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// maximum over the four lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    int x = static_cast<int>(v);
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    x = max(x, __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
    return static_cast<uint32_t>(x);
}

// four int8 codes of x / unit (inv = 1 / unit): exact scaling, one rounding
__device__ __forceinline__ uint32_t mx8_encode4(float a, float b, float c, float d, float inv) {
    const uint32_t ua = __float_as_uint(__builtin_amdgcn_fmed3f(a * inv, -127.0f, 127.0f) + kMxMagic);
    const uint32_t ub = __float_as_uint(__builtin_amdgcn_fmed3f(b * inv, -127.0f, 127.0f) + kMxMagic);
    const uint32_t uc = __float_as_uint(__builtin_amdgcn_fmed3f(c * inv, -127.0f, 127.0f) + kMxMagic);
    const uint32_t ud = __float_as_uint(__builtin_amdgcn_fmed3f(d * inv, -127.0f, 127.0f) + kMxMagic);
    return __builtin_amdgcn_perm(ub, ua, 0x0c0c0400u) | __builtin_amdgcn_perm(ud, uc, 0x04000c0cu);
}
// eight int8 codes and the block's scale byte, the block being this lane's quad
__device__ __forceinline__ u32x2 mx8_encode_quad(const float (&x)[8], int& scale) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x[i]));
    scale = mx8_scale(quad_max(m));
    if (scale == kMxNan) return u32x2{0u, 0u};
    const float inv = mx_inverse<133>(scale);
    return u32x2{mx8_encode4(x[0], x[1], x[2], x[3], inv), mx8_encode4(x[4], x[5], x[6], x[7], inv)};
}

// eight E2M1 codes of x / unit: gfx950's conversions divide by the scale they are
// given, a power of two here, and round half to even and to 6 at most
__device__ __forceinline__ uint32_t mx4_encode8(const float (&x)[8], float unit) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
    return w;
}
// the same of four words of two bf16
__device__ __forceinline__ uint32_t mx4_encode8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float unit) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, a), unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, b), unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, c), unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, d), unit, 3);
    return w;
}
// the scale byte's power of two, 2^(E - 127), E from mx4_scale
__device__ __forceinline__ float mx4_unit(int e) { return __uint_as_float(static_cast<uint32_t>(e) << 23); }

// four int8 codes as floats (one conversion each, the byte picked by the instruction)
__device__ __forceinline__ void mx8_floats4(uint32_t word, float* x) {
    const int w = static_cast<int>(word);
    x[0] = static_cast<float>(static_cast<int8_t>(w));
    x[1] = static_cast<float>(static_cast<int8_t>(w >> 8));
    x[2] = static_cast<float>(static_cast<int8_t>(w >> 16));
    x[3] = static_cast<float>(w >> 24);
}
// x[i] = codes of a word pair times the unit
__device__ __forceinline__ void mx8_decode8(u32x2 w, float unit, float (&x)[8]) {
    mx8_floats4(w[0], x);
    mx8_floats4(w[1], x + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= unit;
}

// An array that a call reads or writes once, end to end, goes past the caches'
// replacement order (non-temporal, `once`): it would only displace what is used again.
// Not where rows start off 16 bytes: the pieces of a line that lanes share would each go
// to memory by itself (backward norms of 8192 x 2731 bf16 so 168 us, 2736: 74). A read
// takes the alignment of its elements for granted and no more: the group across a row's
// end starts off 16 bytes where the rows start on them.
template <typename V, typename T>
__device__ __forceinline__ V get_vector(const T* p, bool once) {
    typedef V at_elements __attribute__((aligned(alignof(T))));
    if (once) return __builtin_nontemporal_load(reinterpret_cast<const at_elements*>(p));
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
// (with `once`, p is on the vector's alignment)
template <typename V>
__device__ __forceinline__ void put_vector(void* p, V v, bool once) {
    if (once) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else __builtin_memcpy(p, &v, sizeof(V));
}

template <typename T>
inline bool rows_on_16(const T* p, int64_t ld, int64_t stride, int batch) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * sizeof(T) % 16 == 0 && (batch == 1 || stride * sizeof(T) % 16 == 0);
}

// Entries e .. e + 7 of a row of n >= 1 as they are stored, zeros past its end (once
// `settle` has run). The group that crosses the end is loaded as the row's last eight, in
// one load like the others, and shifted when it is used: entry by entry it would hold
// the row up for a memory latency each. e is a multiple of 8; where it is
// past the row's end nothing is read.
template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const bf16_t* row, int e, int n, bool once = false) {
        if (n >= 8) {
            clear();
            if (e < n) w = get_vector<u32x4>(row + min(e, n - 8), once);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (e + 2 * i < n ? row[min(2 * i, n - 1)].bits : 0u) |
                       (e + 2 * i + 1 < n ? static_cast<uint32_t>(row[min(2 * i + 1, n - 1)].bits) << 16 : 0u);
        }
    }
    __device__ __forceinline__ void settle(int e, int n) {
        if ((n & 7) == 0 || n < 8) return;
        if (e + 8 <= n || e >= n) return;
        for (int k = e + 8 - n; k > 0; --k) {
            w[0] = __builtin_amdgcn_alignbit(w[1], w[0], 16);
            w[1] = __builtin_amdgcn_alignbit(w[2], w[1], 16);
            w[2] = __builtin_amdgcn_alignbit(w[3], w[2], 16);
            w[3] >>= 16;
        }
    }
    __device__ __forceinline__ void clear() { w = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ float operator[](int i) const {
        return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
};
template <>
struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void load(const float* row, int e, int n, bool once = false) {
        if (n >= 8) {
            clear();
            if (e < n) {
                const float* p = row + min(e, n - 8);
                const f32x4 a = get_vector<f32x4>(p, once);
                const f32x4 b = get_vector<f32x4>(p + 4, once);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = a[i];
                    v[4 + i] = b[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = e + i < n ? row[min(i, n - 1)] : 0.0f;
                asm("" : "+v"(v[i]));   // waited for here: otherwise the loads of the long rows wait in its place
            }
        }
    }
    __device__ __forceinline__ void settle(int e, int n) {
        if ((n & 7) == 0 || n < 8) return;
        if (e + 8 <= n || e >= n) return;
        for (int k = e + 8 - n; k > 0; --k) {
#pragma unroll
            for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
            v[7] = 0.0f;
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
template <typename T>
__device__ __forceinline__ void load8(const T* row, int e, int n, float (&x)[8]) {
    Eight<T> r;
    r.load(row, e, n);
    r.settle(e, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r[i];
}

// two bfloat16 nearest to a and b (ties to even; NaN stays NaN)
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    bf16x2_t v;
    v[0] = static_cast<__bf16>(a);
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ void store8(float* p, int64_t valid, const float (&x)[8], bool once = false) {
    if (valid >= 8) {
        put_vector(p, f32x4{x[0], x[1], x[2], x[3]}, once);
        put_vector(p + 4, f32x4{x[4], x[5], x[6], x[7]}, once);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = x[i];
    }
}
__device__ __forceinline__ void store8(bf16_t* p, int64_t valid, const float (&x)[8], bool once = false) {
    const u32x4 w = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    if (valid >= 8) {
        put_vector(p, w, once);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i].bits = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
    }
}

// `bytes` of memory from p on (a uniform address), for loads at 32-bit offsets that
// cost no address arithmetic; reads past them return zero
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0,
                                             static_cast<int>(bytes < 0xffffffffll ? bytes : 0xffffffffll), 0x00027000);
}

// One 32 x 32 block of a product's accumulators to C (rounded once; added to C with
// `add`). A lane holds column c and rows r0 + (v & 3) + 8 (v >> 2), r0 with the 4
// of its half.
template <typename OutT>
__device__ __forceinline__ void store_block(OutT* C, int64_t ldc, int r0, int c, int M, int N, const f32x16& acc, bool add) {
    OutT* dst = C + static_cast<int64_t>(r0) * ldc + c;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int dr = (v & 3) + 8 * (v >> 2);
        if (r0 + dr < M && c < N) {
            float s = acc[v];
            if (add) s += to_f32(dst[dr * ldc]);
            if constexpr (sizeof(OutT) == 2) dst[dr * ldc].bits = static_cast<uint16_t>(bf16_pair(s, 0.0f));
            else dst[dr * ldc] = s;
        }
    }
}
// The same inside C, without bounds. In bf16 (rows on 4 bytes) lanes 2 i and 2 i + 1
// exchange values so that each stores two columns of one row: half the stores, of
// four bytes each.
template <typename OutT>
__device__ __forceinline__ void store_whole_block(OutT* C, int64_t ldc, int r0, int c, const f32x16& acc, bool add) {
    if constexpr (sizeof(OutT) == 2) {
        const bool odd = (c & 1) != 0;
        OutT* dst = C + static_cast<int64_t>(r0 + (odd ? 1 : 0)) * ldc + (c & ~1);
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
            const int give = static_cast<int>(__float_as_uint(odd ? acc[v] : acc[v + 1]));
            const float got = __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(give, 0xB1, 0xf, 0xf, true)));
            float lo = odd ? got : acc[v], hi = odd ? acc[v + 1] : got;
            uint32_t* p = reinterpret_cast<uint32_t*>(dst + ((v & 3) + 8 * (v >> 2)) * ldc);
            if (add) {
                const uint32_t old = *p;
                lo += __uint_as_float(old << 16);
                hi += __uint_as_float(old & 0xffff0000u);
            }
            *p = bf16_pair(lo, hi);
        }
    } else {
        OutT* dst = C + static_cast<int64_t>(r0) * ldc + c;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            OutT* p = dst + ((v & 3) + 8 * (v >> 2)) * ldc;
            *p = add ? acc[v] + *p : acc[v];
        }
    }
}
// Tile of MB x NB blocks of one wave, its first row (with the lane's 4) and column
template <int MB, int NB, typename OutT>
__device__ __forceinline__ void store_tile(OutT* C, int64_t ldc, int r0, int c0, int M, int N, const f32x16 (&acc)[MB][NB],
                                           bool add, int lane) {
    const bool whole = c0 + 32 * NB <= N && (r0 & ~31) + 32 * MB <= M &&
                       (sizeof(OutT) == 4 || (ldc % 2 == 0 && reinterpret_cast<uintptr_t>(C) % 4 == 0));
    if (__builtin_amdgcn_readfirstlane(whole)) {
#pragma unroll
        for (int x = 0; x < MB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                store_whole_block(C, ldc, r0 + 32 * x, c0 + 32 * y + (lane & 31), acc[x][y], add);
                __builtin_amdgcn_sched_barrier(0);   // one block's addresses at a time
            }
    } else {
#pragma unroll
        for (int x = 0; x < MB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                store_block(C, ldc, r0 + 32 * x, c0 + 32 * y + (lane & 31), M, N, acc[x][y], add);
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// Rows of a streaming kernel: workgroups of 256 threads, `width` (a power of two,
// 4 .. 256) of them along a row's groups of eight values and the others down its
// rows, so that narrow rows fill a workgroup too. A launch's work-items along x fit
// 32 bits, so a workgroup walks over the rows past 2^22 workgroups.
struct RowGrid {
    dim3 grid, block;
};
inline RowGrid row_grid(int64_t rows, int64_t groups, int batch) {
    unsigned width = 4;
    while (width < 256 && width < groups) width *= 2;
    const unsigned down = 256 / width;
    const int64_t x = (rows + down - 1) / down;
    return {dim3(static_cast<unsigned>(x < (1 << 22) ? x : (1 << 22)), static_cast<unsigned>((groups + width - 1) / width),
                 static_cast<unsigned>(batch)),
            dim3(width, down)};
}

__device__ __forceinline__ int64_t first_row() { return static_cast<int64_t>(blockIdx.x) * blockDim.y + threadIdx.y; }
__device__ __forceinline__ int64_t row_step() { return static_cast<int64_t>(gridDim.x) * blockDim.y; }

// The code matrices of the entry points, checked by the host side
struct MxMatrix {
    uint8_t* codes;      // rows of ldq bytes (a multiple of 16), base on 16 bytes
    int64_t ldq, stride_q;
    uint8_t* scales;     // rows of lds bytes (a multiple of 4), base on 4 bytes
    int64_t lds, stride_s;
    // the batch from its matrix b on
    __host__ __device__ MxMatrix from(int64_t b) const {
        MxMatrix q = *this;
        q.codes += b * stride_q;
        q.scales += b * stride_s;
        return q;
    }
};

// codes and scale of eight values whose block is this lane's quad
__device__ __forceinline__ void put_codes(const MxMatrix& q, int64_t row, int64_t g, int64_t nb, const float (&x)[8]) {
    int scale;
    const u32x2 w = mx8_encode_quad(x, scale);
    if (g < 4 * nb) put_vector(q.codes + row * q.ldq + 8 * g, w, true);
    if ((g & 3) == 0 && g < 4 * ((nb + 3) / 4 * 4)) q.scales[row * q.lds + (g >> 2)] = static_cast<uint8_t>(g < 4 * nb ? scale : 0);
}

}  // namespace galore
