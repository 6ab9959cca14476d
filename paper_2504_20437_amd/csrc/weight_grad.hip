// Weight gradient from an 8-bit checkpoint: G = dY^T X (+ G), the sum over the
// tokens of the incoming gradient's outer products with the layer's input, read
// from its codes.
//
// Both operands have the tokens, the axis of the sum, as their rows. A stage of
// 32 tokens of each is held in LDS as it lies in memory (the checkpoint decoded
// to bfloat16, exactly, on its way there) and the transposing LDS reads hand the
// matrix cores eight tokens of one column. An fp32 gradient is cut into three
// bfloat16 planes, x = h1 + h2 + h3 exactly (3 x 8 bits of its 24), and takes
// three products; sums are held in fp32.
//
// Few tiles (small weights, long batches): the tokens are split over workgroups
// that each write an fp32 partial sum, and a second launch adds them in order.
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "dispatch.hpp"
#include "training.hpp"

namespace galore {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int KS = 32;   // tokens of a stage

struct GradArgs {
    const void* dY;
    int64_t ldy, strideY;
    MxMatrix X;
    void* G;
    int64_t ldg, strideG;
    int T, m, n;
    int num_m, num_n, splits, per;   // per: stages of a split
    int accumulate;
};

// offset of column c of stage row kk: rows of W bf16, its 16-byte chunks permuted so
// that the four rows of a transposing read lie on different banks
template <int W>
__device__ __forceinline__ int stage_offset(int kk, int c) {
    const int x = W >= 128 ? 4 * (kk & 3) : 4 * ((kk >> 1) & 1);
    return kk * (2 * W) + 16 * ((c >> 3) ^ x) + 2 * (c & 7);
}

__device__ __forceinline__ bf16x4 read_tr(const unsigned char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<__attribute__((address_space(3))) bf16x4*>(
        reinterpret_cast<__attribute__((address_space(3))) unsigned char*>(reinterpret_cast<size_t>(p))));
}

// eight tokens kb .. kb + 7 (kb = 16 ks + 8 (lane / 32)) of column cb + lane % 32
template <int W>
__device__ __forceinline__ bf16x8 fragment(const unsigned char* stage, int cb, int ks, int lane) {
    const int L = lane & 15;
    const int c = cb + 16 * ((lane >> 4) & 1) + 4 * (L & 3);
    bf16x4 h[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) h[i] = read_tr(stage + stage_offset<W>(16 * ks + 8 * (lane >> 5) + 4 * i + (L >> 2), c));
    return __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = bf16_bits_rn(v); }

// eight entries of a row of dY as the planes' words
__device__ __forceinline__ void planes_of(const float (&x)[8], u32x4 (&w)[3]) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[p][i] = __builtin_amdgcn_perm(__float_as_uint(r[2 * i + 1]), __float_as_uint(r[2 * i]), 0x07060302u);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] -= __uint_as_float(__float_as_uint(r[i]) & 0xffff0000u);
    }
}

template <int TM, int TN, int WM, int WN, typename InT, typename OutT>
__global__ __launch_bounds__(64 * WM * WN, 2) void weight_grad_kernel(GradArgs g) {
    constexpr int PA = std::is_same<InT, float>::value ? 3 : 1;
    constexpr int MB = TM / WM / 32, NB = TN / WN / 32, kThreads = 64 * WM * WN;
    constexpr int kPlane = KS * TM * 2, kStageA = PA * kPlane, kStage = kStageA + KS * TN * 2;
    constexpr int QA = KS * TM / 8 / kThreads, QB = KS * TN / 16 / kThreads;   // groups of 8 gradients, of 16 codes
    static_assert(QA >= 1 && QB >= 1, "whole groups for each thread");
    __shared__ __attribute__((aligned(16))) unsigned char sm[2 * kStage];

    const int tiles = g.num_m * g.num_n;
    const int logical = xcd_logical_id(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
    const int slice = logical / tiles;                 // matrix and split
    const int64_t bz = slice / g.splits;
    const int split = slice - static_cast<int>(bz) * g.splits;
    int tm, tn;
    grouped_tile(logical - slice * tiles, g.num_m, g.num_n, 8, tm, tn);
    const int row0 = tm * TM, col0 = tn * TN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int first = split * g.per;
    const int stages = max(0, min(g.per, (g.T + KS - 1) / KS - first));

    const InT* dY = static_cast<const InT*>(g.dY) + bz * g.strideY;
    const uint8_t* codes = g.X.codes + bz * g.X.stride_q;
    const uint8_t* scales = g.X.scales + bz * g.X.stride_s;
    const int groups_n = 2 * static_cast<int>(mx_blocks(g.n));

    float ga[QA][8];
    u32x4 cb[QB];
    int sb[QB];
    auto load = [&](int stage) {
        const int t0 = (first + stage) * KS;
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            const int q = i * kThreads + tid, t = t0 + q / (TM / 8), c = row0 + 8 * (q % (TM / 8));
            load8(dY + static_cast<int64_t>(t) * g.ldy + c, t < g.T ? g.m - c : 0, ga[i]);
        }
#pragma unroll
        for (int i = 0; i < QB; ++i) {
            const int q = i * kThreads + tid, t = t0 + q / (TN / 16), c = min(col0 / 16 + q % (TN / 16), groups_n - 1);
            cb[i] = u32x4{0u, 0u, 0u, 0u};
            sb[i] = 0;
            if (t < g.T) {
                cb[i] = *reinterpret_cast<const u32x4*>(codes + static_cast<int64_t>(t) * g.X.ldq + 16 * c);
                sb[i] = scales[static_cast<int64_t>(t) * g.X.lds + (c >> 1)];
            }
        }
    };
    auto store = [&](int buf) {
        unsigned char* st = sm + buf * kStage;
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            const int q = i * kThreads + tid;
            unsigned char* dst = st + stage_offset<TM>(q / (TM / 8), 8 * (q % (TM / 8)));
            u32x4 w[3];
            planes_of(ga[i], w);
#pragma unroll
            for (int p = 0; p < PA; ++p) *reinterpret_cast<u32x4*>(dst + p * kPlane) = w[p];
        }
#pragma unroll
        for (int i = 0; i < QB; ++i) {
            const int q = i * kThreads + tid;
            const float unit = mx_unit<133>(sb[i]);
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = static_cast<float>(static_cast<int8_t>(cb[i][e >> 2] >> (8 * (e & 3)))) * unit;
            u32x4 w[2];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e >> 2][e & 3] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<u32x4*>(st + kStageA + stage_offset<TN>(q / (TN / 16), 16 * (q % (TN / 16)) + 8 * e)) = w[e];
        }
    };

    f32x16 acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.0f;

    if (stages > 0) {
        load(0);
        store(0);
    }
    for (int s = 0; s < stages; ++s) {
        __syncthreads();
        if (s + 1 < stages) load(s + 1);
        const unsigned char* st = sm + (s & 1) * kStage;
#pragma unroll
        for (int ks = 0; ks < KS / 16; ++ks) {
            bf16x8 a[PA][MB], b[NB];
#pragma unroll
            for (int p = 0; p < PA; ++p)
#pragma unroll
                for (int x = 0; x < MB; ++x) a[p][x] = fragment<TM>(st + p * kPlane, 32 * (wm * MB + x), ks, lane);
#pragma unroll
            for (int y = 0; y < NB; ++y) b[y] = fragment<TN>(st + kStageA, 32 * (wn * NB + y), ks, lane);
#pragma unroll
            for (int p = PA - 1; p >= 0; --p)
#pragma unroll
                for (int x = 0; x < MB; ++x)
#pragma unroll
                    for (int y = 0; y < NB; ++y)
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[p][x], b[y], acc[x][y], 0, 0, 0);
        }
        if (s + 1 < stages) store((s + 1) & 1);
    }

    OutT* G = static_cast<OutT*>(g.G) + slice * g.strideG;   // a split's own partial sum, or the matrix
    store_tile<MB, NB>(G, g.ldg, row0 + 32 * wm * MB + 4 * (lane >> 5), col0 + 32 * wn * NB, g.m, g.n, acc, g.accumulate != 0,
                       lane);
}

// The bulk of a large call: tiles of 256 x 256, four waves of 128 x 128 each, one to a
// SIMD, since a fragment read from LDS then feeds four matrix instructions and the
// LDS keeps up with them (96 KB a stage at 128 bytes a cycle against 1024 cycles of
// matrix work; waves of 128 x 64 would need 128 KB). With no second wave to fill a
// SIMD's gaps, the loop is laid out so that every wait is behind matrix work: while
// the 16 tokens of one step are multiplied, the fragments of the next step are read,
// and the stage after the next is decoded and written, from registers filled two
// stages ahead. One barrier a stage, between its two steps: past it, stage s + 1 is
// whole and stage s is in registers, so its buffer takes stage s + 2.
// dY bf16 with 16-byte aligned rows, m a multiple of 8, 32 tokens or more, and
// pitches below 2^25.
template <typename OutT>
__global__ __launch_bounds__(256, 1) void weight_grad_wide_kernel(GradArgs g) {
    constexpr int TM = 256, TN = 256, MB = 4, NB = 4;
    constexpr int kStageA = KS * TM * 2, kStage = kStageA + KS * TN * 2;
    constexpr int Q = 4;                               // groups of 8 gradients, and of 8 codes, of a thread and stage
    __shared__ __attribute__((aligned(16))) unsigned char sm[2 * kStage];

    const int tiles = g.num_m * g.num_n;
    const int logical = xcd_logical_id(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
    const int slice = logical / tiles;                 // matrix and split
    const int64_t bz = slice / g.splits;
    const int split = slice - static_cast<int>(bz) * g.splits;
    int tm, tn;
    grouped_tile(logical - slice * tiles, g.num_m, g.num_n, 8, tm, tn);
    const int row0 = tm * TM, col0 = tn * TN;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int first = split * g.per;
    const int stages = max(0, min(g.per, (g.T + KS - 1) / KS - first));

    // Group i of a stage: token 8 i + tid / 32, columns 8 (tid % 32) .. + 7; columns
    // past the last read its last group (never stored). A stage starts at a uniform
    // row, so that a load is a scalar address and an offset that stays. Past the end
    // of this split's tokens a stage starts at its last 32 instead: the order of
    // tokens within a sum is free, and those that an earlier stage has counted take
    // the unit zero.
    const int end = min(g.T, (first + g.per) * KS);
    const int tr = tid >> 5, ca = min(row0 + 8 * (tid & 31), g.m - 8);
    const int cb = min(col0 / 8 + (tid & 31), 4 * static_cast<int>(mx_blocks(g.n)) - 1);
    const unsigned char* dY = reinterpret_cast<const unsigned char*>(static_cast<const uint16_t*>(g.dY) + bz * g.strideY);
    const uint8_t* codes = g.X.codes + bz * g.X.stride_q;
    const uint8_t* scales = g.X.scales + bz * g.X.stride_s;
    const uint32_t ldy = static_cast<uint32_t>(g.ldy), ldq = static_cast<uint32_t>(g.X.ldq), lds = static_cast<uint32_t>(g.X.lds);
    uint32_t oa[Q], oc[Q], oe[Q];
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        oa[i] = 2 * ((8 * i + tr) * ldy + ca);
        oc[i] = (8 * i + tr) * ldq + 8 * cb;
        oe[i] = (8 * i + tr) * lds + (cb >> 2);
    }

    struct Regs {
        u32x4 a[Q];
        u32x2 c[Q];
        int e[Q];
    };
    const auto start = [&](int s) { return min((first + s) * KS, end - KS); };   // first token of a stage
    constexpr int64_t kAll = 0xffffffffll;   // every offset used lies inside the matrix: nothing is left to the bounds check
    auto load = [&](int s, Regs& r, int i) {
        const uint64_t t = static_cast<uint32_t>(start(s));
        r.a[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer_of(dY + 2 * t * ldy, kAll), oa[i], 0, 0));
        r.c[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(buffer_of(codes + t * ldq, kAll), oc[i], 0, 0));
        r.e[i] = __builtin_amdgcn_raw_buffer_load_b8(buffer_of(scales + t * lds, kAll), oe[i], 0, 0);
    };
    // where this thread's group 0 goes in a stage of either buffer: the others are 8 i
    // rows further, whose chunks are permuted alike
    const uint32_t put_a = stage_offset<TM>(tr, 8 * (tid & 31)), put_b = kStageA + stage_offset<TN>(tr, 8 * (tid & 31));
    auto store_a = [&](int buf, const Regs& r, int i) {
        *reinterpret_cast<u32x4*>(sm + put_a + (buf * kStage + 8 * i * (2 * TM))) = r.a[i];
    };
    auto store_b = [&](int buf, int i, const u32x4& w) {
        *reinterpret_cast<u32x4*>(sm + put_b + (buf * kStage + 8 * i * (2 * TN))) = w;
    };
    auto unit_of = [&](int s, const Regs& r, int i) {
        const int counted = (first + s) * KS - start(s);   // rows of the stage, by earlier ones
        return 8 * i + tr >= counted ? mx_unit<133>(r.e[i]) : 0.0f;
    };
    // codes 2 j and 2 j + 1 of a group as a word of two bf16 (exact)
    auto decode2 = [&](const Regs& r, int i, int j, float unit) {
        const int w = static_cast<int>(r.c[i][j >> 1]);
        const float lo = static_cast<float>(static_cast<int8_t>(j & 1 ? w >> 16 : w)) * unit;
        const float hi = (j & 1 ? static_cast<float>(w >> 24) : static_cast<float>(static_cast<int8_t>(w >> 8))) * unit;
        return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    };
    auto store = [&](int s, const Regs& r, int i) {
        const float unit = unit_of(s, r, i);
        store_a(s & 1, r, i);
        store_b(s & 1, i, u32x4{decode2(r, i, 0, unit), decode2(r, i, 1, unit), decode2(r, i, 2, unit), decode2(r, i, 3, unit)});
    };
    // the fragments of a step: 0 .. 3 those of dY, 4 .. 7 those of the checkpoint
    struct Frags {
        bf16x4 h[MB + NB][2];
        __device__ __forceinline__ bf16x8 get(int j) const {
            return __builtin_shufflevector(h[j][0], h[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    // where fragment j starts: the permutation of chunks depends on j and the lane
    // alone, so that the other reads of it are at fixed distances
    uint32_t at[MB + NB];
#pragma unroll
    for (int j = 0; j < MB + NB; ++j) {
        const int L = lane & 15;
        const int c = 32 * (j < MB ? wm * MB + j : wn * NB + j - MB) + 16 * ((lane >> 4) & 1) + 4 * (L & 3);
        at[j] = (j < MB ? 0 : kStageA) + stage_offset<TM>(8 * (lane >> 5) + (L >> 2), c);
    }
    static_assert(TM == TN, "one stage row for both");
    // read k (0 .. 15) of a step's fragments, those first that are multiplied first
    auto fetch = [&](int buf, int ks, Frags& f, int k) {
        constexpr int order[MB + NB] = {0, 4, 5, 6, 7, 1, 2, 3};
        const int j = order[k >> 1], h = k & 1;
        f.h[j][h] = read_tr(sm + at[j] + (buf * kStage + (16 * ks + 4 * h) * (2 * TM)));
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.0f;
    auto multiply = [&](const Frags& f, int k) {
        const int x = k / NB, y = k % NB;
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.get(x), f.get(MB + y), acc[x][y], 0, 0, 0);
    };

    Frags f0, f1;
    Regs r0, r1;
    if (stages > 0) {
#pragma unroll
        for (int i = 0; i < Q; ++i) load(0, r0, i);
#pragma unroll
        for (int i = 0; i < Q; ++i) load(1, r1, i);
#pragma unroll
        for (int i = 0; i < Q; ++i) store(0, r0, i);
#pragma unroll
        for (int i = 0; i < Q; ++i) store(1, r1, i);
        // in the order of the loop, which waits for the older ones alone
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            load(2, r0, i);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            load(3, r1, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k) fetch(0, 0, f0, k);
#pragma unroll
        for (int k = 0; k < 16; ++k) multiply(f0, k);
#pragma unroll
        for (int k = 0; k < 16; ++k) fetch(0, 1, f1, k);
        __syncthreads();
    }
    // between two barriers: step 1 of stage s, step 0 of stage s + 1; stage s + 2
    // from `r` to LDS, stage s + 4 to `r`. Each of the 32 matrix instructions leaves
    // the issue slots of 32 cycles to what stands behind it here; left to the
    // compiler, the reads and the decoding stand in blocks of their own and the
    // matrix unit waits for them. Nothing of the LDS is pending at the barrier.
    // (Past the last stage everything still runs, on units of zero: two steps of
    // matrix work for each split of a tile.)
    auto turn = [&](int s, auto buffer, Regs& r) {
        constexpr int cur = decltype(buffer)::value, next = cur ^ 1;   // buffers of stages s and s + 2, and of s + 1
        float unit = 0.0f;
        u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            if (k < 16) {
                multiply(f1, k);
                fetch(next, 0, f0, k);
            } else {
                multiply(f0, k - 16);
                if (k < 24) {
                    fetch(next, 1, f1, 2 * (k - 16));
                    fetch(next, 1, f1, 2 * (k - 16) + 1);
                }
            }
            if (k < 24 && k % 3 != 2) {                // decoding: two codes of group i
                const int piece = k / 3 * 2 + k % 3, i = piece >> 2, j = piece & 3;
                if (j == 0) unit = unit_of(s + 2, r, i);
                w[j] = decode2(r, i, j, unit);
                if (j == 3) store_b(cur, i, w);
            }
            if (k < 24 && k % 6 == 2) store_a(cur, r, k / 6);
            if (k >= 24 && k % 2 == 0) load(s + 4, r, (k - 24) / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
    };
    for (int s = 0; s < stages; s += 2) {
        turn(s, std::integral_constant<int, 0>(), r0);
        turn(s + 1, std::integral_constant<int, 1>(), r1);
    }

    OutT* G = static_cast<OutT*>(g.G) + slice * g.strideG;   // a split's own partial sum, or the matrix
    store_tile<MB, NB>(G, g.ldg, row0 + 32 * wm * MB + 4 * (lane >> 5), col0 + 32 * wn * NB, g.m, g.n, acc, g.accumulate != 0,
                       lane);
}

// G = sum of the splits' partial sums (+ G), four entries a thread
template <typename OutT>
__global__ __launch_bounds__(256) void join_kernel(const float* part, int splits, OutT* Gb, int64_t ldg, int64_t strideG,
                                                   int64_t m, int64_t n, int accumulate) {
    const int64_t c = 4 * (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x);
    const int64_t b = blockIdx.z;
    if (c >= n) return;
    for (int64_t r = first_row(); r < m; r += row_step()) {
        const float* p = part + (b * splits * m + r) * n + c;
        const int valid = static_cast<int>(min(n - c, static_cast<int64_t>(4)));
        float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < splits; ++k, p += m * n) {
            if (valid == 4) {
                const f32x4 v = *reinterpret_cast<const f32x4_a4*>(p);
    #pragma unroll
                for (int e = 0; e < 4; ++e) s[e] += v[e];
            } else {
    #pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < valid) s[e] += p[e];
            }
        }
        OutT* G = Gb + b * strideG + r * ldg + c;
    #pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < valid) put(G + e, accumulate ? s[e] + to_f32(G[e]) : s[e]);
    }
}

template <int TM, int TN, int WM, int WN, typename InT, typename OutT>
hipError_t launch_tiles(GradArgs g, int batch, hipStream_t stream) {
    g.num_m = (g.m + TM - 1) / TM;
    g.num_n = (g.n + TN - 1) / TN;
    const int64_t total = static_cast<int64_t>(g.num_m) * g.num_n * g.splits * batch;
    if (total >= 1 << 24) return hipErrorInvalidValue;   // work-items along x fit 32 bits
    hipLaunchKernelGGL((weight_grad_kernel<TM, TN, WM, WN, InT, OutT>), dim3(static_cast<unsigned>(total)),
                       dim3(64 * WM * WN), 0, stream, g);
    return hipGetLastError();
}

template <typename InT, typename OutT>
hipError_t launch(GradArgs g, bool wide, int batch, hipStream_t stream) {
    if (!wide) return launch_tiles<128, 128, 2, 2, InT, OutT>(g, batch, stream);
    g.num_m = (g.m + 255) / 256;
    g.num_n = (g.n + 255) / 256;
    const int64_t total = static_cast<int64_t>(g.num_m) * g.num_n * g.splits * batch;
    if (total >= 1 << 24) return hipErrorInvalidValue;
    hipLaunchKernelGGL((weight_grad_wide_kernel<OutT>), dim3(static_cast<unsigned>(total)), dim3(256), 0, stream, g);
    return hipGetLastError();
}

template <typename InT>
hipError_t launch_in(const WeightGradArgs& a, GradArgs g, bool wide, int batch, hipStream_t stream) {
    if (g.splits > 1) {
        g.G = a.part;
        g.ldg = a.n;
        g.strideG = a.m * a.n;
        g.accumulate = 0;
        const hipError_t e = launch<InT, float>(g, wide, batch, stream);
        if (e != hipSuccess) return e;
        const RowGrid r = row_grid(a.m, (a.n + 3) / 4, batch);
        if (a.g_bf16)
            hipLaunchKernelGGL(join_kernel<bf16_t>, r.grid, r.block, 0, stream, a.part, g.splits, static_cast<bf16_t*>(a.G),
                               a.ldg, a.strideG, a.m, a.n, a.accumulate ? 1 : 0);
        else
            hipLaunchKernelGGL(join_kernel<float>, r.grid, r.block, 0, stream, a.part, g.splits, static_cast<float*>(a.G),
                               a.ldg, a.strideG, a.m, a.n, a.accumulate ? 1 : 0);
        return hipGetLastError();
    }
    return a.g_bf16 ? launch<InT, bf16_t>(g, wide, batch, stream) : launch<InT, float>(g, wide, batch, stream);
}

constexpr int64_t kMaxPitch = int64_t{1} << 25;   // of the wide kernel's 32-bit offsets within a stage

bool wide_ok(const WeightGradArgs& a, int batch) {
    return a.dy_bf16 && a.T >= KS && a.m % 8 == 0 && a.ldy % 8 == 0 && (batch == 1 || a.strideY % 8 == 0) &&
           reinterpret_cast<uintptr_t>(a.dY) % 16 == 0 && a.ldy < kMaxPitch && a.X.ldq < kMaxPitch && a.X.lds < kMaxPitch;
}

}  // namespace

// the largest number of splits that a call of these sizes takes, whatever its type and alignment
int weight_grad_splits(int64_t T, int64_t m, int64_t n, int64_t batch) {
    return std::max(weight_grad_plan(T, m, n, batch, T >= KS && m % 8 == 0, false).splits,
                    std::max(weight_grad_plan(T, m, n, batch, false, false).splits,
                             weight_grad_plan(T, m, n, batch, false, true).splits));
}

hipError_t launch_weight_grad(const WeightGradArgs& a, int batch, hipStream_t stream) {
    const GradPlan plan = weight_grad_plan(a.T, a.m, a.n, batch, wide_ok(a, batch), !a.dy_bf16);
    const int stages = static_cast<int>((a.T + KS - 1) / KS), splits = a.part != nullptr ? plan.splits : 1;
    const GradArgs g{a.dY,  a.ldy, a.strideY, a.X, a.G, a.ldg, a.strideG, static_cast<int>(a.T), static_cast<int>(a.m),
                     static_cast<int>(a.n), 0, 0, splits, (stages + splits - 1) / splits, a.accumulate ? 1 : 0};
    return a.dy_bf16 ? launch_in<bf16_t>(a, g, plan.wide, batch, stream) : launch_in<float>(a, g, plan.wide, batch, stream);
}

}  // namespace galore
