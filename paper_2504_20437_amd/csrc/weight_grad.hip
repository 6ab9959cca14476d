// Weight gradient from an 8-bit checkpoint: G = dY^T X (+ G), the sum over the
// tokens of the incoming gradient's outer products with the layer's input, read
// from its codes.
//
// Both operands have the tokens, the axis of the sum, as their rows. A stage of
// 32 tokens of each is held in LDS as it lies in memory (the checkpoint decoded
// to bfloat16, exactly, on its way there) and the transposing LDS reads hand the
// matrix cores eight tokens of one column. An fp32 gradient is cut into three
// bfloat16 planes, x = h1 + h2 + h3 exactly (3 x 8 bits of its 24; what lies below
// 2^-133, bfloat16's least step, is lost), and takes three products; sums are held in
// fp32.
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
__device__ __forceinline__ void planes_of(const Eight<bf16_t>& x, u32x4 (&w)[1]) { w[0] = x.w; }
__device__ __forceinline__ void planes_of(const Eight<float>& x, u32x4 (&w)[3]) {
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
    constexpr int BUFS = PA == 3 ? 1 : 2;   // three planes: one stage in LDS, so that three workgroups fit a CU, not two
                                            // (509 tokens, 2048 x 5461: 52 us with two stages, 45 with one)
    constexpr int kPlane = KS * TM * 2, kStageA = PA * kPlane, kStage = kStageA + KS * TN * 2;
    constexpr int QA = KS * TM / 8 / kThreads, QB = KS * TN / 16 / kThreads;   // groups of 8 gradients, of 16 codes
    static_assert(QA >= 1 && QB >= 1, "whole groups for each thread");
    __shared__ __attribute__((aligned(16))) unsigned char sm[BUFS * kStage];

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

    Eight<InT> ga[QA];
    u32x4 cb[QB];
    int sb[QB];
    auto load = [&](int stage) {
        const int t0 = (first + stage) * KS;
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            const int q = i * kThreads + tid, t = t0 + q / (TM / 8), c = row0 + 8 * (q % (TM / 8));
            ga[i].load(dY + static_cast<int64_t>(t) * g.ldy, t < g.T ? c : g.m, g.m);   // past the tokens: zeros
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
        unsigned char* st = sm + (BUFS == 2 ? buf * kStage : 0);
        if (row0 + TM > g.m) {
#pragma unroll
            for (int i = 0; i < QA; ++i) ga[i].settle(row0 + 8 * ((i * kThreads + tid) % (TM / 8)), g.m);
        }
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            const int q = i * kThreads + tid;
            unsigned char* dst = st + stage_offset<TM>(q / (TM / 8), 8 * (q % (TM / 8)));
            u32x4 w[PA];
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
        const unsigned char* st = sm + (BUFS == 2 ? (s & 1) * kStage : 0);
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
        if (BUFS == 1) __syncthreads();
        if (s + 1 < stages) store((s + 1) & 1);
    }

    OutT* G = static_cast<OutT*>(g.G) + slice * g.strideG;   // a split's own partial sum, or the matrix
    store_tile<MB, NB>(G, g.ldg, row0 + 32 * wm * MB + 4 * (lane >> 5), col0 + 32 * wn * NB, g.m, g.n, acc, g.accumulate != 0,
                       lane);
}

// The bulk of a large call: four waves, one to a SIMD, of 128 x 128 outputs each (tiles
// of 256 x 256; with an fp32 gradient 64 x 128, tiles of 128 x 256), since a fragment
// read from LDS then feeds four matrix instructions and the LDS keeps up with them (96
// KB a stage at 128 bytes a cycle against 1024 cycles of matrix work; waves of 128 x 64
// would need 128 KB). With no second wave to fill a SIMD's gaps, the loop is laid out
// so that every wait is behind matrix work: while the 16 tokens of one step are
// multiplied, the fragments of the next step are read, and the stage after the next is
// decoded and written, from registers filled two stages ahead. One barrier a stage,
// between its two steps: past it, stage s + 1 is whole and stage s is in registers, so
// its buffer takes stage s + 2.
// 8192 tokens, 11008 x 4096, bf16: 713 to 742 us, 1.0 PFLOP/s, the matrix units busy 41%
// of the cycles; 4096, 4096 x 4096: 135 to 146; fp32, 4096 x 4096 and 8192 tokens: 694 to
// 709, 388 to 396 TFLOP/s (three times that in matrix products). Time (of 742) is taken by whatever stands beside the matrix work, not
// by one of them: without the loads 593 us, the decoding 626, both 552, the LDS writes
// too 479, matrix work alone 463; with every load a cache hit, four stages in flight or
// operands transposed on their way in and read by plain 16-byte reads (half the LDS
// time) 742 to 776.
// 32 tokens or more, rows of dY on 4 bytes, pitches below 2^25.
template <typename InT, typename OutT>
__global__ __launch_bounds__(256, 1) void weight_grad_wide_kernel(GradArgs g) {
    constexpr bool F32 = std::is_same<InT, float>::value;
    constexpr int PA = F32 ? 3 : 1, TM = F32 ? 128 : 256, TN = 256, MB = TM / 64, NB = 4;
    constexpr int kPlane = KS * TM * 2, kStageA = PA * kPlane, kStage = kStageA + KS * TN * 2;
    constexpr int W = TM / 8;                          // threads along a token's gradients
    constexpr int QA = KS * TM / 8 / 256, QB = 4;      // groups of 8 gradients, and of 8 codes, of a thread and stage
    constexpr int RA = 256 / W;                        // tokens between a thread's groups of gradients
    constexpr int F = PA * MB + NB;                    // fragments of a step
    constexpr int N = PA * MB * NB;                    // matrix instructions of a step
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

    // Group i of a stage: token RA i + tid / W of dY (8 i + tid / 32 of the codes),
    // eight columns. Those past a row's end read on into the next row, or into the
    // bounds check at the matrix's end, and are never stored. A stage starts at a
    // uniform row, so that a load is a scalar address and an offset that stays. Past
    // the end of this split's tokens a stage starts at its last 32 instead: the order
    // of tokens within a sum is free, and those that an earlier stage has counted take
    // the unit zero.
    const int end = min(g.T, (first + g.per) * KS);
    const int ta = tid / W, tb = tid >> 5;
    const int cb = min(col0 / 8 + (tid & 31), 4 * static_cast<int>(mx_blocks(g.n)) - 1);
    const InT* dY = static_cast<const InT*>(g.dY) + bz * g.strideY;
    const uint8_t* codes = g.X.codes + bz * g.X.stride_q;
    const uint8_t* scales = g.X.scales + bz * g.X.stride_s;
    const uint32_t ldy = static_cast<uint32_t>(g.ldy), ldq = static_cast<uint32_t>(g.X.ldq), lds = static_cast<uint32_t>(g.X.lds);
    uint32_t oa[QA], oc[QB], oe[QB];
#pragma unroll
    for (int i = 0; i < QA; ++i) oa[i] = sizeof(InT) * ((RA * i + ta) * ldy + row0 + 8 * (tid % W));
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        oc[i] = (8 * i + tb) * ldq + 8 * cb;
        oe[i] = (8 * i + tb) * lds + (cb >> 2);
    }

    struct Regs {
        u32x4 a[QA][F32 ? 2 : 1];
        u32x2 c[QB];
        int e[QB];
    };
    const auto start = [&](int s) { return min((first + s) * KS, end - KS); };   // first token of a stage
    constexpr int64_t kAll = 0xffffffffll;   // every offset lies inside the codes: nothing is left to the bounds check
    auto load_a = [&](int s, Regs& r, int i) {
        const int64_t t = start(s);
        // in whole words: the last one may hold a single bf16
        const int64_t bytes = (static_cast<int64_t>(sizeof(InT)) * ((g.T - 1 - t) * ldy + g.m) + 3) & ~int64_t{3};
        const __amdgpu_buffer_rsrc_t rows = buffer_of(dY + t * ldy, bytes);
        r.a[i][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, oa[i], 0, 0));
        if constexpr (F32) r.a[i][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, oa[i] + 16, 0, 0));
    };
    auto load_b = [&](int s, Regs& r, int i) {
        const uint64_t t = static_cast<uint32_t>(start(s));
        r.c[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(buffer_of(codes + t * ldq, kAll), oc[i], 0, 0));
        r.e[i] = __builtin_amdgcn_raw_buffer_load_b8(buffer_of(scales + t * lds, kAll), oe[i], 0, 0);
    };
    // where this thread's group 0 goes in a stage of either buffer: the others are some
    // rows (a multiple of 8) further, whose chunks are permuted alike
    const uint32_t put_a = stage_offset<TM>(ta, 8 * (tid % W)), put_b = kStageA + stage_offset<TN>(tb, 8 * (tid & 31));
    auto store_a = [&](int buf, int i, int p, const u32x4& w) {
        *reinterpret_cast<u32x4*>(sm + put_a + (buf * kStage + p * kPlane + RA * i * (2 * TM))) = w;
    };
    auto store_b = [&](int buf, int i, const u32x4& w) {
        *reinterpret_cast<u32x4*>(sm + put_b + (buf * kStage + 8 * i * (2 * TN))) = w;
    };
    auto unit_of = [&](int s, const Regs& r, int i) {
        const int counted = (first + s) * KS - start(s);   // rows of the stage, by earlier ones
        return 8 * i + tb >= counted ? mx_unit<133>(r.e[i]) : 0.0f;
    };
    // codes 2 j and 2 j + 1 of a group as a word of two bf16 (exact)
    auto decode2 = [&](const Regs& r, int i, int j, float unit) {
        const int w = static_cast<int>(r.c[i][j >> 1]);
        const float lo = static_cast<float>(static_cast<int8_t>(j & 1 ? w >> 16 : w)) * unit;
        const float hi = (j & 1 ? static_cast<float>(w >> 24) : static_cast<float>(static_cast<int8_t>(w >> 8))) * unit;
        return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    };
    // word j of the planes of a group of dY
    auto plane2 = [&](const Regs& r, int i, int j, u32x4 (&w)[PA]) {
        if constexpr (F32) {
            float lo = __uint_as_float(r.a[i][j >> 1][2 * (j & 1)]), hi = __uint_as_float(r.a[i][j >> 1][2 * (j & 1) + 1]);
#pragma unroll
            for (int p = 0; p < PA; ++p) {
                w[p][j] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
                lo -= __uint_as_float(__float_as_uint(lo) & 0xffff0000u);
                hi -= __uint_as_float(__float_as_uint(hi) & 0xffff0000u);
            }
        } else {
            w[0][j] = r.a[i][0][j];
        }
    };
    auto store = [&](int s, const Regs& r) {
#pragma unroll
        for (int i = 0; i < QA; ++i) {
            u32x4 w[PA];
#pragma unroll
            for (int j = 0; j < 4; ++j) plane2(r, i, j, w);
#pragma unroll
            for (int p = 0; p < PA; ++p) store_a(s & 1, i, p, w[p]);
        }
#pragma unroll
        for (int i = 0; i < QB; ++i) {
            const float unit = unit_of(s, r, i);
            store_b(s & 1, i, u32x4{decode2(r, i, 0, unit), decode2(r, i, 1, unit), decode2(r, i, 2, unit), decode2(r, i, 3, unit)});
        }
    };
    // in the order of the loop, which waits for the older loads alone
    auto load = [&](int s, Regs& r) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < QA) load_a(s, r, i);
            load_b(s, r, i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the fragments of a step: those of dY, plane by plane, then those of the checkpoint
    struct Frags {
        bf16x4 h[F][2];
        __device__ __forceinline__ bf16x8 get(int j) const {
            return __builtin_shufflevector(h[j][0], h[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    // where a block's fragments start: the permutation of chunks depends on the block and
    // the lane alone, so that the other reads (steps, planes, buffers) are at fixed distances
    uint32_t at[MB + NB];
#pragma unroll
    for (int j = 0; j < MB + NB; ++j) {
        const int L = lane & 15, kk = 8 * (lane >> 5) + (L >> 2), c = 16 * ((lane >> 4) & 1) + 4 * (L & 3);
        at[j] = j < MB ? stage_offset<TM>(kk, 32 * (wm * MB + j) + c) : kStageA + stage_offset<TN>(kk, 32 * (wn * NB + j - MB) + c);
    }
    // read k (0 .. 2 F - 1) of a step's fragments, those first that are multiplied first:
    // the last plane's block 0, the checkpoint's blocks, the rest from the last plane on
    auto fetch = [&](int buf, int ks, Frags& f, int k) {
        const int o = k >> 1, h = k & 1;
        const bool mine = o >= 1 && o <= NB;           // of the checkpoint
        const int q = mine ? 0 : o == 0 ? 0 : o - NB;  // q-th block of dY, planes from the last
        const int p = PA - 1 - q / MB, x = q % MB, y = o - 1;
        const int j = mine ? PA * MB + y : p * MB + x;
        const uint32_t from = mine ? at[MB + y] : at[x];
        f.h[j][h] = read_tr(sm + from + (buf * kStage + (mine ? 0 : p * kPlane) + (16 * ks + 4 * h) * 2 * (mine ? TN : TM)));
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.0f;
    auto multiply = [&](const Frags& f, int k) {
        const int p = PA - 1 - k / (MB * NB), x = k / NB % MB, y = k % NB;
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.get(p * MB + x), f.get(PA * MB + y), acc[x][y], 0, 0, 0);
    };

    Frags f0, f1;
    Regs r0, r1;
    if (stages > 0) {
        load(0, r0);
        load(1, r1);
        store(0, r0);
        store(1, r1);
        __builtin_amdgcn_sched_barrier(0);
        load(2, r0);
        load(3, r1);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2 * F; ++k) fetch(0, 0, f0, k);
#pragma unroll
        for (int k = 0; k < N; ++k) multiply(f0, k);
#pragma unroll
        for (int k = 0; k < 2 * F; ++k) fetch(0, 1, f1, k);
        __syncthreads();
    }
    // between two barriers: step 1 of stage s, step 0 of stage s + 1; stage s + 2
    // from `r` to LDS, stage s + 4 to `r`. Each of the matrix instructions leaves the
    // issue slots of 32 cycles to what stands behind it here; left to the compiler, the
    // reads and the decoding stand in blocks of their own and the matrix unit waits for
    // them. Nothing of the LDS is pending at the barrier. (Past the last stage everything
    // still runs, on units of zero: two steps of matrix work for each split of a tile.)
    constexpr int kWork = 2 * N - 8;                   // instructions by which all is decoded: the loads follow
    constexpr int kPieces = 4 * (QA * (F32 ? 1 : 0) + QB);
    auto turn = [&](int s, auto buffer, Regs& r) {
        constexpr int cur = decltype(buffer)::value, next = cur ^ 1;   // buffers of stages s and s + 2, and of s + 1
        float unit = 0.0f;
        u32x4 w = {0u, 0u, 0u, 0u}, wa[PA];
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) {
            if (k < N) {
                multiply(f1, k);
                if (k < 2 * F) fetch(next, 0, f0, k);
            } else {
                multiply(f0, k - N);
                if (2 * (k - N) < 2 * F) {
                    fetch(next, 1, f1, 2 * (k - N));
                    fetch(next, 1, f1, 2 * (k - N) + 1);
                }
            }
            // pieces of two values, evenly over the first kWork instructions
            const int piece = (k + 1) * kPieces / kWork - 1;
            if (k < kWork && piece >= 0 && piece != k * kPieces / kWork - 1) {
                const int i = piece >> 2, j = piece & 3;
                if (i < QB) {
                    if (j == 0) unit = unit_of(s + 2, r, i);
                    w[j] = decode2(r, i, j, unit);
                    if (j == 3) store_b(cur, i, w);
                } else if constexpr (F32) {
                    plane2(r, i - QB, j, wa);
                    if (j == 3) {
#pragma unroll
                        for (int p = 0; p < PA; ++p) store_a(cur, i - QB, p, wa[p]);
                    }
                }
            }
            if constexpr (!F32) {
                if (k < kWork && k % 6 == 2) store_a(cur, k / 6, 0, r.a[k / 6][0]);
            }
            if (k >= kWork && k % 2 == 0) {
                const int i = (k - kWork) / 2;
                if (i < QA) load_a(s + 4, r, i);
                load_b(s + 4, r, i);
            }
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

// the kernel over the tiles of every matrix, in as many launches as their number takes (one but for long
// batches of large gradients)
template <typename InT, typename OutT>
hipError_t launch_tiles(void (*kernel)(GradArgs), GradArgs g, int tile_m, int tile_n, int batch, hipStream_t stream) {
    g.num_m = (g.m + tile_m - 1) / tile_m;
    g.num_n = (g.n + tile_n - 1) / tile_n;
    const int64_t tiles = static_cast<int64_t>(g.num_m) * g.num_n * g.splits;
    const int step = matrices_a_launch(tiles, batch);
    if (step == 0) return hipErrorInvalidValue;
    for (int b = 0; b < batch; b += step) {
        GradArgs part = g;
        part.dY = static_cast<const InT*>(g.dY) + b * g.strideY;
        part.X = g.X.from(b);
        part.G = static_cast<OutT*>(g.G) + static_cast<int64_t>(b) * g.splits * g.strideG;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tiles * std::min(step, batch - b))), dim3(256), 0, stream, part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename InT, typename OutT>
hipError_t launch(const GradArgs& g, bool wide, int batch, hipStream_t stream) {
    if (!wide) return launch_tiles<InT, OutT>(weight_grad_kernel<128, 128, 2, 2, InT, OutT>, g, 128, 128, batch, stream);
    return launch_tiles<InT, OutT>(weight_grad_wide_kernel<InT, OutT>, g, std::is_same<InT, float>::value ? 128 : 256, 256,
                                   batch, stream);
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
    const bool words = !a.dy_bf16 || (a.ldy % 2 == 0 && (batch == 1 || a.strideY % 2 == 0) && reinterpret_cast<uintptr_t>(a.dY) % 4 == 0);
    return words && a.T >= KS && a.ldy < kMaxPitch && a.X.ldq < kMaxPitch && a.X.lds < kMaxPitch;
}

}  // namespace

// the largest number of splits that a call of these sizes takes, whatever its type and alignment
int weight_grad_splits(int64_t T, int64_t m, int64_t n, int64_t batch) {
    int most = 1;
    for (const bool fp32 : {false, true})
        for (const bool wide : {false, true}) most = std::max(most, weight_grad_plan(T, m, n, batch, wide && T >= KS, fp32).splits);
    return most;
}

hipError_t launch_weight_grad(const WeightGradArgs& a, int batch, hipStream_t stream) {
    const GradPlan plan = weight_grad_plan(a.T, a.m, a.n, batch, wide_ok(a, batch), !a.dy_bf16);
    const int stages = static_cast<int>((a.T + KS - 1) / KS), splits = a.part != nullptr ? plan.splits : 1;
    const GradArgs g{a.dY,  a.ldy, a.strideY, a.X, a.G, a.ldg, a.strideG, static_cast<int>(a.T), static_cast<int>(a.m),
                     static_cast<int>(a.n), 0, 0, splits, (stages + splits - 1) / splits, a.accumulate ? 1 : 0};
    return a.dy_bf16 ? launch_in<bf16_t>(a, g, plan.wide, batch, stream) : launch_in<float>(a, g, plan.wide, batch, stream);
}

}  // namespace galore
