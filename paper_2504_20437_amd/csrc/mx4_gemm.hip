// Product of two matrices of microscaled 4-bit floating point, C = A B^T, on the
// scaled matrix cores (v_mfma_scale_f32_*_f8f6f4): a lane's operand is one block
// of 32 codes (16 bytes) and the scale byte that goes with it, so codes and
// scales go from memory to the matrix unit as they are stored. Sums are held in
// fp32; a product of two codes and its scale is exact.
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "dispatch.hpp"
#include "training.hpp"

namespace galore {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(1))) void glb_void_t;

constexpr int kFp4 = 4;   // operand format of the matrix instruction: E2M1

__device__ const u32x4 kZeroBlock = {0u, 0u, 0u, 0u};

__device__ __forceinline__ i32x8 operand(u32x4 v) {
    return i32x8{static_cast<int>(v[0]), static_cast<int>(v[1]), static_cast<int>(v[2]), static_cast<int>(v[3]), 0, 0, 0, 0};
}

struct Mx4Args {
    MxMatrix A, B;
    void* C;
    int64_t ldc, strideC;
    int M, N, nblk;      // nblk: blocks of 32 along K
    int num_m, num_n;
};

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { p->bits = bf16_bits_rn(v); }

// wait until at most n direct loads of this wave are outstanding
template <int n>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
}
// `ahead`: stages of L loads issued after the one needed now (0 .. S - 2)
template <int L, int S>
__device__ __forceinline__ void wait_stages(int ahead) {
    if constexpr (S >= 4) {
        if (ahead >= 2) {
            wait_loads<2 * L>();
            return;
        }
    }
    if constexpr (S >= 3) {
        if (ahead >= 1) {
            wait_loads<L>();
            return;
        }
    }
    wait_loads<0>();
}

// Tile of TM x TN outputs, stages of 8 blocks (256 codes, 128 bytes a row) loaded
// straight to LDS, S - 1 of them in flight while one is multiplied. Chunk c (16 bytes) of stage row r sits
// at slot c ^ ((r >> 1) & 7): the 16 lanes of a fragment read (16 rows, one
// chunk) fall on distinct banks. The order of k within a stage is free as long as
// A and B share it: lane half h takes blocks 4 h .. 4 h + 3 one after the other,
// so that one dword holds the scales of its four steps.
template <int MB, int NB, int WM, int WN, int S, typename OutT>
__global__ __launch_bounds__(64 * WM * WN, 2) void mx4_tile_gemm_kernel(Mx4Args g) {
    constexpr int TM = 32 * MB * WM, TN = 32 * NB * WN, kRows = TM + TN, kWaves = WM * WN;
    constexpr int kData = kRows * 128, kStage = kData + kRows * 8;
    constexpr int LD = kData / 1024 / kWaves;        // direct loads of codes per wave and stage (8 rows each)
    constexpr int LS = kRows / 32 / kWaves;          // and of scales (32 rows each)
    static_assert(kData % (1024 * kWaves) == 0 && kRows % (32 * kWaves) == 0, "whole direct loads per wave");
    __shared__ __attribute__((aligned(16))) unsigned char sm[S * kStage];

    const int tiles = g.num_m * g.num_n;
    const int logical = xcd_logical_id(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
    const int bz = logical / tiles;
    int tm, tn;
    grouped_tile(logical - bz * tiles, g.num_m, g.num_n, 8, tm, tn);
    const int row0 = tm * TM, col0 = tn * TN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int l32 = lane & 31, lk = lane >> 5;

    const uint8_t* src[LD];
    int chunk[LD];
#pragma unroll
    for (int i = 0; i < LD; ++i) {
        const int sr = 8 * (wave * LD + i) + (lane >> 3);
        chunk[i] = (lane & 7) ^ ((sr >> 1) & 7);
        const bool isA = sr < TM;
        const MxMatrix& q = isA ? g.A : g.B;
        const int64_t r = isA ? min(row0 + sr, g.M - 1) : min(col0 + sr - TM, g.N - 1);
        src[i] = q.codes + bz * q.stride_q + r * q.ldq + 16 * chunk[i];
    }
    const uint8_t* ssrc[LS];
#pragma unroll
    for (int i = 0; i < LS; ++i) {
        const int sr = 32 * (wave * LS + i) + (lane >> 1);
        const bool isA = sr < TM;
        const MxMatrix& q = isA ? g.A : g.B;
        const int64_t r = isA ? min(row0 + sr, g.M - 1) : min(col0 + sr - TM, g.N - 1);
        ssrc[i] = q.scales + bz * q.stride_s + r * q.lds;
    }
    const int KT = (g.nblk + 7) / 8;
    const int last_dword = (g.nblk + 3) / 4 - 1;
    auto issue = [&](int buf, int kt) {
        unsigned char* base = sm + buf * kStage;
        const bool whole = 8 * kt + 8 <= g.nblk;   // blocks past the row's end read as zero codes
#pragma unroll
        for (int i = 0; i < LD; ++i) {
            const uint8_t* p = src[i] + static_cast<int64_t>(kt) * 128;
            if (!whole && 8 * kt + chunk[i] >= g.nblk) p = reinterpret_cast<const uint8_t*>(&kZeroBlock);
            __builtin_amdgcn_global_load_lds((glb_void_t*)p, (lds_void_t*)(base + (wave * LD + i) * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < LS; ++i) {
            const uint8_t* p = ssrc[i] + 4 * min(2 * kt + (lane & 1), last_dword);
            __builtin_amdgcn_global_load_lds((glb_void_t*)p, (lds_void_t*)(base + kData + (wave * LS + i) * 256), 4, 0, 0);
        }
    };

    f32x16 acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.0f;

    // scale bytes past the row's last block belong to zero codes, but could be
    // the NaN byte: mask of this lane's dword in the last stage
    const int tail = min(max(g.nblk - 8 * (KT - 1) - 4 * lk, 0), 4);
    const uint32_t tail_mask = tail == 4 ? 0xffffffffu : (1u << (8 * tail)) - 1u;

#pragma unroll
    for (int st = 0; st < S - 1; ++st)
        if (st < KT) issue(st, st);
    for (int kt = 0; kt < KT; ++kt) {
        // stage kt landed for this wave, then for every wave; past the barrier every
        // wave has also finished stage kt - 1, whose buffer is filled again
        wait_stages<LD + LS, S>(min(S - 2, KT - 1 - kt));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (kt + S - 1 < KT) issue((kt + S - 1) % S, kt + S - 1);
        const unsigned char* st = sm + (kt % S) * kStage;
        const uint32_t mask = kt == KT - 1 ? tail_mask : 0xffffffffu;
        int sa[MB], sb[NB];
#pragma unroll
        for (int x = 0; x < MB; ++x)
            sa[x] = static_cast<int>(*reinterpret_cast<const uint32_t*>(st + kData + (wm * 32 * MB + 32 * x + l32) * 8 + 4 * lk) & mask);
#pragma unroll
        for (int y = 0; y < NB; ++y)
            sb[y] = static_cast<int>(*reinterpret_cast<const uint32_t*>(st + kData + (TM + wn * 32 * NB + 32 * y + l32) * 8 + 4 * lk) & mask);
        // all of the stage's fragments first: their latency is paid once a stage
        u32x4 a[4][MB], b[4][NB];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 4 * lk + j;
#pragma unroll
            for (int x = 0; x < MB; ++x) {
                const int r = wm * 32 * MB + 32 * x + l32;
                a[j][x] = *reinterpret_cast<const u32x4*>(st + r * 128 + 16 * (c ^ ((r >> 1) & 7)));
            }
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                const int r = TM + wn * 32 * NB + 32 * y + l32;
                b[j][y] = *reinterpret_cast<const u32x4*>(st + r * 128 + 16 * (c ^ ((r >> 1) & 7)));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        auto step = [&](auto jc) {
            constexpr int j = decltype(jc)::value;
#pragma unroll
            for (int x = 0; x < MB; ++x)
#pragma unroll
                for (int y = 0; y < NB; ++y)
                    acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a[j][x]), operand(b[j][y]), acc[x][y],
                                                                                kFp4, kFp4, j, sa[x], j, sb[y]);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
    }

    OutT* C = static_cast<OutT*>(g.C) + bz * g.strideC;
    store_tile<MB, NB>(C, g.ldc, row0 + wm * 32 * MB + 4 * lk, col0 + wn * 32 * NB, g.M, g.N, acc, false, lane);
}

// The bulk of a large call: tiles of 256 x 256, four waves of 128 x 128, one to a
// SIMD: a stage of 256 codes a row is 64 matrix instructions a wave, 2150 cycles,
// against 196 KB through the LDS, 1530 cycles. With no second wave to fill a SIMD's
// gaps, the order is laid out so that every wait stands behind matrix work: a step's
// fragments are read while the step before it is multiplied, and the one barrier of
// a stage stands before its last step, whose fragments are in registers by then: past
// it the stage's buffer is free and takes the stage after the next, and the next
// stage is whole and its first fragments and scales are read.
// 8192 x 8192, k = 16384: 528 us, 4.17 PFLOP/s; 8192 x 11008, k = 4096: 214 to 231 us on
// the same operands call after call, 3.2 to 3.5 PFLOP/s, and 264 on others each time.
// Matrix instructions alone, on registers, reach 6.5 PFLOP/s on random codes (8.6 on
// zeros: the clock falls with the bits that toggle, to 1.65 GHz); a loop that spends
// fewer cycles a stage (workgroups that start at different stages) ran at a lower
// clock and was no faster. The rest is the tile's first loads and its stores, 20000 of
// 95000 cycles at k = 4096.
// Pitches below 2^22.
template <typename OutT>
__global__ __launch_bounds__(256, 1) void mx4_wide_gemm_kernel(Mx4Args g) {
    constexpr int TM = 256, TN = 256, MB = 4, NB = 4, kRows = TM + TN;
    constexpr int kStage = kRows * 128, kScales = kRows * 16;
    constexpr int LD = kStage / 1024 / 4, LS = kScales / 1024 / 4;   // direct loads of a wave: codes, scales
    static_assert(LD == 16 && LS == 2, "as they stand between the matrix instructions of a step");
    // two stages of codes, then two of scales
    __shared__ __attribute__((aligned(16))) unsigned char sm[2 * kStage + 2 * kScales];

    const int tiles = g.num_m * g.num_n;
    const int logical = xcd_logical_id(static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
    const int bz = logical / tiles;
    int tm, tn;
    grouped_tile(logical - bz * tiles, g.num_m, g.num_n, 8, tm, tn);
    const int row0 = tm * TM, col0 = tn * TN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int l32 = lane & 31, lk = lane >> 5;

    // waves 0 and 1 load the rows of A, 2 and 3 those of B
    const bool isA = wave < 2;
    const MxMatrix& q = isA ? g.A : g.B;
    const int64_t line0 = isA ? row0 : col0;
    const int lines = (isA ? g.M : g.N) - 1 - static_cast<int>(line0);   // last row there is, from line0
    // up to the end of the matrix's last row, and no further: the last stage of a row
    // may read past it
    const __amdgpu_buffer_rsrc_t rc = buffer_of(q.codes + bz * q.stride_q + line0 * q.ldq,
                                                lines * q.ldq + 16 * static_cast<int64_t>(g.nblk));
    const __amdgpu_buffer_rsrc_t rs = buffer_of(q.scales + bz * q.stride_s + line0 * q.lds,
                                                lines * q.lds + (g.nblk + 3) / 4 * 4);
    uint32_t oc[LD], os[LS];
    const int w2 = wave & 1;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
        const int r = 8 * (w2 * LD + i) + (lane >> 3);
        oc[i] = static_cast<uint32_t>(min(r, lines)) * static_cast<uint32_t>(q.ldq) + 16 * ((lane & 7) ^ ((r >> 1) & 7));
    }
#pragma unroll
    for (int i = 0; i < LS; ++i)
        os[i] = static_cast<uint32_t>(min(64 * (w2 * LS + i) + lane, lines)) * static_cast<uint32_t>(q.lds);
    const int KT = (g.nblk + 7) / 8;
    // The last stage of a row that is not whole goes on into what lies behind it, or
    // into the bounds check. Both operands' scale bytes are masked to zero there,
    // 2^-254 together, under which every product of codes is zero in fp32 (a code
    // itself is always finite).
    const int left = min(max(g.nblk - 8 * (KT - 1) - 4 * lk, 0), 4);   // of this lane's four in the last stage
    const uint32_t tail_mask = left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1u;
    // direct load i of stage kt (past the last one: the last again, never read): LD of
    // codes, LS of scales, of which a row takes the 16 bytes from the stage's eight on:
    // one load a row
    auto load = [&](int kt, int i) {
        const int st = min(kt, KT - 1);
        if (i < LD)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rc, (lds_void_t*)(sm + (kt & 1) * kStage + (wave * LD + i) * 1024), 16,
                                                     oc[i], st * 128, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (lds_void_t*)(sm + 2 * kStage + (kt & 1) * kScales + (wave * LS + i - LD) * 1024), 16, os[i - LD], st * 8, 0, 0);
    };

    struct Frags {
        u32x4 v[MB + NB];   // rows of A, rows of B
    };
    // chunk 4 lk + j of this lane's row of block 0 in the present buffer: the other
    // blocks are 32 rows (4 KB) further, whose chunks are permuted alike
    uint32_t at[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t o = l32 * 128 + 16 * ((4 * lk + j) ^ ((l32 >> 1) & 7));
        at[0][j] = o + wm * (32 * MB * 128);
        at[1][j] = o + (TM + wn * 32 * NB) * 128;
    }
    const uint32_t sat[2] = {static_cast<uint32_t>(2 * kStage + (wm * 32 * MB + l32) * 16 + 4 * lk),
                             static_cast<uint32_t>(2 * kStage + (TM + wn * 32 * NB + l32) * 16 + 4 * lk)};
    // those first that are multiplied first: A 0, B 0 .. 3, A 1 .. 3
    constexpr int order[MB + NB] = {0, 4, 5, 6, 7, 1, 2, 3};
    auto fetch = [&](int j, Frags& f, int k) {
        const int b = order[k];
        f.v[b] = *reinterpret_cast<const u32x4*>(sm + at[b >> 2][j] + (b & 3) * 4096);
    };
    int c[MB + NB], cn[MB + NB];   // scales of the present stage and the next
    auto fetch_scale = [&](int kt, int b) {
        cn[b] = *reinterpret_cast<const int*>(sm + sat[b >> 2] + (kt & 1) * kScales + (b & 3) * 512);
    };
    f32x16 acc[MB][NB];
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[x][y][v] = 0.0f;
    auto multiply = [&](auto jc, const Frags& f, int k) {
        constexpr int j = decltype(jc)::value;
        const int x = k / NB, y = k % NB;
        acc[x][y] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(f.v[x]), operand(f.v[MB + y]), acc[x][y], kFp4,
                                                                    kFp4, j, c[x], j, c[MB + y]);
    };
    // multiply step j from `f`, read step j + 1 to `n`
    auto step = [&](auto jc, const Frags& f, Frags& n, auto more) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            multiply(jc, f, k);
            if (k < 8) fetch(decltype(jc)::value + 1, n, k);
            more(k);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    Frags f0, f1;
#pragma unroll
    for (int i = 0; i < LD + LS; ++i) load(0, i);
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < LD / 2; ++i) load(1, i);   // the other half: in the loop's first step
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        fetch(0, f0, k);
        fetch_scale(0, k);
    }
    for (int kt = 0; kt < KT; ++kt) {
        const uint32_t mask = kt == KT - 1 ? tail_mask : 0xffffffffu;
#pragma unroll
        for (int b = 0; b < MB + NB; ++b) c[b] = static_cast<int>(static_cast<uint32_t>(cn[b]) & mask);
        __builtin_amdgcn_sched_barrier(0);
        step(std::integral_constant<int, 0>(), f0, f1, [&](int k) {
            if (k & 1) load(kt + 1, LD / 2 + (k >> 1));
            if (k >= 16 - LS) load(kt + 1, LD + k - (16 - LS));
        });
        step(std::integral_constant<int, 1>(), f1, f0, [](int) {});
        step(std::integral_constant<int, 2>(), f0, f1, [](int) {});
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const uint32_t turn = kt & 1 ? -kStage : kStage;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            at[0][j] += turn;
            at[1][j] += turn;
        }
        __builtin_amdgcn_sched_barrier(0);
        // (past the last stage these read what the other buffer holds, for nothing)
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            multiply(std::integral_constant<int, 3>(), f1, k);
            if (k < 8) {
                fetch(0, f0, k);
                fetch_scale(kt + 1, k);
            }
            if (k & 1) load(kt + 2, k >> 1);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no direct load outlives the workgroup's LDS
    OutT* C = static_cast<OutT*>(g.C) + bz * g.strideC;
    store_tile<MB, NB>(C, g.ldc, row0 + wm * 32 * MB + 4 * lk, col0 + wn * 32 * NB, g.M, g.N, acc, false, lane);
}

// Few rows of A (up to 16 MT): the weights B are read once, straight to
// registers, and bound the call. A wave takes 16 rows of B and a share of K; the
// waves of a workgroup share its 16 rows and join their sums in LDS in a fixed
// order, so that the chip is full whatever N is, with no second launch. M = 1, K =
// 4096: N = 11008 9.5 us (24 MB, 2.5 TB/s: the loads of one wave are all in flight at
// once, and their latency, the join and the launch are what is left), N = 4096 5.4.
template <int MT, typename OutT>
__global__ __launch_bounds__(1024) void mx4_few_rows_kernel(Mx4Args g) {
    __shared__ f32x4 part[16][MT][64];
    const int nw = blockDim.x >> 6;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, kg = lane >> 4;
    const int64_t bz = blockIdx.y;
    const int n0 = blockIdx.x * 16;
    const int steps = (g.nblk + 3) / 4;              // steps of four blocks, one to each group of 16 lanes
    const int per = (steps + nw - 1) / nw;
    const int first = wave * per, last = min(first + per, steps);
    const int64_t rb = min(n0 + l16, g.N - 1);
    const uint8_t* qb = g.B.codes + bz * g.B.stride_q + rb * g.B.ldq + 16 * kg;
    const uint8_t* sb = g.B.scales + bz * g.B.stride_s + rb * g.B.lds;
    const uint8_t* qa[MT];
    const uint8_t* sa[MT];
#pragma unroll
    for (int x = 0; x < MT; ++x) {
        const int64_t ra = min(16 * x + l16, g.M - 1);
        qa[x] = g.A.codes + bz * g.A.stride_q + ra * g.A.ldq + 16 * kg;
        sa[x] = g.A.scales + bz * g.A.stride_s + ra * g.A.lds;
    }
    f32x4 acc[MT];
#pragma unroll
    for (int x = 0; x < MT; ++x) acc[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int U = MT == 1 ? 8 : 4;               // steps whose loads are in flight together
    static_assert(MT <= 2, "up to 32 rows");
    for (int s0 = first; s0 < last; s0 += U) {
        u32x4 b[U], a[U][MT];
        uint32_t fb[U], fa[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u, steps - 1);    // steps past `last` are loaded and not used
            const int64_t off = 64 * static_cast<int64_t>(min(s, (g.nblk - 1 - kg) / 4));
            b[u] = *reinterpret_cast<const u32x4*>(qb + (kg < g.nblk ? off : -16 * static_cast<int64_t>(kg)));
            fb[u] = *reinterpret_cast<const uint32_t*>(sb + 4 * s);
#pragma unroll
            for (int x = 0; x < MT; ++x) {
                a[u][x] = *reinterpret_cast<const u32x4*>(qa[x] + (kg < g.nblk ? off : -16 * static_cast<int64_t>(kg)));
                fa[u][x] = *reinterpret_cast<const uint32_t*>(sa[x] + 4 * s);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u >= last) break;
            const bool in = 4 * (s0 + u) + kg < g.nblk;   // a block past the row's end: zero codes and scale
            const u32x4 zero = {0u, 0u, 0u, 0u};
            const i32x8 bv = operand(in ? b[u] : zero);
            const int sbv = in ? static_cast<int>((fb[u] >> (8 * kg)) & 255u) : 0;
#pragma unroll
            for (int x = 0; x < MT; ++x) {
                const i32x8 av = operand(in ? a[u][x] : zero);
                const int sav = in ? static_cast<int>((fa[u][x] >> (8 * kg)) & 255u) : 0;
                acc[x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bv, av, acc[x], kFp4, kFp4, 0, sbv, 0, sav);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < MT; ++x) part[wave][x][lane] = acc[x];
    __syncthreads();
    OutT* C = static_cast<OutT*>(g.C) + bz * g.strideC;
    for (int i = threadIdx.x; i < MT * 64; i += blockDim.x) {
        const int x = i >> 6, l = i & 63;
        f32x4 s = part[0][x][l];
        for (int w = 1; w < nw; ++w) s += part[w][x][l];
        const int m = 16 * x + (l & 15), n = n0 + 4 * (l >> 4);
        if (m >= g.M) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (n + v < g.N) put(C + m * g.ldc + n + v, s[v]);
    }
}

// the kernel over the tiles of every product, in as many launches as their number takes (one but for long
// batches of large products)
template <typename OutT>
hipError_t tile_gemm(void (*kernel)(Mx4Args), Mx4Args g, int tile, int batch, hipStream_t stream) {
    g.num_m = (g.M + tile - 1) / tile;
    g.num_n = (g.N + tile - 1) / tile;
    const int64_t tiles = static_cast<int64_t>(g.num_m) * g.num_n;
    const int step = matrices_a_launch(tiles, batch);
    if (step == 0) return hipErrorInvalidValue;
    for (int b = 0; b < batch; b += step) {
        Mx4Args part = g;
        part.A = g.A.from(b);
        part.B = g.B.from(b);
        part.C = static_cast<OutT*>(g.C) + b * g.strideC;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(tiles * std::min(step, batch - b))), dim3(256), 0, stream, part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int64_t kMaxPitch = int64_t{1} << 22;   // of the wide kernel's 32-bit offsets within a tile

template <typename OutT>
hipError_t gemm(const Mx4Args& g, int batch, hipStream_t stream) {
    if (mx4_few_rows(g.M, g.N, 32 * static_cast<int64_t>(g.nblk))) {
        const int groups = (g.N + 15) / 16;
        const int waves = groups >= 512 ? 4 : groups >= 128 ? 8 : 16;
        const dim3 grid(groups, batch), block(64 * waves);
        if (g.M <= 16) hipLaunchKernelGGL((mx4_few_rows_kernel<1, OutT>), grid, block, 0, stream, g);
        else hipLaunchKernelGGL((mx4_few_rows_kernel<2, OutT>), grid, block, 0, stream, g);
        return hipGetLastError();
    }
    const Mx4Tile tile = mx4_tile(g.M, g.N, batch);
    if (tile == kMx4Tile64) return tile_gemm<OutT>(mx4_tile_gemm_kernel<1, 1, 2, 2, 4, OutT>, g, 64, batch, stream);
    if (tile == kMx4Tile128 || std::max(std::max(g.A.ldq, g.B.ldq), std::max(g.A.lds, g.B.lds)) >= kMaxPitch)
        return tile_gemm<OutT>(mx4_tile_gemm_kernel<2, 2, 2, 2, 2, OutT>, g, 128, batch, stream);
    return tile_gemm<OutT>(mx4_wide_gemm_kernel<OutT>, g, 256, batch, stream);
}

}  // namespace

hipError_t launch_mx4_gemm(const MxMatrix& A, const MxMatrix& B, void* C, bool bf16, int64_t ldc, int64_t strideC, int64_t M,
                           int64_t N, int64_t K, int batch, hipStream_t stream) {
    const Mx4Args g{A, B, C, ldc, strideC, static_cast<int>(M), static_cast<int>(N), static_cast<int>(mx_blocks(K)), 0, 0};
    return bf16 ? gemm<bf16_t>(g, batch, stream) : gemm<float>(g, batch, stream);
}

}  // namespace galore
