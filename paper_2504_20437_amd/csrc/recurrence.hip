// A gated linear recurrence over tokens, in each channel by itself:
//   a = sigmoid(f),  h_t = a_t h_{t-1} + (1 - a_t) x_t
// and backward
//   g_t = dh_t + a_{t+1} g_{t+1};  dx = (1 - a) g;  df = g (h_{t-1} - x) a (1 - a)
// 1 - a is sigmoid(-f), not a difference: it keeps its digits where a gate hardly forgets.
//
// Steps h -> A h + B compose, (A, B) after (A', B') is (A A', A B' + B), so the tokens are
// cut into chunks and a chunk into the runs of its threads: each run's composition, then
// the compositions before it, then its states. Backward the carry is u_t = a_t g_t, with
// u_t = a_t (dh_t + u_{t+1}) from the last token on; the states before each token are
// made again from x, f and the state kept every 64 tokens, so that h itself need not be
// kept. Packed sequences: at a sequence's first token the state before it is its h0,
// at its last one the carry from behind is its gradient of the last state.
// All in fp32.
#include <algorithm>

#include "mx.hpp"
#include "layers.hpp"

namespace galore {
namespace {

constexpr int kC = 4;                        // channels of a thread
constexpr int kTx = 16;                      // threads along the channels: a row's piece of a workgroup is a line
constexpr int kTy = 16;                      // threads along the tokens
constexpr int kThreads = kTx * kTy, kWaves = kThreads / 64;
constexpr int kForward = 8, kBackward = 4;   // tokens of a thread's run

// sigmoid(f) and sigmoid(-f): exp(-|f|) as a power of two whose exponent's rounding is made up for
__device__ __forceinline__ void gates(float f, float& a, float& z) {
    const float m = __builtin_fabsf(f);
    const float hi = m * 1.44269502f;                                     // log2 e in two parts
    const float lo = __builtin_fmaf(m, 1.44269502f, -hi) + m * 1.92596299e-8f;
    const float p = __builtin_amdgcn_exp2f(-hi);
    const float e = p - p * (lo * 0.693147181f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e), s = e * r;
    a = f >= 0.0f ? r : s;
    z = f >= 0.0f ? s : r;
}

// four values of a row as they are stored, `n` of them inside it
template <typename T>
struct Four;
template <>
struct Four<bf16_t> {
    u32x2 w;
    __device__ __forceinline__ void load(const bf16_t* p, int n) {
        if (n >= kC) {
            w = get_vector<u32x2>(p, false);
        } else {
            w[0] = (n > 0 ? p[0].bits : 0u) | (n > 1 ? static_cast<uint32_t>(p[1].bits) << 16 : 0u);
            w[1] = n > 2 ? p[2].bits : 0u;
        }
    }
    __device__ __forceinline__ void clear() { w = u32x2{0u, 0u}; }
    __device__ __forceinline__ float operator[](int i) const {
        return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
};
template <>
struct Four<float> {
    f32x4 v;
    __device__ __forceinline__ void load(const float* p, int n) {
        if (n >= kC) {
            v = get_vector<f32x4>(p, false);
        } else {
#pragma unroll
            for (int i = 0; i < kC; ++i) v[i] = i < n ? p[i] : 0.0f;
        }
    }
    __device__ __forceinline__ void clear() { v = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
__device__ __forceinline__ void store4(float* p, int n, const float (&x)[kC]) {
    if (n >= kC) {
        put_vector(p, f32x4{x[0], x[1], x[2], x[3]}, false);
    } else {
#pragma unroll
        for (int i = 0; i < kC; ++i)
            if (i < n) p[i] = x[i];
    }
}
__device__ __forceinline__ void store4(bf16_t* p, int n, const float (&x)[kC]) {
    const u32x2 w = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    if (n >= kC) {
        put_vector(p, w, false);
    } else {
#pragma unroll
        for (int i = 0; i < kC; ++i)
            if (i < n) p[i].bits = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
    }
}
// four values of a float32 matrix (zeros where it is null)
__device__ __forceinline__ void load4(const float* p, int64_t at, int n, float (&x)[kC]) {
    Four<float> v;
    v.clear();
    if (p != nullptr && n > 0) v.load(p + at, n);
#pragma unroll
    for (int i = 0; i < kC; ++i) x[i] = v[i];
}

// A composition of steps for a thread's channels, h -> a h + b; a = -1 (no product of
// gates) where a sequence begins in it: b then is all that comes out, also where what
// came in was no number.
struct Map {
    float a[kC], b[kC];
    __device__ __forceinline__ void identity() {
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            a[i] = 1.0f;
            b[i] = 0.0f;
        }
    }
    // this after `first`
    template <bool PACKED>
    __device__ __forceinline__ void after(const Map& first) {
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            const bool cut = PACKED && a[i] < 0.0f;
            b[i] = cut ? b[i] : __builtin_fmaf(a[i], first.b[i], b[i]);
            a[i] = cut || (PACKED && first.a[i] < 0.0f) ? -1.0f : a[i] * first.a[i];
        }
    }
    __device__ __forceinline__ void into(float (&h)[kC]) const {
#pragma unroll
        for (int i = 0; i < kC; ++i) h[i] = a[i] < 0.0f ? b[i] : __builtin_fmaf(a[i], h[i], b[i]);
    }
};

// `own` of every thread composed over the threads that come before it: `before`, and
// `total` over all of them. Upwards the runs come in the order of the tokens, else the other way round.
template <bool UP, bool PACKED>
__device__ __forceinline__ void compose(const Map& own, Map& before, Map& total, Map (&waves)[kWaves][kTx]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tx = lane % kTx;
    constexpr int kRuns = 64 / kTx;
    const int place = UP ? lane / kTx : kRuns - 1 - lane / kTx;
    Map inc = own;
#pragma unroll
    for (int k = 1; k < kRuns; k *= 2) {
        Map o;
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            o.a[i] = UP ? __shfl_up(inc.a[i], k * kTx) : __shfl_down(inc.a[i], k * kTx);
            o.b[i] = UP ? __shfl_up(inc.b[i], k * kTx) : __shfl_down(inc.b[i], k * kTx);
        }
        if (place >= k) inc.after<PACKED>(o);
    }
#pragma unroll
    for (int i = 0; i < kC; ++i) {
        before.a[i] = UP ? __shfl_up(inc.a[i], kTx) : __shfl_down(inc.a[i], kTx);
        before.b[i] = UP ? __shfl_up(inc.b[i], kTx) : __shfl_down(inc.b[i], kTx);
    }
    if (place == 0) before.identity();
    __syncthreads();
    if (place == kRuns - 1) waves[wave][tx] = inc;
    __syncthreads();
    Map first;
    first.identity();
    total.identity();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const int w = UP ? k : kWaves - 1 - k;
        Map m = waves[w][tx];
        if (UP ? w < wave : w > wave) {
            Map n = m;
            n.after<PACKED>(first);
            first = n;
        }
        m.after<PACKED>(total);
        total = m;
    }
    before.after<PACKED>(first);
}

// What the tokens of a chunk are in packed sequences: -1 for a token of none, else
// 4 sequence + (1: its first token) + (2: its last one)
template <int L>
__device__ __forceinline__ void find_owners(const ScanArgs& a, int64_t t0, int (&owner)[L]) {
    const auto bound = [&](int64_t s) {
        const int64_t o = a.offsets.at(s);
        return o < 0 ? 0 : o > a.T ? a.T : o;
    };
    for (int i = threadIdx.x; i < L; i += kThreads) {
        const int64_t t = t0 + i;
        int code = -1;
        if (t < a.T) {
            int64_t lo = 0, hi = a.sequences;        // the sequences that begin at t or before
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (bound(mid) <= t) lo = mid + 1;
                else hi = mid;
            }
            if (lo > 0) {
                const int64_t end = bound(lo);
                if (t < end) code = static_cast<int>(4 * (lo - 1)) + (bound(lo - 1) == t ? 1 : 0) + (end == t + 1 ? 2 : 0);
            }
        }
        owner[i] = code;
    }
    __syncthreads();
}
// to[s] = from[s] for the sequences without tokens; the workgroups share them
__device__ __forceinline__ void copy_empty(const ScanArgs& a, const float* from, float* to, int64_t ch, int n) {
    for (int64_t s = static_cast<int64_t>(blockIdx.x) * kTy + threadIdx.x / kTx; s < a.sequences;
         s += static_cast<int64_t>(gridDim.x) * kTy) {
        const auto bound = [&](int64_t i) {
            const int64_t o = a.offsets.at(i);
            return o < 0 ? 0 : o > a.T ? a.T : o;
        };
        if (bound(s + 1) > bound(s) || n <= 0) continue;
        float v[kC];
        load4(from, s * a.d + ch, n, v);
        store4(to + s * a.d + ch, n, v);
    }
}

// kWhole: the matrix is one chunk; else kSummary leaves each chunk's composition in
// `summary`, and kStates takes the state that enters it from `enter`
enum Phase { kWhole, kSummary, kStates };

template <typename T, bool PACKED, int PHASE>
__global__ __launch_bounds__(kThreads) void scan_kernel(ScanArgs a, float2* summary, const float* enter) {
    constexpr int S = kForward, L = S * kTy;
    __shared__ Map waves[kWaves][kTx];
    __shared__ int owner[PACKED ? L : 1];
    const int tx = threadIdx.x % kTx, ty = threadIdx.x / kTx;
    const int64_t b = blockIdx.z, chunk = blockIdx.x;
    const int64_t ch = kC * (static_cast<int64_t>(blockIdx.y) * kTx + tx);
    const int n = static_cast<int>(min(a.d - ch, static_cast<int64_t>(kC)));
    const int64_t t0 = chunk * L + ty * S;
    Four<T> x[S], f[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        x[s].clear();
        f[s].clear();
        if (t0 + s < a.T && n > 0) {
            x[s].load(static_cast<const T*>(a.X) + b * a.strideX + (t0 + s) * a.ldx + ch, n);
            f[s].load(static_cast<const T*>(a.F) + b * a.strideF + (t0 + s) * a.ldf + ch, n);
        }
    }
    if (PACKED) find_owners(a, chunk * L, owner);
    float g[S][kC], u[S][kC];
    Map own;
    own.identity();
    bool cut = false;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        bool reset = false;
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            float z;
            gates(f[s][i], g[s][i], z);
            u[s][i] = z * x[s][i];
        }
        if (PACKED) {
            const int code = owner[ty * S + s];
            reset = code < 0 || (code & 1);
            cut = cut || reset;
            if (code < 0) {
#pragma unroll
                for (int i = 0; i < kC; ++i) u[s][i] = 0.0f;
            } else if (code & 1) {
                float h0[kC];
                load4(a.h0, (code >> 2) * a.d + ch, n, h0);
#pragma unroll
                for (int i = 0; i < kC; ++i) u[s][i] = __builtin_fmaf(g[s][i], h0[i], u[s][i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            own.a[i] *= g[s][i];
            own.b[i] = reset ? u[s][i] : __builtin_fmaf(g[s][i], own.b[i], u[s][i]);
        }
    }
    if (PACKED && cut) {
#pragma unroll
        for (int i = 0; i < kC; ++i) own.a[i] = -1.0f;
    }
    const int64_t place = (b * gridDim.x + chunk) * a.d + ch;
    float h[kC];       // read before the barriers: `last` may be h0
    if (PHASE == kStates) load4(enter, place, n, h);
    if (PHASE == kWhole) load4(PACKED ? nullptr : a.h0, b * a.d + ch, n, h);
    Map before, total;
    compose<true, PACKED>(own, before, total, waves);
    if (PHASE == kSummary) {
        if (ty == kTy - 1) {
#pragma unroll
            for (int i = 0; i < kC; ++i)
                if (i < n) summary[place + i] = make_float2(total.a[i], total.b[i]);
        }
        return;
    }
    before.into(h);
    if (!PACKED && a.T == 0 && ty == 0) store4(a.last + b * a.d + ch, n, h);
    if (a.states != nullptr && t0 % kScanStep == 0 && t0 < a.T)
        store4(a.states + (b * ((a.T + kScanStep - 1) / kScanStep) + t0 / kScanStep) * a.d + ch, n, h);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int code = PACKED ? owner[ty * S + s] : 0;
        const bool reset = PACKED && (code < 0 || (code & 1));
#pragma unroll
        for (int i = 0; i < kC; ++i) h[i] = reset ? u[s][i] : __builtin_fmaf(g[s][i], h[i], u[s][i]);
        if (t0 + s < a.T && code >= 0) {
            store4(static_cast<T*>(a.H) + b * a.strideH + (t0 + s) * a.ldh + ch, n, h);
            if (PACKED ? (code & 2) != 0 : t0 + s == a.T - 1) store4(a.last + (PACKED ? code >> 2 : b) * a.d + ch, n, h);
        }
    }
    if (PACKED) copy_empty(a, a.h0, a.last, ch, n);
}

template <typename T, bool PACKED, int PHASE>
__global__ __launch_bounds__(kThreads) void scan_backward_kernel(ScanArgs a, float2* summary, const float* enter) {
    constexpr int S = kBackward, L = S * kTy;
    __shared__ Map waves[kWaves][kTx];
    __shared__ int owner[PACKED ? L : 1];
    const int tx = threadIdx.x % kTx, ty = threadIdx.x / kTx;
    const int64_t b = blockIdx.z, chunk = blockIdx.x;
    const int64_t ch = kC * (static_cast<int64_t>(blockIdx.y) * kTx + tx);
    const int n = static_cast<int>(min(a.d - ch, static_cast<int64_t>(kC)));
    const int64_t t0 = chunk * L + ty * S;
    Four<T> x[S], f[S], dh[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        x[s].clear();
        f[s].clear();
        dh[s].clear();
        if (t0 + s < a.T && n > 0) {
            if (PHASE != kSummary) x[s].load(static_cast<const T*>(a.X) + b * a.strideX + (t0 + s) * a.ldx + ch, n);
            f[s].load(static_cast<const T*>(a.F) + b * a.strideF + (t0 + s) * a.ldf + ch, n);
            dh[s].load(static_cast<const T*>(a.dH) + b * a.strideDH + (t0 + s) * a.lddh + ch, n);
        }
    }
    if (PACKED) find_owners(a, chunk * L, owner);
    // the carry from behind at a sequence's last token; a token of none carries nothing
    const auto code_of = [&](int s) { return PACKED ? owner[ty * S + s] : t0 + s < a.T ? 0 : -1; };
    float g[S][kC], z[S][kC];
    Map own;
    own.identity();
    bool cut = false;
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        const int code = code_of(s);
        float end[kC] = {};
        const bool reset = PACKED && (code < 0 || (code & 2));
        if (PACKED && code >= 0 && (code & 2)) load4(a.dlast, (code >> 2) * a.d + ch, n, end);
        cut = cut || reset;
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            gates(f[s][i], g[s][i], z[s][i]);
            if (reset) {
                own.b[i] = code < 0 ? 0.0f : g[s][i] * (dh[s][i] + end[i]);
            } else if (code >= 0) {
                own.a[i] *= g[s][i];
                own.b[i] = g[s][i] * (dh[s][i] + own.b[i]);
            }
        }
    }
    if (PACKED && cut) {
#pragma unroll
        for (int i = 0; i < kC; ++i) own.a[i] = -1.0f;
    }
    Map before, total;
    compose<false, PACKED>(own, before, total, waves);
    const int64_t place = (b * gridDim.x + chunk) * a.d + ch;
    if (PHASE == kSummary) {
        if (ty == 0) {
#pragma unroll
            for (int i = 0; i < kC; ++i)
                if (i < n) summary[place + i] = make_float2(total.a[i], total.b[i]);
        }
        return;
    }
    float c[kC];       // the carry from behind
    if (PHASE == kStates) load4(enter, place, n, c);
    else load4(PACKED ? nullptr : a.dlast, b * a.d + ch, n, c);
    before.into(c);
    // the states before each token
    own.identity();
    cut = false;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int code = code_of(s);
        float h0[kC] = {};
        const bool first = PACKED && code >= 0 && (code & 1);
        if (first) load4(a.h0, (code >> 2) * a.d + ch, n, h0);
        cut = cut || (PACKED && (code < 0 || first));
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            if (PACKED && (code < 0 || first)) own.b[i] = h0[i];
            own.a[i] *= g[s][i];
            own.b[i] = __builtin_fmaf(g[s][i], own.b[i], z[s][i] * x[s][i]);
        }
    }
    if (PACKED && cut) {
#pragma unroll
        for (int i = 0; i < kC; ++i) own.a[i] = -1.0f;
    }
    compose<true, PACKED>(own, before, total, waves);
    float h[kC], prev[S][kC];
    if (a.T > 0) load4(a.states, (b * ((a.T + kScanStep - 1) / kScanStep) + chunk * L / kScanStep) * a.d + ch, n, h);
    else load4(nullptr, 0, 0, h);
    before.into(h);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int code = code_of(s);
        if (PACKED && code >= 0 && (code & 1)) load4(a.h0, (code >> 2) * a.d + ch, n, h);
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            prev[s][i] = h[i];
            h[i] = __builtin_fmaf(g[s][i], h[i], z[s][i] * x[s][i]);
        }
    }
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        const int code = code_of(s);
        if (PACKED && code >= 0 && (code & 2)) load4(a.dlast, (code >> 2) * a.d + ch, n, c);
        if (code < 0) continue;
        float dx[kC], df[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            const float dg = dh[s][i] + c[i];
            dx[i] = z[s][i] * dg;
            df[i] = dg * (prev[s][i] - x[s][i]) * (g[s][i] * z[s][i]);
            c[i] = g[s][i] * dg;
        }
        store4(static_cast<T*>(a.dX) + b * a.strideDX + (t0 + s) * a.lddx + ch, n, dx);
        store4(static_cast<T*>(a.dF) + b * a.strideDF + (t0 + s) * a.lddf + ch, n, df);
        if (PACKED ? (code & 1) != 0 : t0 + s == 0) store4(a.dh0 + (PACKED ? code >> 2 : b) * a.d + ch, n, c);
    }
    if (PACKED) copy_empty(a, a.dlast, a.dh0, ch, n);
    else if (a.T == 0 && ty == 0) store4(a.dh0 + b * a.d + ch, n, c);
}

// the state that enters each chunk, in the order of the tokens or (!UP) against it
template <bool UP>
__global__ __launch_bounds__(64) void carry_kernel(const float2* summary, float* enter, const float* start, int64_t chunks,
                                                   int64_t d) {
    const int64_t ch = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x, b = blockIdx.y;
    if (ch >= d) return;
    float h = start != nullptr ? start[b * d + ch] : 0.0f;
#pragma unroll 8
    for (int64_t k = 0; k < chunks; ++k) {
        const int64_t at = (b * chunks + (UP ? k : chunks - 1 - k)) * d + ch;
        enter[at] = h;
        const float2 m = summary[at];
        h = m.x < 0.0f ? m.y : __builtin_fmaf(m.x, h, m.y);
    }
}

template <int S>
int64_t chunk_count(int64_t T) {
    return std::max<int64_t>((T + S * kTy - 1) / (S * kTy), 1);
}

template <typename T, bool PACKED>
hipError_t scan(const ScanArgs& a, int batch, hipStream_t stream) {
    const int64_t chunks = chunk_count<kForward>(a.T);
    const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>((a.d + kC * kTx - 1) / (kC * kTx)),
                    static_cast<unsigned>(batch));
    if (chunks == 1) {
        hipLaunchKernelGGL((scan_kernel<T, PACKED, kWhole>), grid, dim3(kThreads), 0, stream, a, nullptr, nullptr);
        return hipGetLastError();
    }
    float2* summary = static_cast<float2*>(a.workspace);
    float* enter = reinterpret_cast<float*>(summary + chunks * batch * a.d);
    hipLaunchKernelGGL((scan_kernel<T, PACKED, kSummary>), grid, dim3(kThreads), 0, stream, a, summary, enter);
    hipLaunchKernelGGL(carry_kernel<true>, dim3(static_cast<unsigned>((a.d + 63) / 64), static_cast<unsigned>(batch)), dim3(64),
                       0, stream, summary, enter, PACKED ? nullptr : a.h0, chunks, a.d);
    hipLaunchKernelGGL((scan_kernel<T, PACKED, kStates>), grid, dim3(kThreads), 0, stream, a, summary, enter);
    return hipGetLastError();
}

template <typename T, bool PACKED>
hipError_t scan_backward(const ScanArgs& a, int batch, hipStream_t stream) {
    const int64_t chunks = chunk_count<kBackward>(a.T);
    const dim3 grid(static_cast<unsigned>(chunks), static_cast<unsigned>((a.d + kC * kTx - 1) / (kC * kTx)),
                    static_cast<unsigned>(batch));
    if (chunks == 1) {
        hipLaunchKernelGGL((scan_backward_kernel<T, PACKED, kWhole>), grid, dim3(kThreads), 0, stream, a, nullptr, nullptr);
        return hipGetLastError();
    }
    float2* summary = static_cast<float2*>(a.workspace);
    float* enter = reinterpret_cast<float*>(summary + chunks * batch * a.d);
    hipLaunchKernelGGL((scan_backward_kernel<T, PACKED, kSummary>), grid, dim3(kThreads), 0, stream, a, summary, enter);
    hipLaunchKernelGGL(carry_kernel<false>, dim3(static_cast<unsigned>((a.d + 63) / 64), static_cast<unsigned>(batch)), dim3(64),
                       0, stream, summary, enter, PACKED ? nullptr : a.dlast, chunks, a.d);
    hipLaunchKernelGGL((scan_backward_kernel<T, PACKED, kStates>), grid, dim3(kThreads), 0, stream, a, summary, enter);
    return hipGetLastError();
}

}  // namespace

size_t scan_bytes(int64_t T, int64_t d, int64_t batch) {
    const int64_t chunks = chunk_count<kBackward>(T);
    return chunks == 1 ? 0 : static_cast<size_t>(chunks * d * batch) * (sizeof(float2) + sizeof(float));
}

hipError_t launch_scan(const ScanArgs& a, bool bf16, int batch, hipStream_t stream) {
    const bool packed = a.offsets.p != nullptr;
    if (bf16) return packed ? scan<bf16_t, true>(a, batch, stream) : scan<bf16_t, false>(a, batch, stream);
    return packed ? scan<float, true>(a, batch, stream) : scan<float, false>(a, batch, stream);
}
hipError_t launch_scan_backward(const ScanArgs& a, bool bf16, int batch, hipStream_t stream) {
    const bool packed = a.offsets.p != nullptr;
    if (bf16) return packed ? scan_backward<bf16_t, true>(a, batch, stream) : scan_backward<bf16_t, false>(a, batch, stream);
    return packed ? scan_backward<float, true>(a, batch, stream) : scan_backward<float, false>(a, batch, stream);
}

}  // namespace galore
