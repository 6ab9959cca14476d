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
//
// Bound by memory, next by the two transcendental and about 25 other instructions a
// value (half of the time of the bytes) and the waits of the chain. bf16, forward with
// states: 24 x 8192 x 2048 521 us (4.7 TB/s, a workgroup to each tile of channels, no
// chain), 4 x 8192 x 2048 97 (4.2), 1 x 8192 x 4096 54 (3.8), packed into eleven sequences
// 60. Backward 948 (4.3), 163 (4.1), 89 (3.8) and packed 120. fp32 1 x 8192 x 4096: 85 (4.8)
// and 146 (4.6). Where the tiles are not a multiple of the workgroups that run at a time,
// the last of them leave places empty: 24 x 8192 x 2048 backward is one such (runs of 4,
// three workgroups to a CU, took 840), 5 x 8192 x 4096 backward 536 (3.2), 8 x 8192 x 3200
// forward 326 (3.9). In three launches (compositions, carries, states), with x and f
// read twice: 177 for 4 x 8192 x 2048.
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "layers.hpp"

namespace galore {
namespace {

constexpr int kC = 4;                        // channels of a thread
constexpr int kTx = 16;                      // threads along the channels: a row's piece of a workgroup is a line of bf16
constexpr int kTy = 16;                      // threads along the tokens
constexpr int kTile = kC * kTx;              // channels of a workgroup
constexpr int kThreads = kTx * kTy, kWaves = kThreads / 64;
constexpr int kForward = 8;                  // tokens of a thread's run
// backward: in fp32 what a run holds would not fit the registers at 8
template <typename T>
constexpr int kBackward = sizeof(T) == 2 ? 8 : 4;
constexpr int kChunk = kTy * 8;              // tokens of a chunk at most

// sigmoid(f) and sigmoid(-f) from e = exp(-f), a power of two whose exponent's rounding is
// made up for: a bf16's product with the upper 15 bits of log2 e is exact. e is taken at
// -87 at least, where it does not overflow and its reciprocal is still a normal number;
// under -87 the gate, less than 1.7e-38, is zero, so that nothing is left of what it
// forgets. Past 100 (e is no normal number) it stays one.
template <typename T>
__device__ __forceinline__ void gates(float f, float& a, float& z) {
    constexpr float kUpper = 0x1.7154p+0f, kLower = 0x1.d94ae0p-18f;          // log2 e in 15 bits and the rest
    constexpr float kFull = 0x1.715476p+0f, kRest = 0x1.4ae0c0p-26f;          // and in 24 bits
    constexpr float kLn2 = 0x1.62e430p-1f;
    const float m = __builtin_elementwise_minimum(__builtin_elementwise_maximum(f, -87.0f), 100.0f);   // a NaN stays one
    float p, low;
    if constexpr (sizeof(T) == 2) {
        p = __builtin_amdgcn_exp2f(m * -kUpper);
        low = m * (-kLower * kLn2);
    } else {
        const float hi = m * -kFull;
        p = __builtin_amdgcn_exp2f(hi);
        low = (__builtin_fmaf(m, -kFull, -hi) - m * kRest) * kLn2;
    }
    const float e = __builtin_fmaf(p, low, p), gate = __builtin_amdgcn_rcpf(1.0f + e);
    a = f < -87.0f ? 0.0f : gate;
    z = e * gate;
}

// Four values of a row as they are stored, `n` of them inside it. FULL: four or none, and
// rows that are written start on four values, so that they go past the caches
template <typename T>
struct Four;
template <>
struct Four<bf16_t> {
    u32x2 w;
    template <bool FULL>
    __device__ __forceinline__ void load(const bf16_t* p, int n) {
        if (FULL || n >= kC) {
            w = get_vector<u32x2>(p, true);
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
    template <bool FULL>
    __device__ __forceinline__ void load(const float* p, int n) {
        if (FULL || n >= kC) {
            v = get_vector<f32x4>(p, true);
        } else {
#pragma unroll
            for (int i = 0; i < kC; ++i) v[i] = i < n ? p[i] : 0.0f;
        }
    }
    __device__ __forceinline__ void clear() { v = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};
template <bool FULL>
__device__ __forceinline__ void store4(float* p, int n, const float (&x)[kC]) {
    if (n >= kC) {
        put_vector(p, f32x4{x[0], x[1], x[2], x[3]}, FULL);
    } else if (!FULL) {
#pragma unroll
        for (int i = 0; i < kC; ++i)
            if (i < n) p[i] = x[i];
    }
}
template <bool FULL>
__device__ __forceinline__ void store4(bf16_t* p, int n, const float (&x)[kC]) {
    const u32x2 w = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    if (n >= kC) {
        put_vector(p, w, FULL);
    } else if (!FULL) {
#pragma unroll
        for (int i = 0; i < kC; ++i)
            if (i < n) p[i].bits = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
    }
}
// four values of a float32 matrix (zeros where it is null)
template <bool FULL>
__device__ __forceinline__ void load4(const float* p, int64_t at, int n, float (&x)[kC]) {
    Four<float> v;
    v.clear();
    if (p != nullptr && n > 0) v.load<FULL>(p + at, n);
#pragma unroll
    for (int i = 0; i < kC; ++i) x[i] = v[i];
}

// A composition of steps for N channels, h -> a h + b; a = -1 (no product of gates) where
// a sequence begins in it: b then is all that comes out, also where what came in was no
// number.
template <int N>
struct Map {
    float a[N], b[N];
    __device__ __forceinline__ void copy(const Map& o) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = o.a[i];
            b[i] = o.b[i];
        }
    }
    __device__ __forceinline__ void identity() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a[i] = 1.0f;
            b[i] = 0.0f;
        }
    }
    __device__ __forceinline__ void cut() {
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = -1.0f;
    }
    // this after `first`
    template <bool PACKED>
    __device__ __forceinline__ void after(const Map& first) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool cut = PACKED && a[i] < 0.0f;
            b[i] = cut ? b[i] : __builtin_fmaf(a[i], first.b[i], b[i]);
            a[i] = cut || (PACKED && first.a[i] < 0.0f) ? -1.0f : a[i] * first.a[i];
        }
    }
    template <bool PACKED>
    __device__ __forceinline__ void into(float (&h)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = PACKED && a[i] < 0.0f ? b[i] : __builtin_fmaf(a[i], h[i], b[i]);
    }
};
typedef Map<kC> Run;

// A wave's runs composed with those before them: `before` of a thread's own, the wave's
// total to LDS. Upwards the runs come in the order of the tokens, else the other way round.
template <bool UP, bool PACKED>
__device__ __forceinline__ void compose_wave(const Run& own, Run& before, Run& total_of_wave) {
    const int lane = threadIdx.x & 63;
    constexpr int kRuns = 64 / kTx;
    const int place = UP ? lane / kTx : kRuns - 1 - lane / kTx;
    Run inc;
    inc.copy(own);
#pragma unroll
    for (int k = 1; k < kRuns; k *= 2) {
        Run o;
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            o.a[i] = UP ? __shfl_up(inc.a[i], k * kTx) : __shfl_down(inc.a[i], k * kTx);
            o.b[i] = UP ? __shfl_up(inc.b[i], k * kTx) : __shfl_down(inc.b[i], k * kTx);
        }
        if (place >= k) inc.after<PACKED>(o);
    }
#pragma unroll
    for (int i = 0; i < kC; ++i) {
        const float pa = UP ? __shfl_up(inc.a[i], kTx) : __shfl_down(inc.a[i], kTx);
        const float pb = UP ? __shfl_up(inc.b[i], kTx) : __shfl_down(inc.b[i], kTx);
        before.a[i] = place == 0 ? 1.0f : pa;
        before.b[i] = place == 0 ? 0.0f : pb;
    }
    if (place == kRuns - 1) total_of_wave.copy(inc);
}
// `before` after the waves that come before this one
template <bool UP, bool PACKED>
__device__ __forceinline__ void compose_waves(Run& before, const Run (&waves)[kWaves][kTx]) {
    const int wave = threadIdx.x >> 6, tx = threadIdx.x % kTx;
    Run first;
    first.identity();
#pragma unroll
    for (int k = 0; k < kWaves - 1; ++k) {
        const int w = UP ? k : kWaves - 1 - k;
        if (UP ? w < wave : w > wave) {
            Run m;
            m.copy(waves[w][tx]);
            m.after<PACKED>(first);
            first.copy(m);
        }
    }
    before.after<PACKED>(first);
}

__device__ __forceinline__ int64_t bound(const ScanArgs& a, int64_t s) {
    const int64_t o = a.offsets.at(s);
    return o < 0 ? 0 : o > a.T ? a.T : o;
}

// What a token is in packed sequences: -1 for one of none, else 4 sequence + (1: its first
// token) + (2: its last one)
__device__ __forceinline__ int code_at(const ScanArgs& a, int64_t t) {
    if (t >= a.T) return -1;
    int64_t lo = 0, hi = a.sequences;        // the sequences that begin at t or before
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (bound(a, mid) <= t) lo = mid + 1;
        else hi = mid;
    }
    if (lo == 0) return -1;
    const int64_t end = bound(a, lo);
    if (t >= end) return -1;
    return static_cast<int>(4 * (lo - 1)) + (bound(a, lo - 1) == t ? 1 : 0) + (end == t + 1 ? 2 : 0);
}
// The codes of a chunk's L tokens, in threads first, first + 1 ... (first a multiple of 64):
// from memory, where the launch before left them, or looked up
template <int L>
__device__ __forceinline__ int get_code(const ScanArgs& a, const int* codes, int64_t t0, int first) {
    const int i = static_cast<int>(threadIdx.x) - first;
    if (i < 0 || i >= L) return 0;
    if (codes == nullptr) return code_at(a, t0 + i);
    return t0 + i < a.T ? codes[t0 + i] : -1;
}
// to LDS; marks: whether 64 tokens hold any but ones inside a sequence
template <int L>
__device__ __forceinline__ void put_code(int code, int* owner, int (&marks)[2], int first) {
    const int i = static_cast<int>(threadIdx.x) - first;
    if (i < 0 || i >= L) return;
    owner[i] = code;
    const bool any = __any(code < 0 || (code & 3));
    if ((i & 63) == 0) marks[i >> 6] = any ? 1 : 0;
    if (L <= 64 && i == 0) marks[1] = 0;
}
// to[s] = from[s] for the sequences without tokens; the chunks share them
template <bool FULL>
__device__ __forceinline__ void copy_empty(const ScanArgs& a, const float* from, float* to, int64_t chunk, int64_t chunks,
                                           int64_t ch, int n) {
    for (int64_t s = chunk * kTy + threadIdx.x / kTx; s < a.sequences; s += chunks * kTy) {
        if (bound(a, s + 1) > bound(a, s) || n <= 0) continue;
        float v[kC];
        load4<FULL>(from, s * a.d + ch, n, v);
        store4<FULL>(to + s * a.d + ch, n, v);
    }
}

// ---- chunks in a chain ----------------------------------------------------------------
//
// One launch over all chunks, so that x and f are read once. Where a workgroup takes all
// chunks of its channels itself (`link` null), what one leaves enters the next. Else it
// takes them from a counter, so that whoever waits for an earlier chunk knows that it is
// being worked on, by a workgroup that waits for still earlier ones only. It leaves its
// chunk's composition in `link` before it waits for anything. What enters a chunk is
// folded, in the order of the chunks, from the state after the last whole group of
// kGroup chunks (the first chunk, in the first group) and the compositions since:
// sixteen words at most, read together. Only the last chunk of a group (and the first of
// all) leaves its state and not its composition, so the chain of waits has a link for
// each group, and the order of the sums does not depend on who comes first. A word holds
// both halves of a composition and is written at once: it is its own flag (kEmpty until
// then), and nothing else is handed over.
constexpr int kGroup = 16;
constexpr uint64_t kEmpty = ~0ull;
constexpr int kTicketStep = 32;            // counters on lines of their own

struct Chain {
    uint64_t* link;        // batch x chunks x d
    uint32_t* ticket;      // (batch x tiles) x kTicketStep
    const int* codes;      // of the tokens of packed sequences, or null: looked up
    int64_t chunks;
    int tiles;
};

template <bool PACKED, bool BACK>
struct Shared {
    Run forward[kWaves][kTx], back[BACK ? kWaves : 1][kTx];     // the waves' totals
    float enter_a[kWaves][kTile], enter_b[kWaves][kTile];       // what enters the chunk, a part from each wave
    int next;
    int owner[2][PACKED ? kChunk : 1], marks[2][2];
};

// barrier over the workgroup's LDS; what is on its way from memory stays there
__device__ __forceinline__ void join_waves() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ void put_word(uint64_t* p, float a, float b) {
    // (a NaN's bits could be those of kEmpty)
    const uint32_t x = a != a ? 0x7fc00000u : __float_as_uint(a);
    __hip_atomic_store(p, static_cast<uint64_t>(__float_as_uint(b)) << 32 | x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The composition of words first .. first + kPart - 1 of the `words` before chunk k, whose
// word at this lane's channel is `link`; the first word of all is a state (a = 0)
constexpr int kPart = kGroup / kWaves;
template <bool PACKED>
__device__ __forceinline__ Map<1> wait_for(const uint64_t* link, int first, int words, int64_t d, bool in) {
    uint64_t w[kPart];
    bool missing;
    do {
        missing = false;
#pragma unroll
        for (int i = 0; i < kPart; ++i) {
            w[i] = 0;
            if (first + i < words && in) {
                w[i] = __hip_atomic_load(link - (words - first - i) * d, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                missing = missing || w[i] == kEmpty;
            }
        }
        if (__any(missing)) __builtin_amdgcn_s_sleep(1);
    } while (__any(missing));
    Map<1> all;
    all.identity();
#pragma unroll
    for (int i = 0; i < kPart; ++i) {
        if (first + i >= words) continue;
        Map<1> m;
        m.a[0] = __uint_as_float(static_cast<uint32_t>(w[i]));
        m.b[0] = __uint_as_float(static_cast<uint32_t>(w[i] >> 32));
        if (first + i > 0) m.after<PACKED>(all);
        all.copy(m);
    }
    return all;
}

// What a workgroup keeps from one chunk to the next: the last wave, at its lane's channel,
// the state that enters the first chunk, or any where it takes all chunks itself
template <bool PACKED, bool BACK>
struct Link {
    float state = 0.0f;
    Map<1> total;
    // the next chunk of these channels
    static __device__ __forceinline__ int64_t take(const Chain& chain, int pair, int64_t last) {
        if (chain.link == nullptr) return last + 1;
        return __hip_atomic_fetch_add(chain.ticket + static_cast<int64_t>(pair) * kTicketStep, 1u, __ATOMIC_RELAXED,
                                      __HIP_MEMORY_SCOPE_AGENT);
    }
    __device__ __forceinline__ void start(const ScanArgs& a, int64_t tile, int64_t b) {
        const int64_t ch = tile * kTile + (threadIdx.x & 63);
        const float* from = BACK ? a.dlast : a.h0;
        if (!PACKED && from != nullptr && ch < a.d) state = from[b * a.d + ch];
    }
    // after the barrier behind the waves' totals: leaves this chunk's composition, and
    // this wave's part of what enters it
    __device__ __forceinline__ void enter(const ScanArgs& a, const Chain& chain, int64_t k, int64_t tile, int64_t b,
                                          Shared<PACKED, BACK>& sh) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int64_t ch = tile * kTile + lane;
        const bool in = ch < a.d, solo = chain.link == nullptr, last = wave == kWaves - 1;
        uint64_t* link = chain.link + (b * chain.chunks + k) * a.d + ch;
        if (last) {
            total.identity();
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const int w = BACK ? kWaves - 1 - i : i;
                const Run& r = BACK ? sh.back[w][lane / kC] : sh.forward[w][lane / kC];
                Map<1> m;
                m.a[0] = r.a[lane % kC];
                m.b[0] = r.b[lane % kC];
                m.after<PACKED>(total);
                total.copy(m);
            }
            if (!solo && in && !leaves_state(k)) put_word(link, total.a[0], total.b[0]);
        }
        Map<1> part;
        part.identity();
        if (solo || k == 0) {
            if (last) {
                part.a[0] = 0.0f;
                part.b[0] = state;
            }
        } else {
            const int words = static_cast<int>(k - (k < kGroup ? 0 : k / kGroup * kGroup - 1));
            if (kPart * wave < words) part.copy(wait_for<PACKED>(link, kPart * wave, words, a.d, in));
        }
        sh.enter_a[wave][lane] = part.a[0];
        sh.enter_b[wave][lane] = part.b[0];
    }
    static __device__ __forceinline__ bool leaves_state(int64_t k) { return k == 0 || k % kGroup == kGroup - 1; }
    // N channels from `at` on, after the barrier behind the parts. (Solo, and at the first
    // chunk, the last wave's part is the state and the others are identities.)
    template <int N>
    static __device__ __forceinline__ void entered(const Shared<PACKED, BACK>& sh, int at, bool from_last, float (&h)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = from_last ? sh.enter_b[kWaves - 1][at + i] : sh.enter_b[0][at + i];
        if (from_last) return;
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float m = sh.enter_a[w][at + i], c = sh.enter_b[w][at + i];
                h[i] = PACKED && m < 0.0f ? c : __builtin_fmaf(m, h[i], c);
            }
    }
    // the state that leaves the chunk
    __device__ __forceinline__ void leave(const ScanArgs& a, const Chain& chain, int64_t k, int64_t tile, int64_t b,
                                          const Shared<PACKED, BACK>& sh) {
        const bool solo = chain.link == nullptr;
        if (static_cast<int>(threadIdx.x >> 6) != kWaves - 1 || !(solo || leaves_state(k))) return;
        const int lane = threadIdx.x & 63;
        const int64_t ch = tile * kTile + lane;
        float h[1];
        entered<1>(sh, lane, solo || k == 0, h);
        total.template into<PACKED>(h);
        if (solo) state = h[0];
        else if (ch < a.d) put_word(chain.link + (b * chain.chunks + k) * a.d + ch, 0.0f, h[0]);
    }
};

// a thread's rows as they are stored: `count` from p on
template <typename T, int S, bool FULL>
struct Rows {
    Four<T> v[S];
    __device__ __forceinline__ void load(const T* p, int64_t ld, int count, int n) {
        if (count >= S && n > 0) {
#pragma unroll
            for (int s = 0; s < S; ++s, p += ld) v[s].template load<FULL>(p, n);
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s, p += ld) {
                v[s].clear();
                if (s < count && n > 0) v[s].template load<FULL>(p, n);
            }
        }
    }
};

// where a thread stands
struct Place {
    int tx, ty, wave, n;       // n: of its channels, those below d (none where it is not positive)
    int64_t tile, b, ch;
    __device__ __forceinline__ Place(int64_t d, int64_t tile_, int64_t b_) {
        tx = threadIdx.x % kTx;
        ty = threadIdx.x / kTx;
        wave = threadIdx.x >> 6;
        tile = tile_;
        b = b_;
        ch = tile * kTile + kC * tx;
        n = static_cast<int>(min(d - ch, static_cast<int64_t>(kC)));
    }
};
// tokens from t0 on, S at most
template <int S>
__device__ __forceinline__ int tokens_from(int64_t T, int64_t t0) {
    return static_cast<int>(min(max(T - t0, static_cast<int64_t>(0)), static_cast<int64_t>(S)));
}

// What a thread's tokens are, a bit each: inside a sequence, its first, its last. The
// codes are looked at where the chunk has any but tokens inside sequences.
struct Marks {
    int inside, first, last;
    template <int S, bool PACKED>
    __device__ __forceinline__ void get(int count, const int* codes, bool any) {
        inside = (1 << count) - 1;
        first = last = 0;
        if (!PACKED || !any) return;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int code = codes[s];
            if (code < 0) inside &= ~(1 << s);
            else if (code & 3) {
                first |= (code & 1) << s;
                last |= (code >> 1 & 1) << s;
            }
        }
    }
};

// one chunk; the next one
template <typename T, bool PACKED, bool FULL>
__device__ __forceinline__ int64_t forward_chunk(const ScanArgs& a, const Chain& chain, const Place& at, int64_t k, int64_t next,
                                                 int buffer, Link<PACKED, false>& link, const Rows<T, kForward, FULL>& x,
                                                 const Rows<T, kForward, FULL>& f, Shared<PACKED, false>& sh) {
    constexpr int S = kForward, L = kTy * S;
    const int ty = at.ty, n = at.n;
    const int64_t t0 = k * L + ty * S, ch = at.ch;
    const int count = tokens_from<S>(a.T, t0);
    const int* codes = &sh.owner[buffer][PACKED ? ty * S : 0];
    Marks marks;
    marks.get<S, PACKED>(count, codes, (sh.marks[buffer][0] | sh.marks[buffer][1]) != 0);
    const int cuts = marks.first | ~marks.inside;
    const auto cut = [&](int s) { return PACKED && (cuts >> s & 1) != 0; };
    float g[S][kC], u[S][kC];
    Run own, before;
    own.identity();
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            float z;
            gates<T>(f.v[s][i], g[s][i], z);
            u[s][i] = z * x.v[s][i];
        }
        if (cut(s)) {
            float h0[kC];
            const bool first = (marks.first >> s & 1) != 0;
            load4<FULL>(first ? a.h0 : nullptr, (codes[s] >> 2) * a.d + ch, n, h0);
#pragma unroll
            for (int i = 0; i < kC; ++i) u[s][i] = first ? __builtin_fmaf(g[s][i], h0[i], u[s][i]) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            own.a[i] *= g[s][i];
            own.b[i] = cut(s) ? u[s][i] : __builtin_fmaf(g[s][i], own.b[i], u[s][i]);
        }
    }
    if (PACKED && (cuts & ((1 << S) - 1)) != 0) own.cut();
    compose_wave<true, PACKED>(own, before, sh.forward[at.wave][at.tx]);
    if (threadIdx.x == 0) sh.next = static_cast<int>(next);
    join_waves();
    next = sh.next;
    const int code_ahead = PACKED && next < chain.chunks ? get_code<L>(a, chain.codes, next * L, 64) : 0;
    link.enter(a, chain, k, at.tile, at.b, sh);
    if constexpr (PACKED) put_code<L>(code_ahead, sh.owner[buffer ^ 1], sh.marks[buffer ^ 1], 64);
    compose_waves<true, PACKED>(before, sh.forward);
    join_waves();
    link.leave(a, chain, k, at.tile, at.b, sh);
    float h[kC];
    link.template entered<kC>(sh, kC * at.tx, chain.link == nullptr || k == 0, h);
    before.template into<PACKED>(h);
    if (!PACKED && a.T == 0 && ty == 0) store4<FULL>(a.last + at.b * a.d + ch, n, h);
    if (a.states != nullptr && ty % (kScanStep / S) == 0 && count > 0)
        store4<FULL>(a.states + (at.b * ((a.T + kScanStep - 1) / kScanStep) + t0 / kScanStep) * a.d + ch, n, h);
    T* row = static_cast<T*>(a.H) + at.b * a.strideH + t0 * a.ldh + ch;
#pragma unroll
    for (int s = 0; s < S; ++s, row += a.ldh) {
#pragma unroll
        for (int i = 0; i < kC; ++i) h[i] = cut(s) ? u[s][i] : __builtin_fmaf(g[s][i], h[i], u[s][i]);
        if (marks.inside >> s & 1) store4<FULL>(row, n, h);
        if (PACKED && (marks.last >> s & 1)) store4<FULL>(a.last + (codes[s] >> 2) * a.d + ch, n, h);
        if (!PACKED && t0 + s == a.T - 1) store4<FULL>(a.last + at.b * a.d + ch, n, h);
    }
    if (PACKED) copy_empty<FULL>(a, a.h0, a.last, k, chain.chunks, ch, n);
    return __builtin_amdgcn_readfirstlane(static_cast<int>(next));
}

template <typename T, bool PACKED, bool FULL>
__device__ __forceinline__ int64_t backward_chunk(const ScanArgs& a, const Chain& chain, const Place& at, int64_t k,
                                                  int64_t next, int buffer, Link<PACKED, true>& link,
                                                  const Rows<T, kBackward<T>, FULL>& x, const Rows<T, kBackward<T>, FULL>& f,
                                                  const Rows<T, kBackward<T>, FULL>& dh, const float (&entering)[kC],
                                                  Shared<PACKED, true>& sh) {
    constexpr int S = kBackward<T>, L = kTy * S;
    const int ty = at.ty, n = at.n;
    const int64_t chunk = chain.chunks - 1 - k, t0 = chunk * L + ty * S, ch = at.ch;
    const int count = tokens_from<S>(a.T, t0);
    const int* codes = &sh.owner[buffer][PACKED ? ty * S : 0];
    Marks marks;
    marks.get<S, PACKED>(count, codes, (sh.marks[buffer][0] | sh.marks[buffer][1]) != 0);
    const int cuts = marks.first | ~marks.inside, ends = marks.last | ~marks.inside;
    const auto cut = [&](int s) { return PACKED && (cuts >> s & 1) != 0; };
    const auto end = [&](int s) { return PACKED && (ends >> s & 1) != 0; };
    const auto row_of = [&](const float* p, int which, int s, float (&v)[kC]) {       // of the token's sequence
        load4<FULL>(which >> s & 1 ? p : nullptr, (codes[s] >> 2) * a.d + ch, n, v);
    };
    float g[S][kC], z[S][kC], h[kC];
    Run own, back, before, behind;
    // upwards, the states; a sequence's first token has its h0 before it
    own.identity();
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (cut(s)) row_of(a.h0, marks.first, s, own.b);
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            gates<T>(f.v[s][i], g[s][i], z[s][i]);
            own.a[i] *= g[s][i];
            own.b[i] = __builtin_fmaf(g[s][i], own.b[i], z[s][i] * x.v[s][i]);
        }
    }
    if (PACKED && (cuts & ((1 << S) - 1)) != 0) own.cut();
    compose_wave<true, PACKED>(own, before, sh.forward[at.wave][at.tx]);
    // downwards, the carries; at a sequence's last token comes the gradient of its last state
    back.identity();
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        if (end(s)) row_of(a.dlast, marks.last, s, back.b);
        if (marks.inside >> s & 1) {
#pragma unroll
            for (int i = 0; i < kC; ++i) {
                back.a[i] *= g[s][i];
                back.b[i] = g[s][i] * (dh.v[s][i] + back.b[i]);
            }
        }
    }
    if (PACKED && (ends & ((1 << S) - 1)) != 0) back.cut();
    compose_wave<false, PACKED>(back, behind, sh.back[at.wave][at.tx]);
    if (threadIdx.x == 0) sh.next = static_cast<int>(next);
    join_waves();
    next = sh.next;
    const int code_ahead =
        PACKED && next < chain.chunks ? get_code<L>(a, chain.codes, (chain.chunks - 1 - next) * L, 64) : 0;
    link.enter(a, chain, k, at.tile, at.b, sh);
    if constexpr (PACKED) put_code<L>(code_ahead, sh.owner[buffer ^ 1], sh.marks[buffer ^ 1], 64);
    compose_waves<true, PACKED>(before, sh.forward);
    compose_waves<false, PACKED>(behind, sh.back);
#pragma unroll
    for (int i = 0; i < kC; ++i) h[i] = entering[i];
    before.template into<PACKED>(h);
    // what f's gradient is of the carry: (the state before - x) a (1 - a)
    float w[S][kC];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (cut(s)) row_of(a.h0, marks.first, s, h);
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            const float v = x.v[s][i];
            w[s][i] = (h[i] - v) * (g[s][i] * z[s][i]);
            h[i] = __builtin_fmaf(g[s][i], h[i], z[s][i] * v);
        }
    }
    join_waves();
    link.leave(a, chain, k, at.tile, at.b, sh);
    float c[kC];
    link.template entered<kC>(sh, kC * at.tx, chain.link == nullptr || k == 0, c);
    behind.template into<PACKED>(c);
    if (!PACKED && a.T == 0 && ty == 0) store4<FULL>(a.dh0 + at.b * a.d + ch, n, c);
    T* to_x = static_cast<T*>(a.dX) + at.b * a.strideDX + (t0 + S - 1) * a.lddx + ch;
    T* to_f = static_cast<T*>(a.dF) + at.b * a.strideDF + (t0 + S - 1) * a.lddf + ch;
#pragma unroll
    for (int s = S - 1; s >= 0; --s, to_x -= a.lddx, to_f -= a.lddf) {
        if (end(s)) row_of(a.dlast, marks.last, s, c);
        if (!(marks.inside >> s & 1)) continue;
        float dx[kC], df[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            const float dg = dh.v[s][i] + c[i];
            dx[i] = z[s][i] * dg;
            df[i] = dg * w[s][i];
            c[i] = g[s][i] * dg;
        }
        store4<FULL>(to_x, n, dx);
        store4<FULL>(to_f, n, df);
        if (PACKED && (marks.first >> s & 1)) store4<FULL>(a.dh0 + (codes[s] >> 2) * a.d + ch, n, c);
        if (!PACKED && t0 + s == 0) store4<FULL>(a.dh0 + at.b * a.d + ch, n, c);
    }
    if (PACKED) copy_empty<FULL>(a, a.dlast, a.dh0, chunk, chain.chunks, ch, n);
    return __builtin_amdgcn_readfirstlane(static_cast<int>(next));
}

// Workgroups to a CU: what the registers of a thread's run leave. Backward in bf16 holds
// runs of 8 tokens in 256 registers: 8192 x 4096 89 us (before a gate under -87 was zero
// 86; then runs of 4 and three workgroups took 97, of 8 and three 201 for their spills).
// Forward in registers for four: bf16 8 x 8192 x 3200 339 us, for three 315 (calls in a row).
template <typename T, bool BACK>
constexpr int kResident = BACK && sizeof(T) == 2 ? 2 : 3;

template <typename T, bool PACKED, bool BACK, bool FULL>
__global__ __launch_bounds__(kThreads, (kResident<T, BACK>)) void scan_kernel(ScanArgs a, Chain chain, int pairs) {
    constexpr int S = BACK ? kBackward<T> : kForward, L = kTy * S;
    __shared__ Shared<PACKED, BACK> sh;
    const int pair = static_cast<int>(blockIdx.x) % pairs;
    const Place at(a.d, pair % chain.tiles, pair / chain.tiles);
    Link<PACKED, BACK> link;
    link.start(a, at.tile, at.b);
    if (threadIdx.x == 0) sh.next = static_cast<int>(link.take(chain, pair, -1));
    join_waves();
    int64_t k = __builtin_amdgcn_readfirstlane(sh.next);
    if (k >= chain.chunks) return;
    join_waves();
    const auto chunk_of = [&](int64_t i) { return BACK ? chain.chunks - 1 - i : i; };
    Rows<T, S, FULL> x, f, dh;
    float entering[kC];
    const auto load = [&](int64_t chunk) {
        const int64_t t0 = chunk * L + at.ty * S;
        const int count = tokens_from<S>(a.T, t0);
        x.load(static_cast<const T*>(a.X) + at.b * a.strideX + t0 * a.ldx + at.ch, a.ldx, count, at.n);
        f.load(static_cast<const T*>(a.F) + at.b * a.strideF + t0 * a.ldf + at.ch, a.ldf, count, at.n);
        if constexpr (BACK) {
            dh.load(static_cast<const T*>(a.dH) + at.b * a.strideDH + t0 * a.lddh + at.ch, a.lddh, count, at.n);
            load4<FULL>(a.T > 0 ? a.states : nullptr,
                        (at.b * ((a.T + kScanStep - 1) / kScanStep) + chunk * (L / kScanStep)) * a.d + at.ch, at.n, entering);
        }
    };
    load(chunk_of(k));
    if constexpr (PACKED) {
        put_code<L>(get_code<L>(a, chain.codes, chunk_of(k) * L, 0), sh.owner[0], sh.marks[0], 0);
        join_waves();
    }
    for (int buffer = 0;; buffer ^= 1) {
        int64_t next = 0;
        if (threadIdx.x == 0) next = link.take(chain, pair, k);
        if constexpr (BACK) k = backward_chunk<T, PACKED, FULL>(a, chain, at, k, next, buffer, link, x, f, dh, entering, sh);
        else k = forward_chunk<T, PACKED, FULL>(a, chain, at, k, next, buffer, link, x, f, sh);
        if (k >= chain.chunks) return;
        load(chunk_of(k));
    }
}

// Few tokens of each sequence, as answers take them: a thread to a channel, no barriers.
// 16 x 1 x 2048 bf16: 2.7 us (as a chunk 6.9).
constexpr int kStepMax = 8;
template <typename T>
__global__ __launch_bounds__(256) void step_kernel(ScanArgs a) {
    const int64_t ch = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, b = blockIdx.z;
    if (ch >= a.d) return;
    const T* x = static_cast<const T*>(a.X) + b * a.strideX + ch;
    const T* f = static_cast<const T*>(a.F) + b * a.strideF + ch;
    T* to = static_cast<T*>(a.H) + b * a.strideH + ch;
    float xs[kStepMax], fs[kStepMax];
    float h = a.h0 != nullptr ? a.h0[b * a.d + ch] : 0.0f;
#pragma unroll
    for (int t = 0; t < kStepMax; ++t) {
        xs[t] = fs[t] = 0.0f;
        if (t < a.T) {
            xs[t] = to_f32(x[t * a.ldx]);
            fs[t] = to_f32(f[t * a.ldf]);
        }
    }
    if (a.states != nullptr && a.T > 0) a.states[b * a.d + ch] = h;
#pragma unroll
    for (int t = 0; t < kStepMax; ++t) {
        if (t >= a.T) break;
        float g, z;
        gates<T>(fs[t], g, z);
        h = __builtin_fmaf(g, h, z * xs[t]);
        if constexpr (sizeof(T) == 2) to[t * a.ldh].bits = static_cast<uint16_t>(bf16_pair(h, 0.0f));
        else to[t * a.ldh] = h;
    }
    a.last[b * a.d + ch] = h;
}

// before the chunks: no word is there yet, no chunk is taken; what the tokens are
__global__ __launch_bounds__(256) void prepare_kernel(ScanArgs a, uint64_t* link, int64_t words, uint32_t* ticket,
                                                      int64_t tickets, int* codes) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, step = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = at; i < words; i += step) link[i] = kEmpty;
    for (int64_t i = at; i < tickets; i += step) ticket[i] = 0;
    if (codes != nullptr)
        for (int64_t t = at; t < a.T; t += step) codes[t] = code_at(a, t);
}

// the batch from its matrix b on (without offsets, where b > 0)
template <typename T>
ScanArgs from_matrix(ScanArgs a, int64_t b) {
    const auto move = [&](auto& p, int64_t stride) {
        if (p != nullptr) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + b * stride);
    };
    const int64_t e = sizeof(T), row = sizeof(float) * a.d;
    move(a.X, e * a.strideX);
    move(a.F, e * a.strideF);
    move(a.dH, e * a.strideDH);
    move(a.H, e * a.strideH);
    move(a.dX, e * a.strideDX);
    move(a.dF, e * a.strideDF);
    move(a.h0, row);
    move(a.dlast, row);
    move(a.last, row);
    move(a.dh0, row);
    move(a.states, row * ((a.T + kScanStep - 1) / kScanStep));
    return a;
}

int64_t chunk_count(int64_t T, int run) { return std::max<int64_t>((T + kTy * run - 1) / (kTy * run), 1); }
int64_t tile_count(int64_t d) { return (d + kTile - 1) / kTile; }

// Workgroups of a launch: as many as run at a time (three to a CU at most; with four the
// chain has more waits and no more rows on their way)
template <typename T, bool BACK>
constexpr int64_t kWorkgroups = BACK && sizeof(T) == 2 ? 512 : 768;

// workgroups that share the chunks of a tile of channels
int64_t sharers(int64_t chunks, int64_t pairs, int64_t workgroups) {
    return std::min(chunks, std::max<int64_t>(workgroups / pairs, 1));
}

template <typename T, bool PACKED, bool BACK>
hipError_t scan(const ScanArgs& a, int batch, hipStream_t stream) {
    const int64_t chunks = chunk_count(a.T, BACK ? kBackward<T> : kForward), tiles = tile_count(a.d);
    if (!BACK && !PACKED && a.T <= kStepMax) {
        hipLaunchKernelGGL(step_kernel<T>, dim3(static_cast<unsigned>((a.d + 255) / 256), 1, static_cast<unsigned>(batch)),
                           dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    const int64_t each = sharers(chunks, tiles * batch, kWorkgroups<T, BACK>);
    uint64_t* link = nullptr;
    uint32_t* ticket = nullptr;
    int* codes = nullptr;
    hipError_t e = hipSuccess;
    if (each > 1 || (PACKED && chunks > 1)) {
        const int64_t words = each > 1 ? chunks * batch * a.d : 0, tickets = each > 1 ? tiles * batch * kTicketStep : 0;
        uint64_t* w = static_cast<uint64_t*>(a.workspace);
        if (each > 1) {
            link = w;
            ticket = reinterpret_cast<uint32_t*>(w + words);
        }
        if (PACKED) codes = reinterpret_cast<int*>(w + words) + tickets;
        const int64_t clear = std::min<int64_t>((std::max(words, a.T) + 1023) / 1024, 2048);
        hipLaunchKernelGGL(prepare_kernel, dim3(static_cast<unsigned>(clear)), dim3(256), 0, stream, a, link, words, ticket,
                           tickets, codes);
        e = hipGetLastError();
    }
    // as many matrices to a launch as keep its threads under 2^32
    const int64_t slice = std::max<int64_t>((int64_t{1} << 22) / tiles, 1);
    for (int64_t b0 = 0; b0 < batch && e == hipSuccess; b0 += slice) {
        const int64_t pairs = std::min(slice, batch - b0) * tiles;
        const Chain chain{link, ticket, codes, chunks, static_cast<int>(tiles)};       // (shared: one slice, as pairs are few)
        const auto launch = [&](auto full) {
            hipLaunchKernelGGL((scan_kernel<T, PACKED, BACK, decltype(full)::value>), dim3(static_cast<unsigned>(pairs * each)),
                               dim3(kThreads), 0, stream, from_matrix<T>(a, b0), chain, static_cast<int>(pairs));
        };
        const auto whole = [&](const void* p, int64_t ld, int64_t stride) {      // rows start on four values
            return reinterpret_cast<uintptr_t>(p) % (kC * sizeof(T)) == 0 && ld % kC == 0 && (batch == 1 || stride % kC == 0);
        };
        const auto state = [](const float* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
        if (a.d % kC == 0 && whole(a.H, a.ldh, a.strideH) && whole(a.dX, a.lddx, a.strideDX) && whole(a.dF, a.lddf, a.strideDF) &&
            state(a.last) && state(a.dh0) && state(a.states))
            launch(std::true_type());
        else launch(std::false_type());
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t scan_bytes(int64_t T, int64_t d, int64_t batch) {
    size_t most = 0;
    for (const int run : {kForward, kBackward<bf16_t>, kBackward<float>}) {
        const int64_t chunks = chunk_count(T, run);
        if (chunks == 1) continue;
        size_t bytes = batch == 1 ? sizeof(int) * static_cast<size_t>(T) : 0;        // (it may be packed)
        if (sharers(chunks, tile_count(d) * batch, kWorkgroups<float, false>) > 1)
            bytes += static_cast<size_t>(chunks * d * batch) * sizeof(uint64_t) +
                     static_cast<size_t>(tile_count(d) * batch * kTicketStep) * sizeof(uint32_t);
        most = std::max(most, bytes);
    }
    return most;
}

hipError_t launch_scan(const ScanArgs& a, bool bf16, int batch, hipStream_t stream) {
    const bool packed = a.offsets.p != nullptr;
    if (bf16) return packed ? scan<bf16_t, true, false>(a, batch, stream) : scan<bf16_t, false, false>(a, batch, stream);
    return packed ? scan<float, true, false>(a, batch, stream) : scan<float, false, false>(a, batch, stream);
}
hipError_t launch_scan_backward(const ScanArgs& a, bool bf16, int batch, hipStream_t stream) {
    const bool packed = a.offsets.p != nullptr;
    if (bf16) return packed ? scan<bf16_t, true, true>(a, batch, stream) : scan<bf16_t, false, true>(a, batch, stream);
    return packed ? scan<float, true, true>(a, batch, stream) : scan<float, false, true>(a, batch, stream);
}

}  // namespace galore
