// Embedding: rows of a matrix by token id, and the matrix's gradient, the rows of the
// incoming gradient summed by token id in the order of the tokens.
//
// Lookup is one read of a row and one write of it: 16384 of 4096 bf16 54 us (5.0 TB/s).
//
// The gradient first sorts the tokens by id, stable. Up to 16384 tokens in one launch: its
// workgroups own consecutive ranges of ids; each reads all ids (from the caches), keeps
// those of its range in token order, sorts them in LDS, which holds them all if need be,
// and writes them where the count of smaller ids says. More tokens take the digits of the
// id in turn, eight bits each, the least first, two launches to a digit: the workgroups,
// 256 at most, count the digits of their tokens, then place these behind those of smaller
// digits and of workgroups before. Either way no workgroup waits for another, the ids are
// read equally often whichever there are, and the order is always the same (atomics count
// within a workgroup, or set bits). The next launch clears the rows that no token has and
// walks over chunks of the sorted tokens, a thread eight columns, several rows on their way
// at a time: a run of one id inside a chunk, or one that ends within the next, is summed
// and stored by the chunk in which it begins; a longer one (padding words, the commonest
// tokens) leaves a partial sum in each chunk, which the last launch adds in order. Sums in
// fp32, one rounding to G's type.
// 16384 tokens of 4096 bf16, 32000 ids as text has them: sorted 14 us, summed and cleared
// 83 (4.8 TB/s; two thirds of it writes, which alone reach 5.0), joined 9; 1003 tokens of
// 1024 fp32: 6, 27 and 5; half of the 16384 one id: 26, 86 and 33. 2^20 tokens of 1024 bf16,
// ids by frequency: 85, 459 (4.8 TB/s) and 317, where a workgroup to 512 columns adds the
// parts of the commonest id. The sort in LDS is latency: one workgroup to a CU, steps over
// the ids with a barrier each (sorting there by 4-bit digits with the ids read twice took
// 98 us). By digits of the id the sort of few tokens is longer: a call on rows of 64 takes
// 63 us so, 49 by ranges at 16384 tokens (ids spread evenly 53 and 29), 38 and 24 at 1003.
#include <algorithm>

#include "mx.hpp"
#include "layers.hpp"

namespace galore {
namespace {

template <typename T, typename O>
__global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a) {
    const int64_t g = static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x, e = 8 * g;
    if (e >= a.d) return;
    const int d = static_cast<int>(a.d);
    for (int64_t row = first_row(); row < a.tokens; row += row_step()) {
        const int64_t id = a.ids.at(row);
        float x[8];
        if (id >= 0 && id < a.vocab) {
            load8(static_cast<const T*>(a.W) + id * a.ldw, e, d, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= a.scale;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = id < 0 ? 0.0f : __uint_as_float(0x7fc00000u);
        }
        store8(static_cast<O*>(a.out) + row * a.ldo + e, a.d - e, x);
    }
}

// ---- the gradient's tokens by id --------------------------------------------------

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kTokenBits = 14, kSortMax = 1 << kTokenBits;        // tokens in LDS: two buffers of 4 bytes each
constexpr int kRange = 32768;             // ids of a workgroup's range, at most
static_assert(kRange <= 1 << (32 - kTokenBits), "a place in the range and a token's number fit a word");
constexpr int kRankMax = 512;             // tokens of a range that are sorted by counting
constexpr int kDigit = 8, kBins = 1 << kDigit;
constexpr int kPerThread = 8, kScan = kPerThread * kSortThreads;   // tokens of a step over the ids

struct Sorted {
    int* token;                // token numbers by id, then by number
    int* id;
    int* count;                // tokens that have a row
    uint32_t* present;         // a bit for every row: whether a token has it
    float* part;               // chunks x 2 x d: the run that comes from the chunk before, the one that goes on
    int chunk;                 // sorted tokens to a workgroup's walk
    bool once_in, once_out;    // rows of dY, of G are bf16 on 16 bytes: past the caches
};

struct SortArgs {
    Indices ids;
    int64_t tokens, vocab, per;     // per: ids of a range, a multiple of 32
    Sorted s;
};

// exclusive sum over the threads of a workgroup, and the total; `red` holds kSortWaves
__device__ __forceinline__ int exclusive_sum(int v, int* red, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const int o = __shfl_up(s, k);
        if (lane >= k) s += o;
    }
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        const int r = red[w];
        before += w < wave ? r : 0;
        all += r;
    }
    total = all;
    return before + s - v;
}

// the lanes that are `in` and have this lane's digit (a ballot for each of its bits)
__device__ __forceinline__ uint64_t same_digit(int digit, bool in) {
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
        const uint64_t m = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? m : ~m;
    }
    return same;
}

// Calls put(place, token, id) for the tokens with lo <= id < hi, places in token order.
// `inside`: their number, `under`: that of tokens with 0 <= id < lo.
template <typename F>
__device__ __forceinline__ void gather_range(const SortArgs& a, int64_t lo, int64_t hi, int* red, int& inside, int& under,
                                             F put) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0, below = 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kScan) {
        // a wave's tokens are neighbours, and so are a ballot's
        const int64_t first = t0 + wave * (64 * kPerThread) + lane;
        int64_t id[kPerThread];
        if (a.ids.wide) {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i)
                id[i] = first + 64 * i < a.tokens ? static_cast<const int64_t*>(a.ids.p)[first + 64 * i] : -1;
        } else {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i)
                id[i] = first + 64 * i < a.tokens ? static_cast<const int32_t*>(a.ids.p)[first + 64 * i] : -1;
        }
        int of_wave = 0, at[kPerThread];
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const uint64_t m = __ballot(id[i] >= lo && id[i] < hi);
            at[i] = of_wave + __popcll(m & ((1ull << lane) - 1));
            of_wave += __popcll(m);
            below += id[i] >= 0 && id[i] < lo;
        }
        __syncthreads();
        if (lane == 0) red[wave] = of_wave;
        __syncthreads();
        int before = base;
        for (int w = 0; w < kSortWaves; ++w) {
            const int r = red[w];
            before += w < wave ? r : 0;
            base += r;
        }
#pragma unroll
        for (int i = 0; i < kPerThread; ++i)
            if (id[i] >= lo && id[i] < hi) put(before + at[i], static_cast<int>(first + 64 * i), static_cast<int>(id[i]));
    }
    inside = base;
    exclusive_sum(below, red, under);
}

__global__ __launch_bounds__(kSortThreads) void sort_kernel(SortArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t buffer[2][kSortMax];     // place in the range, token's number
    __shared__ int red[kSortWaves];
    __shared__ int bins[kSortWaves][kBins];
    __shared__ uint32_t present[kRange / 32];    // bits of the range's ids
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t lo = a.per * blockIdx.x, hi = min(lo + a.per, a.vocab);
    for (int w = threadIdx.x; w < kRange / 32; w += kSortThreads) present[w] = 0;
    int inside, under;
    gather_range(a, lo, hi, red, inside, under, [&](int at, int t, int id) {
        buffer[0][at] = static_cast<uint32_t>(id - lo) << kTokenBits | static_cast<uint32_t>(t);
    });
    if (hi == a.vocab && threadIdx.x == 0) *a.s.count = inside + under;
    int from = 0;
    if (inside <= kRankMax) {
        // few: a token's place is the number of smaller words
        const int p = threadIdx.x;
        if (p >= inside && p < (inside + 3) / 4 * 4) buffer[0][p] = 0xffffffffu;
        __syncthreads();
        const uint32_t mine = p < inside ? buffer[0][p] : 0xffffffffu;
        int place = 0;
        if (wave * 64 < inside) {
            for (int i = 0; i < inside; i += 4) {
                const u32x4 k = *reinterpret_cast<const u32x4*>(buffer[0] + i);
                place += (k[0] < mine) + (k[1] < mine) + (k[2] < mine) + (k[3] < mine);
            }
        }
        if (p < inside) buffer[1][place] = mine;
        from = 1;
        __syncthreads();
    } else {
        __syncthreads();
        // stable sort by digits of the id, the least first: each wave has a run of the
        // tokens, places are by digit, then by wave, then by place in the run
        const int run = (inside + kSortThreads - 1) / kSortThreads * 64;
        for (int shift = kTokenBits; (hi - 1 - lo) >> (shift - kTokenBits); shift += kDigit, from ^= 1) {
            for (int b = threadIdx.x; b < kSortWaves * kBins; b += kSortThreads) bins[b / kBins][b % kBins] = 0;
            __syncthreads();
            // the first of a wave's lanes with the same digit counts them
            for (int i = 0; i < run; i += 64) {
                const int p = wave * run + i + lane;
                const bool in = p < inside;
                const int digit = in ? static_cast<int>(buffer[from][p] >> shift) & (kBins - 1) : 0;
                const uint64_t same = same_digit(digit, in);
                if (in && __builtin_ctzll(same) == lane) atomicAdd(&bins[wave][digit], __popcll(same));
            }
            __syncthreads();
            // where the tokens of each digit go, wave by wave
            constexpr int kEach = kSortWaves * kBins / kSortThreads;
            int v[kEach], all = 0, total;
#pragma unroll
            for (int b = 0; b < kEach; ++b) {
                const int at = kEach * threadIdx.x + b;
                v[b] = bins[at % kSortWaves][at / kSortWaves];
                all += v[b];
            }
            int before = exclusive_sum(all, red, total);
#pragma unroll
            for (int b = 0; b < kEach; ++b) {
                const int at = kEach * threadIdx.x + b;
                bins[at % kSortWaves][at / kSortWaves] = before;
                before += v[b];
            }
            __syncthreads();
            for (int i = 0; i < run; i += 64) {
                const int p = wave * run + i + lane;
                const bool in = p < inside;
                const uint32_t mine = in ? buffer[from][p] : 0;
                const int digit = static_cast<int>(mine >> shift) & (kBins - 1);
                const uint64_t same = same_digit(digit, in);
                const int start = bins[wave][digit];
                if (in) buffer[from ^ 1][start + __popcll(same & ((1ull << lane) - 1))] = mine;
                __builtin_amdgcn_wave_barrier();
                if (in && __builtin_ctzll(same) == lane) atomicAdd(&bins[wave][digit], __popcll(same));
                __builtin_amdgcn_wave_barrier();
            }
            __syncthreads();
        }
    }
    for (int p = threadIdx.x; p < inside; p += kSortThreads) {
        const uint32_t mine = buffer[from][p], place = mine >> kTokenBits;
        a.s.token[under + p] = static_cast<int>(mine & (kSortMax - 1));
        a.s.id[under + p] = static_cast<int>(lo + place);
        if (p == 0 || buffer[from][p - 1] >> kTokenBits != place) atomicOr(present + place / 32, 1u << (place & 31));
    }
    __syncthreads();
    for (int64_t w = threadIdx.x; lo + 32 * w < hi; w += kSortThreads) a.s.present[lo / 32 + w] = present[w];
}

// ---- the same for long lists, by digits of the id ------------------------------------
//
// A workgroup's tokens are `span` neighbours, taken in steps of kStep; of a step a wave has
// neighbours too.
constexpr int kEachStep = 4, kStep = kEachStep * kSortThreads;
constexpr int kDigitGroups = 256;          // workgroups at most: each reads the counts of all

struct DigitArgs {
    Indices ids;                           // FIRST: tokens are their numbers; else
    const int *from_token, *from_id;       // as the digit before left them
    int *to_token, *to_id;
    int* count;                            // tokens that have a row: written with the first digit, read later
    uint32_t* present;                     // cleared with the first digit
    int* bins;                             // workgroups x kBins: their tokens of each digit
    int64_t tokens, vocab, span;
    int shift;
};

// the id at place p, or -1: none there, or none that has a row
template <bool FIRST>
__device__ __forceinline__ int id_of_place(const DigitArgs& a, int64_t p, int64_t n) {
    if (p >= n) return -1;
    if (!FIRST) return a.from_id[p];
    const int64_t id = a.ids.at(p);
    return id >= 0 && id < a.vocab ? static_cast<int>(id) : -1;
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void count_kernel(DigitArgs a) {
    __shared__ int bins[kSortWaves][kBins];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (FIRST) {
        const int64_t at = static_cast<int64_t>(blockIdx.x) * kSortThreads + threadIdx.x;
        for (int64_t w = at; w < (a.vocab + 31) / 32; w += static_cast<int64_t>(gridDim.x) * kSortThreads) a.present[w] = 0;
    }
    for (int b = threadIdx.x; b < kSortWaves * kBins; b += kSortThreads) bins[b / kBins][b % kBins] = 0;
    __syncthreads();
    const int64_t n = FIRST ? a.tokens : *a.count, stop = min(a.span * (blockIdx.x + 1), n);
    for (int64_t t0 = a.span * blockIdx.x; t0 < stop; t0 += kStep) {
        const int64_t first = t0 + wave * (64 * kEachStep) + lane;
        int id[kEachStep];
#pragma unroll
        for (int i = 0; i < kEachStep; ++i) id[i] = id_of_place<FIRST>(a, first + 64 * i, n);
#pragma unroll
        for (int i = 0; i < kEachStep; ++i) {
            const bool in = id[i] >= 0;
            const int digit = in ? id[i] >> a.shift & (kBins - 1) : 0;
            const uint64_t same = same_digit(digit, in);
            if (in && __builtin_ctzll(same) == lane) atomicAdd(&bins[wave][digit], __popcll(same));
        }
    }
    __syncthreads();
    if (threadIdx.x < kBins) {
        int all = 0;
        for (int w = 0; w < kSortWaves; ++w) all += bins[w][threadIdx.x];
        a.bins[static_cast<int64_t>(blockIdx.x) * kBins + threadIdx.x] = all;
    }
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void place_kernel(DigitArgs a) {
    constexpr int kParts = kSortThreads / kBins;
    __shared__ int bins[kSortWaves][kBins];
    __shared__ int all_of[kParts][kBins], before_of[kParts][kBins], base[kBins];
    __shared__ int red[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // where this workgroup's tokens of each digit go
    {
        const int bin = threadIdx.x % kBins, part = threadIdx.x / kBins;
        int all = 0, before = 0;
        for (int64_t g = part; g < gridDim.x; g += kParts) {
            const int v = a.bins[g * kBins + bin];
            all += v;
            before += g < blockIdx.x ? v : 0;
        }
        all_of[part][bin] = all;
        before_of[part][bin] = before;
        __syncthreads();
        all = before = 0;
        if (threadIdx.x < kBins) {
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                all += all_of[k][bin];
                before += before_of[k][bin];
            }
        }
        int total;
        const int smaller = exclusive_sum(all, red, total);
        if (threadIdx.x < kBins) base[bin] = smaller + before;
        if (FIRST && blockIdx.x == 0 && threadIdx.x == 0) *a.count = total;
    }
    const int64_t n = FIRST ? a.tokens : *a.count, stop = min(a.span * (blockIdx.x + 1), n);
    for (int64_t t0 = a.span * blockIdx.x; t0 < stop; t0 += kStep) {
        const int64_t first = t0 + wave * (64 * kEachStep) + lane;
        int id[kEachStep], token[kEachStep], rank[kEachStep];
#pragma unroll
        for (int i = 0; i < kEachStep; ++i) {
            id[i] = id_of_place<FIRST>(a, first + 64 * i, n);
            token[i] = FIRST ? static_cast<int>(first + 64 * i) : id[i] >= 0 ? a.from_token[first + 64 * i] : 0;
        }
        __syncthreads();                   // (the step before has read its bins)
        for (int b = threadIdx.x; b < kSortWaves * kBins; b += kSortThreads) bins[b / kBins][b % kBins] = 0;
        __syncthreads();
        // a token's rank among its wave's with the same digit; the first of these lanes counts them
#pragma unroll
        for (int i = 0; i < kEachStep; ++i) {
            const bool in = id[i] >= 0;
            const int digit = in ? id[i] >> a.shift & (kBins - 1) : 0;
            const uint64_t same = same_digit(digit, in);
            const int leader = in ? static_cast<int>(__builtin_ctzll(same)) : lane;
            int old = 0;
            if (in && leader == lane) old = atomicAdd(&bins[wave][digit], __popcll(same));
            rank[i] = __shfl(old, leader) + __popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        if (threadIdx.x < kBins) {
            int at = base[threadIdx.x];
            for (int w = 0; w < kSortWaves; ++w) {
                const int v = bins[w][threadIdx.x];
                bins[w][threadIdx.x] = at;
                at += v;
            }
            base[threadIdx.x] = at;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEachStep; ++i) {
            if (id[i] < 0) continue;
            const int at = bins[wave][id[i] >> a.shift & (kBins - 1)] + rank[i];
            a.to_token[at] = token[i];
            a.to_id[at] = id[i];
        }
    }
}

// a bit for every row whose tokens' run begins here
__global__ __launch_bounds__(256) void mark_kernel(Sorted s) {
    const int n = *s.count;
    for (int64_t p = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; p < n; p += static_cast<int64_t>(gridDim.x) * 256) {
        const int id = s.id[p];
        if (p == 0 || s.id[p - 1] != id) atomicOr(s.present + id / 32, 1u << (id & 31));
    }
}

// ---- the sums -----------------------------------------------------------------------

template <typename G>
__device__ __forceinline__ void put_row(const EmbeddingGradArgs& a, bool once, int id, int64_t e, const float (&s)[8]) {
    G* row = static_cast<G*>(a.G) + id * a.ldg;
    float y[8];
    if (a.accumulate) {
        load8(row, static_cast<int>(e), static_cast<int>(a.d), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += s[i] * a.scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = s[i] * a.scale;
    }
    store8(row + e, a.d - e, y, once);
}

// Whether the run of one id that goes on past `end`, a chunk's end, ends within the chunk
// after it (and is then the first one's to sum)
__device__ __forceinline__ bool ends_in_next(const Sorted& s, int64_t end, int64_t n, int id) {
    return end + s.chunk >= n || s.id[end + s.chunk] != id;
}

// The sums of chunk c, columns e to e + 7. A lane knows one sorted token of this chunk and
// the next, so that where runs end is seen by ballots.
constexpr int kChunkMax = 32;
template <typename T, typename G>
__device__ __forceinline__ void sum_chunk(const EmbeddingGradArgs& a, const Sorted& s, int64_t c, int64_t n, int e) {
    constexpr int kRows = sizeof(T) == 2 ? 8 : 4;         // rows on their way at a time
    const int d = static_cast<int>(a.d), lane = threadIdx.x & 63;
    const T* dY = static_cast<const T*>(a.dY);
    const int64_t p0 = c * s.chunk;
    const int my_id = p0 + lane < n ? s.id[p0 + lane] : -1, my_token = p0 + lane < n ? s.token[p0 + lane] : 0;
    const int whole = static_cast<int>(min(static_cast<int64_t>(s.chunk), n - p0));
    const auto id_of = [&](int p) { return __builtin_amdgcn_readlane(my_id, p); };
    // lanes from `p` on with the same id
    const auto run_from = [&](int p) {
        const uint64_t other = ~__ballot(my_id == id_of(p)) >> p;
        return other != 0 ? static_cast<int>(__builtin_ctzll(other)) : 64 - p;
    };
    int p = 0, end = whole;
    bool head = false, tail = false;                      // the first, the last run is a part
    const int first = run_from(0);
    if (c > 0 && s.id[p0 - 1] == id_of(0)) {
        const bool began = c == 1 || s.id[p0 - s.chunk - 1] != id_of(0);      // in the chunk before, which may sum it all
        if (began && first <= whole) p = first;
        else head = true;
    }
    if (p >= whole) return;
    // (a run that fills the chunk and comes from before it is a head only)
    if (id_of(whole) == id_of(whole - 1) && !(head && first >= whole)) {
        const int more = run_from(whole);
        if (more < s.chunk || ends_in_next(s, p0 + whole, n, id_of(whole))) end = whole + min(more, s.chunk);
        else tail = true;
    }
    float sum[8] = {};
    int id = id_of(p);
    const auto load = [&](Eight<T> (&r)[kRows], int from) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            r[i].clear();
            if (from + i < end) r[i].load(dY + __builtin_amdgcn_readlane(my_token, from + i) * a.lddy, e, d, s.once_in);
        }
    };
    const auto add = [&](Eight<T> (&r)[kRows], int from) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (from + i >= end) break;
            const int next = id_of(from + i);
            if (next != id) {
                if (head) store8(s.part + 2 * c * a.d + e, a.d - e, sum);
                else put_row<G>(a, s.once_out, id, e, sum);
                head = false;
                id = next;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
            }
            r[i].settle(e, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += r[i][j];
        }
    };
    for (; p < end; p += kRows) {
        Eight<T> r[kRows];
        load(r, p);
        add(r, p);
    }
    if (head) store8(s.part + 2 * c * a.d + e, a.d - e, sum);
    else if (tail) store8(s.part + (2 * c + 1) * a.d + e, a.d - e, sum);
    else put_row<G>(a, s.once_out, id, e, sum);
}

// The first `sums` workgroups along the grid sum chunks, the others clear 32 rows each
template <typename T, typename G>
__global__ __launch_bounds__(256) void sum_kernel(EmbeddingGradArgs a, Sorted s, int64_t sums) {
    // (lanes past the row's end stay: they know sorted tokens)
    const int64_t e = 8 * (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x);
    if (blockIdx.x < sums) {
        const int64_t n = *s.count, chunks = (n + s.chunk - 1) / s.chunk;
        for (int64_t c = blockIdx.x; c < chunks; c += sums) sum_chunk<T, G>(a, s, c, n, static_cast<int>(e));
        return;
    }
    const float zero[8] = {};
    for (int64_t w = blockIdx.x - sums; w < (a.vocab + 31) / 32; w += gridDim.x - sums) {
        const uint32_t present = s.present[w];
        const int rows = static_cast<int>(min(a.vocab - 32 * w, static_cast<int64_t>(32)));
        G* row = static_cast<G*>(a.G) + 32 * w * a.ldg + e;
        for (int r = 0; r < rows; ++r, row += a.ldg)
            if (!(present >> r & 1) && e < a.d) store8(row, a.d - e, zero, s.once_out);
    }
}

// The runs that lie over several chunks: a workgroup looks at kJoin chunks in which one may
// begin and adds its parts, four slices of them side by side, in order
constexpr int kJoin = 8, kSlices = 4;
template <typename G>
__global__ __launch_bounds__(256) void join_kernel(EmbeddingGradArgs a, Sorted s) {
    __shared__ float red[kSlices][8][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
    const int64_t e = 8 * (static_cast<int64_t>(blockIdx.y) * 64 + lane);
    const int d = static_cast<int>(a.d);
    const int64_t n = *s.count, chunks = (n + s.chunk - 1) / s.chunk;
    for (int64_t c0 = blockIdx.x * static_cast<int64_t>(kJoin); c0 < chunks; c0 += gridDim.x * static_cast<int64_t>(kJoin)) {
        // a lane for each chunk; a run that fills one begins before it
        bool begins = false;
        if (lane < kJoin && c0 + lane < chunks) {
            const int64_t c = c0 + lane, end = (c + 1) * s.chunk;
            const int id = s.id[min(end, n) - 1], after = end < n ? s.id[end] : -1;
            const int further = end + s.chunk < n ? s.id[end + s.chunk] : -1, before = c > 0 ? s.id[c * s.chunk - 1] : -1;
            begins = after == id && further == id && before != id;
        }
        for (uint64_t todo = __ballot(begins); todo != 0; todo &= todo - 1) {
            const int64_t c = c0 + __builtin_ctzll(todo);
            const int id = s.id[(c + 1) * s.chunk];
            // chunks c + 1 .. last begin inside the run
            int64_t lo = c + 1, hi = chunks;
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (s.id[mid * s.chunk] == id) lo = mid + 1;
                else hi = mid;
            }
            const int64_t parts = lo - c, each = (parts + kSlices - 1) / kSlices;
            float sum[8] = {};
            if (e < d) {
                const int64_t stop = min((slice + 1) * each, parts);
#pragma unroll 4
                for (int64_t k = slice * each; k < stop; ++k) {
                    float x[8];
                    load8(s.part + (2 * (c + k) + (k == 0 ? 1 : 0)) * a.d, static_cast<int>(e), d, x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += x[i];
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) red[slice][i][lane] = sum[i];
            __syncthreads();
            if (slice == 0 && e < d) {
#pragma unroll
                for (int w = 1; w < kSlices; ++w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i] += red[w][i][lane];
                put_row<G>(a, s.once_out, id, e, sum);
            }
        }
    }
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }
// sorted tokens to a chunk: fewer where that leaves workgroups to the whole chip
int chunk_of(int64_t tokens) { return tokens >= 8192 ? kChunkMax : 8; }
size_t chunk_count(int64_t tokens) { return static_cast<size_t>((tokens + chunk_of(tokens) - 1) / chunk_of(tokens)); }

// the workspace: count, sorted tokens, their ids, bits of the rows, partial sums; the
// digits' counts and other lists lie where the partial sums come later
struct Layout {
    size_t token, id, present, part, other_id, bins, bytes;
};
Layout layout(int64_t tokens, int64_t vocab, int64_t d) {
    Layout l;
    const size_t list = round_up(sizeof(int) * static_cast<size_t>(tokens));
    l.token = 256;
    l.id = l.token + list;
    l.present = l.id + list;
    l.part = l.present + round_up(sizeof(uint32_t) * static_cast<size_t>((vocab + 31) / 32));
    l.other_id = l.part + list;
    l.bins = l.other_id + list;
    l.bytes = l.part + round_up(sizeof(float) * 2 * chunk_count(tokens) * static_cast<size_t>(d));
    if (tokens > kSortMax) l.bytes = std::max(l.bytes, l.bins + sizeof(int) * kDigitGroups * kBins);
    return l;
}

// the sorted tokens and the bits of their rows
hipError_t sort_by_ranges(const EmbeddingGradArgs& a, const Sorted& s, hipStream_t stream) {
    // ranges of ids: about 64 tokens each where they are spread, 256 ranges at most
    const int64_t want = std::max<int64_t>(std::min<int64_t>(a.tokens / 64, 256), (a.vocab + kRange - 1) / kRange);
    const int64_t per = std::min<int64_t>(((a.vocab + want - 1) / want + 31) / 32 * 32, kRange);
    const SortArgs sort{a.ids, a.tokens, a.vocab, per, s};
    hipLaunchKernelGGL(sort_kernel, dim3(static_cast<unsigned>((a.vocab + per - 1) / per)), dim3(kSortThreads), 0, stream, sort);
    return hipGetLastError();
}
hipError_t sort_by_digits(const EmbeddingGradArgs& a, const Sorted& s, char* workspace, const Layout& l, hipStream_t stream) {
    const int64_t steps = (a.tokens + kStep - 1) / kStep;
    const int64_t span = (steps + kDigitGroups - 1) / kDigitGroups * kStep;
    const unsigned groups = static_cast<unsigned>((a.tokens + span - 1) / span);
    int* lists[2][2] = {{s.token, s.id},
                        {reinterpret_cast<int*>(workspace + l.part), reinterpret_cast<int*>(workspace + l.other_id)}};
    int digits = 1;
    while ((a.vocab - 1) >> (kDigit * digits)) ++digits;
    DigitArgs g{a.ids, nullptr, nullptr, nullptr, nullptr, s.count, s.present, reinterpret_cast<int*>(workspace + l.bins),
                a.tokens, a.vocab, span, 0};
    for (int k = 0; k < digits; ++k) {
        int** to = lists[(digits - 1 - k) & 1];       // the last digit's are the sorted ones
        g.to_token = to[0];
        g.to_id = to[1];
        g.shift = kDigit * k;
        if (k == 0) {
            hipLaunchKernelGGL(count_kernel<true>, dim3(groups), dim3(kSortThreads), 0, stream, g);
            hipLaunchKernelGGL(place_kernel<true>, dim3(groups), dim3(kSortThreads), 0, stream, g);
        } else {
            hipLaunchKernelGGL(count_kernel<false>, dim3(groups), dim3(kSortThreads), 0, stream, g);
            hipLaunchKernelGGL(place_kernel<false>, dim3(groups), dim3(kSortThreads), 0, stream, g);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        g.from_token = to[0];
        g.from_id = to[1];
    }
    hipLaunchKernelGGL(mark_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((a.tokens + 255) / 256, 2048))), dim3(256), 0,
                       stream, s);
    return hipGetLastError();
}

template <typename T, typename G>
hipError_t embedding_grad(const EmbeddingGradArgs& a, hipStream_t stream) {
    char* w = static_cast<char*>(a.workspace);
    const Layout l = layout(a.tokens, a.vocab, a.d);
    const Sorted s{reinterpret_cast<int*>(w + l.token),
                   reinterpret_cast<int*>(w + l.id),
                   reinterpret_cast<int*>(w),
                   reinterpret_cast<uint32_t*>(w + l.present),
                   reinterpret_cast<float*>(w + l.part),
                   chunk_of(a.tokens),
                   sizeof(T) == 2 && rows_on_16(static_cast<const T*>(a.dY), a.lddy, 0, 1),
                   sizeof(G) == 2 && rows_on_16(static_cast<const G*>(a.G), a.ldg, 0, 1)};
    hipError_t e = a.tokens <= kSortMax ? sort_by_ranges(a, s, stream) : sort_by_digits(a, s, w, l, stream);
    if (e != hipSuccess) return e;
    const int64_t groups = (a.d + 7) / 8;
    const unsigned wide = static_cast<unsigned>(std::min<int64_t>((groups + 63) / 64 * 64, 256));
    const int64_t sums = std::min<int64_t>(chunk_count(a.tokens), 1 << 16);
    const int64_t clears = a.accumulate ? 0 : std::min<int64_t>((a.vocab + 31) / 32, 1 << 16);
    if (sums + clears == 0) return hipSuccess;
    hipLaunchKernelGGL((sum_kernel<T, G>),
                       dim3(static_cast<unsigned>(sums + clears), static_cast<unsigned>((groups + wide - 1) / wide)), dim3(wide), 0,
                       stream, a, s, sums);
    e = hipGetLastError();
    if (e != hipSuccess || a.tokens <= 2 * s.chunk) return e;
    hipLaunchKernelGGL(join_kernel<G>, dim3(static_cast<unsigned>((sums + kJoin - 1) / kJoin), static_cast<unsigned>((groups + 63) / 64)),
                       dim3(256), 0, stream, a, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_lookup(const LookupArgs& a, bool w_bf16, bool out_bf16, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    const RowGrid g = row_grid(a.tokens, (a.d + 7) / 8, 1);
    if (w_bf16) {
        if (out_bf16) hipLaunchKernelGGL((lookup_kernel<bf16_t, bf16_t>), g.grid, g.block, 0, stream, a);
        else hipLaunchKernelGGL((lookup_kernel<bf16_t, float>), g.grid, g.block, 0, stream, a);
    } else {
        if (out_bf16) hipLaunchKernelGGL((lookup_kernel<float, bf16_t>), g.grid, g.block, 0, stream, a);
        else hipLaunchKernelGGL((lookup_kernel<float, float>), g.grid, g.block, 0, stream, a);
    }
    return hipGetLastError();
}

size_t embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t d) { return layout(tokens, vocab, d).bytes; }

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, bool dy_bf16, bool g_bf16, hipStream_t stream) {
    if (dy_bf16) return g_bf16 ? embedding_grad<bf16_t, bf16_t>(a, stream) : embedding_grad<bf16_t, float>(a, stream);
    return g_bf16 ? embedding_grad<float, bf16_t>(a, stream) : embedding_grad<float, float>(a, stream);
}

}  // namespace galore
