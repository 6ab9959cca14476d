// Embedding: rows of a matrix by token id, and the matrix's gradient, the rows of the
// incoming gradient summed by token id in the order of the tokens.
//
// Lookup is one read of a row and one write of it.
//
// The gradient's first launch sorts the tokens by id and clears the rows that no token
// has. Its workgroups own consecutive ranges of ids; each reads all ids (from the
// caches), keeps those of its range in token order, sorts them by id in LDS, stable, and
// writes them where the count of smaller ids says: no workgroup waits for another and
// nothing is counted by atomics, so that the order is always the same. A range whose
// tokens do not fit LDS is halved until they do, or until it is one id, whose tokens need
// no sort. The second launch walks over chunks of the sorted tokens, a thread eight
// columns: a run of one id inside a chunk, or one that ends within the next, is summed
// and stored by the chunk in which it begins; a longer one (padding words, the commonest
// tokens) leaves a partial sum in each chunk, which the third launch adds in order.
// Sums in fp32, one rounding to G's type.
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
constexpr int kSortMax = 7168;            // tokens in LDS: two buffers of 8 bytes each
constexpr int kDigit = 4, kBins = 1 << kDigit;
constexpr int kChunk = 32;                // sorted tokens to a workgroup's walk

struct Sorted {
    int* token;                // token numbers by id, then by number
    int* id;
    int* count;                // tokens that have a row
    float* part;               // chunks x 2 x d: the run that comes from the chunk before, the one that goes on
};

struct SortArgs {
    Indices ids;
    int64_t tokens, vocab;
    Sorted s;
    void* G;
    int64_t d, ldg;
    bool clear;
};

// exclusive sum over the threads of a workgroup, and the total; `red` holds kSortWaves + 1
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

// tokens with lo <= id < hi, and those with 0 <= id < lo
__device__ __forceinline__ void count_range(const SortArgs& a, int64_t lo, int64_t hi, int* red, int& inside, int& under) {
    int n = 0, m = 0;
    for (int64_t t = threadIdx.x; t < a.tokens; t += kSortThreads) {
        const int64_t id = a.ids.at(t);
        n += id >= lo && id < hi;
        m += id >= 0 && id < lo;
    }
    exclusive_sum(n, red, inside);
    exclusive_sum(m, red, under);
}

// calls put(place, token, id) for the tokens with lo <= id < hi, places in token order
template <typename F>
__device__ __forceinline__ void gather_range(const SortArgs& a, int64_t lo, int64_t hi, int* red, F put) {
    // a wave takes 64 tokens in a row, the workgroup's waves 1024
    int base = 0;
    for (int64_t t0 = 0; t0 < a.tokens; t0 += kSortThreads) {
        const int64_t t = t0 + threadIdx.x;
        const int64_t id = t < a.tokens ? a.ids.at(t) : -1;
        const bool in = id >= lo && id < hi;
        int total;
        const int at = exclusive_sum(in, red, total);
        if (in) put(base + at, static_cast<int>(t), static_cast<int>(id));
        base += total;
    }
}

template <typename G>
__device__ void clear_rows(const SortArgs& a, int64_t first, int64_t last) {
    const int64_t n = a.d;
    for (int64_t r = first; r < last; ++r) {
        G* row = static_cast<G*>(a.G) + r * a.ldg;
        const float zero[8] = {};
        for (int64_t e = 8 * threadIdx.x; e < n; e += 8 * kSortThreads) store8(row + e, n - e, zero);
    }
}

template <typename G>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(SortArgs a) {
    __shared__ int2 buffer[2][kSortMax];
    __shared__ int red[kSortWaves];
    __shared__ int bins[kSortWaves][kBins];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t per = (a.vocab + gridDim.x - 1) / gridDim.x;
    int64_t lo = per * blockIdx.x;
    const int64_t end = min(lo + per, a.vocab);
    if (blockIdx.x == gridDim.x - 1) {           // the count of all
        int inside, under;
        count_range(a, 0, a.vocab, red, inside, under);
        if (threadIdx.x == 0) *a.s.count = inside;
    }
    int64_t hi = end;
    while (lo < end) {
        int inside, under;
        count_range(a, lo, hi, red, inside, under);
        if (inside > kSortMax && hi - lo > 1) {
            hi = lo + (hi - lo) / 2;
            continue;
        }
        if (hi - lo == 1) {
            gather_range(a, lo, hi, red, [&](int at, int t, int id) {
                a.s.token[under + at] = t;
                a.s.id[under + at] = id;
            });
            if (a.clear && inside == 0) clear_rows<G>(a, lo, hi);
        } else {
            gather_range(a, lo, hi, red, [&](int at, int t, int id) { buffer[0][at] = make_int2(id, t); });
            __syncthreads();
            // stable sort by digits of the id, the least first: each wave has a run of the
            // tokens, places are by digit, then by wave, then by place in the run
            const int run = (inside + kSortThreads - 1) / kSortThreads * 64;
            int from = 0;
            for (int shift = 0; (hi - 1 - lo) >> shift; shift += kDigit, from ^= 1) {
                int mine = 0;                    // lane b: tokens of digit b
                for (int i = 0; i < run; i += 64) {
                    const int p = wave * run + i + lane;
                    const bool in = p < inside;
                    const int digit = in ? static_cast<int>((buffer[from][p].x - lo) >> shift) & (kBins - 1) : 0;
                    for (int b = 0; b < kBins; ++b) {
                        const int n = __popcll(__ballot(in && digit == b));
                        mine += lane == b ? n : 0;
                    }
                }
                if (lane < kBins) bins[wave][lane] = mine;
                __syncthreads();
                // bins in the order (digit, wave)
                const int at = threadIdx.x;
                int v = 0;
                if (at < kBins * kSortWaves) v = bins[at % kSortWaves][at / kSortWaves];
                int total;
                const int before = exclusive_sum(v, red, total);
                __syncthreads();
                if (at < kBins * kSortWaves) bins[at % kSortWaves][at / kSortWaves] = before;
                __syncthreads();
                mine = lane < kBins ? bins[wave][lane] : 0;   // lane b: where the next token of digit b goes
                for (int i = 0; i < run; i += 64) {
                    const int p = wave * run + i + lane;
                    const bool in = p < inside;
                    const int2 v2 = in ? buffer[from][p] : make_int2(0, 0);
                    const int digit = in ? static_cast<int>((v2.x - lo) >> shift) & (kBins - 1) : 0;
                    for (int b = 0; b < kBins; ++b) {
                        const uint64_t m = __ballot(in && digit == b);
                        const int start = __builtin_amdgcn_readlane(mine, b);
                        if (in && digit == b) buffer[from ^ 1][start + __popcll(m & ((1ull << lane) - 1))] = v2;
                        mine += lane == b ? __popcll(m) : 0;
                    }
                }
                __syncthreads();
            }
            for (int p = threadIdx.x; p < inside; p += kSortThreads) {
                const int2 v2 = buffer[from][p];
                a.s.token[under + p] = v2.y;
                a.s.id[under + p] = v2.x;
            }
            if (a.clear) {
                // rows between the ids that are there
                int64_t next = lo;
                for (int p = 0; p < inside; ++p) {
                    const int64_t id = buffer[from][p].x;
                    clear_rows<G>(a, next, id);
                    next = id + 1;
                }
                clear_rows<G>(a, next, hi);
            }
            __syncthreads();
        }
        lo = hi;
        hi = end;
    }
}

// ---- the sums -----------------------------------------------------------------------

template <typename T>
__device__ __forceinline__ void add_row(const T* dY, int64_t ldy, int token, int e, int d, float (&s)[8]) {
    float x[8];
    load8(dY + token * ldy, e, d, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] += x[i];
}

template <typename G>
__device__ __forceinline__ void put_row(const EmbeddingGradArgs& a, int id, int64_t e, const float (&s)[8]) {
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
    store8(row + e, a.d - e, y);
}

// Whether the run of one id that goes on past `end`, a chunk's end, ends within the chunk
// after it (and is then the first one's to sum)
__device__ __forceinline__ bool ends_in_next(const Sorted& s, int64_t end, int64_t n, int id) {
    return end + kChunk >= n || s.id[end + kChunk] != id;
}

template <typename T, typename G>
__global__ __launch_bounds__(256) void sum_kernel(EmbeddingGradArgs a, Sorted s) {
    const int64_t e = 8 * (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x);
    if (e >= a.d) return;
    const int d = static_cast<int>(a.d);
    const int64_t n = *s.count, chunks = (n + kChunk - 1) / kChunk;
    const T* dY = static_cast<const T*>(a.dY);
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int64_t p = c * kChunk;
        const int64_t end = min(p + kChunk, n);
        if (c > 0 && s.id[p - 1] == s.id[p]) {
            // the run that the chunk begins with began before it
            const int id = s.id[p];
            const bool began = c == 1 || s.id[p - kChunk - 1] != id;     // in the chunk before
            const bool owned = began && ends_in_next(s, p, n, id);
            float sum[8] = {};
            for (; p < end && s.id[p] == id; ++p)
                if (!owned) add_row(dY, a.lddy, s.token[p], static_cast<int>(e), d, sum);
            if (!owned) store8(s.part + (2 * c) * a.d + e, a.d - e, sum);
        }
        while (p < end) {
            const int id = s.id[p];
            float sum[8] = {};
            for (; p < end && s.id[p] == id; ++p) add_row(dY, a.lddy, s.token[p], static_cast<int>(e), d, sum);
            if (p == end && end < n && s.id[end] == id) {
                if (!ends_in_next(s, end, n, id)) {
                    store8(s.part + (2 * c + 1) * a.d + e, a.d - e, sum);
                    break;
                }
                for (int64_t q = end; q < n && s.id[q] == id; ++q) add_row(dY, a.lddy, s.token[q], static_cast<int>(e), d, sum);
            }
            put_row<G>(a, id, e, sum);
        }
    }
}

template <typename G>
__global__ __launch_bounds__(256) void join_kernel(EmbeddingGradArgs a, Sorted s) {
    const int64_t e = 8 * (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x);
    if (e >= a.d) return;
    const int d = static_cast<int>(a.d);
    const int64_t n = *s.count, chunks = (n + kChunk - 1) / kChunk;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int64_t end = (c + 1) * kChunk;
        if (end >= n) continue;
        const int id = s.id[end - 1];
        if (s.id[end] != id || ends_in_next(s, end, n, id)) continue;
        if (c > 0 && s.id[c * kChunk - 1] == id) continue;          // began before this chunk
        float sum[8], x[8];
        load8(s.part + (2 * c + 1) * a.d, static_cast<int>(e), d, sum);
        for (int64_t k = c + 1; k < chunks && s.id[k * kChunk] == id; ++k) {
            load8(s.part + 2 * k * a.d, static_cast<int>(e), d, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += x[i];
        }
        put_row<G>(a, id, e, sum);
    }
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }
size_t chunk_count(int64_t tokens) { return static_cast<size_t>((tokens + kChunk - 1) / kChunk); }

template <typename T, typename G>
hipError_t embedding_grad(const EmbeddingGradArgs& a, hipStream_t stream) {
    char* w = static_cast<char*>(a.workspace);
    const size_t list = round_up(sizeof(int) * static_cast<size_t>(a.tokens));
    Sorted s{reinterpret_cast<int*>(w + 256), reinterpret_cast<int*>(w + 256 + list), reinterpret_cast<int*>(w),
             reinterpret_cast<float*>(w + 256 + 2 * list)};
    const SortArgs sort{a.ids, a.tokens, a.vocab, s, a.G, a.d, a.ldg, !a.accumulate};
    const unsigned ranges = static_cast<unsigned>(std::min<int64_t>(a.vocab, 256));
    hipLaunchKernelGGL(sort_kernel<G>, dim3(ranges), dim3(kSortThreads), 0, stream, sort);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.tokens == 0) return e;
    const int64_t groups = (a.d + 7) / 8;
    const unsigned wide = static_cast<unsigned>(std::min<int64_t>((groups + 63) / 64 * 64, 256));
    const unsigned chunks = static_cast<unsigned>(std::min<size_t>(chunk_count(a.tokens), 1 << 16));
    const dim3 grid(chunks, static_cast<unsigned>((groups + wide - 1) / wide));
    hipLaunchKernelGGL((sum_kernel<T, G>), grid, dim3(wide), 0, stream, a, s);
    e = hipGetLastError();
    if (e != hipSuccess || a.tokens <= 2 * kChunk) return e;
    hipLaunchKernelGGL(join_kernel<G>, grid, dim3(wide), 0, stream, a, s);
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

size_t embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t d) {
    (void)vocab;
    return 256 + 2 * round_up(sizeof(int) * static_cast<size_t>(tokens)) +
           round_up(sizeof(float) * 2 * chunk_count(tokens) * static_cast<size_t>(d));
}

hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, bool dy_bf16, bool g_bf16, hipStream_t stream) {
    if (dy_bf16) return g_bf16 ? embedding_grad<bf16_t, bf16_t>(a, stream) : embedding_grad<bf16_t, float>(a, stream);
    return g_bf16 ? embedding_grad<float, bf16_t>(a, stream) : embedding_grad<float, float>(a, stream);
}

}  // namespace galore
