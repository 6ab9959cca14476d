// Launchers of the operators between linear layers (embedding, dropout, head norms
// with rotation, gated recurrence). All return the hipError_t of the launch;
// arguments are checked by the entry points (layers.hip).
#pragma once

#include "mx.hpp"

namespace galore {

// token ids, positions and bounds: 32 or 64 bits each
struct Indices {
    const void* p;
    bool wide;
    __device__ __forceinline__ int64_t at(int64_t i) const {
        return wide ? static_cast<const int64_t*>(p)[i] : static_cast<const int32_t*>(p)[i];
    }
};

// dropout.hip
struct DropoutArgs {
    const void *X, *R;           // R may be null
    void* Y;
    int64_t ldx, strideX, ldr, strideR, ldy, strideY;
    MxMatrix y8;                 // codes null: not written
    int64_t rows, cols;
    uint32_t cut;                // dropped where the 16 random bits are under it
    float scale;                 // 65536 / (65536 - cut), 0 where cut = 65536
    uint32_t key0, key1, index;
};
hipError_t launch_dropout(const DropoutArgs& a, bool bf16, int batch, hipStream_t stream);

// embedding.hip
struct LookupArgs {
    Indices ids;
    const void* W;
    void* out;
    int64_t tokens, vocab, d, ldw, ldo;
    float scale;
};
hipError_t launch_lookup(const LookupArgs& a, bool w_bf16, bool out_bf16, hipStream_t stream);

struct EmbeddingGradArgs {
    Indices ids;
    const void* dY;
    void* G;
    int64_t tokens, vocab, d, lddy, ldg;
    float scale;
    bool accumulate;
    void* workspace;             // embedding_grad_bytes(...)
};
size_t embedding_grad_bytes(int64_t tokens, int64_t vocab, int64_t d);
hipError_t launch_embedding_grad(const EmbeddingGradArgs& a, bool dy_bf16, bool g_bf16, hipStream_t stream);

// head_norm.hip
struct Heads {
    void* p;
    int64_t token, head;         // strides in elements
    int n;
};
struct HeadNormArgs {
    Heads in[2], out[2];         // queries, keys; backward: of the incoming gradients, of their gradients
    Heads saved[2];              // backward: the forward pass's inputs, or null with
    MxMatrix codes[2];           // their checkpoints
    const float* w[2];
    float* dw[2];
    float* part;                 // backward: head_norm_groups(tokens) x 2 x d
    const float* table;
    int64_t table_rows, ld_table;
    Indices positions;           // null: a token's own number
    int64_t tokens;
    int d, rot;
    bool interleaved;
    float eps;
};
constexpr int64_t kHeadMaxWidth = 1024;
constexpr int64_t kMaxHeads = 65535;
int64_t head_norm_groups(int64_t tokens);
hipError_t launch_head_norm(const HeadNormArgs& a, bool bf16, hipStream_t stream);
hipError_t launch_head_norm_backward(const HeadNormArgs& a, bool bf16, hipStream_t stream);

// recurrence.hip
constexpr int kScanStep = 64;    // tokens from one kept state to the next
struct ScanArgs {
    const void *X, *F, *dH;      // dH: backward only
    int64_t ldx, strideX, ldf, strideF, lddh, strideDH;
    void *H, *dX, *dF;           // H forward; dX, dF backward
    int64_t ldh, strideH, lddx, strideDX, lddf, strideDF;
    const float *h0, *dlast;     // sequences x d, may be null: zeros
    float *last, *dh0;           // sequences x d
    float* states;               // batch x ceil(T / kScanStep) x d; written forward (unless null), read backward
    Indices offsets;             // null: every matrix of the batch is a sequence
    int64_t sequences, T, d;
    void* workspace;             // scan_bytes(...)
};
size_t scan_bytes(int64_t T, int64_t d, int64_t batch);
hipError_t launch_scan(const ScanArgs& a, bool bf16, int batch, hipStream_t stream);
hipError_t launch_scan_backward(const ScanArgs& a, bool bf16, int batch, hipStream_t stream);

}  // namespace galore
