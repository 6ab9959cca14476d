// Host side of the operators between linear layers: argument validation and launches.
// As in the rest of the library everything is enqueued on the caller's stream, nothing
// allocates device memory and nothing synchronises.
#include "host_checks.hpp"
#include "layers.hpp"

using namespace galore;

namespace {

// In elements (of checkpoints, bytes): a pitch or stride, and from a matrix's first row to
// its last. With 2^16 matrices or heads, 4 bytes each, every offset stays within 2^60.
constexpr int64_t kMaxPitch = int64_t{1} << 40, kMaxSpan = int64_t{1} << 56;

constexpr int64_t kMaxWidth = int64_t{1} << 24;   // columns of the embedding and of dropout: a grid's second dimension

bool index_ok(int32_t bytes) { return bytes == 4 || bytes == 8; }
bool pitch_ok(int64_t ld, int64_t rows) { return ld <= kMaxPitch && (rows <= 1 || ld <= kMaxSpan / (rows - 1)); }
bool stride_ok(int64_t stride, int32_t batch) { return batch == 1 || stride <= kMaxPitch; }
bool elements_ok(const void* p, int32_t dtype) { return is_aligned(p, dtype == GALORE_BF16 ? 2 : 4); }

// tokens x heads rows of d values that do not share memory
int check_heads(const galore_heads_t* h, int32_t heads, int64_t tokens, int64_t d, int32_t dtype) {
    if (h == nullptr || (h->data == nullptr && tokens > 0) || !elements_ok(h->data, dtype)) return GALORE_ERR_INVALID_ARG;
    const int64_t t = h->token_stride, s = h->head_stride;
    if (t < 0 || s < 0 || !pitch_ok(t, tokens) || !pitch_ok(s, heads)) return GALORE_ERR_SHAPE;
    const bool by_token = (heads == 1 || s >= d) && (tokens <= 1 || t >= (heads - 1) * s + d);
    const bool by_head = (tokens <= 1 || t >= d) && (heads == 1 || s >= (tokens - 1) * t + d);
    return by_token || by_head ? GALORE_OK : GALORE_ERR_SHAPE;
}
Heads heads_of(const galore_heads_t* h, int32_t heads) { return {h->data, h->token_stride, h->head_stride, heads}; }

int check_rotation(const float* w_q, const float* w_k, const float* table, int64_t table_rows, int64_t ld_table, int64_t rot,
                   const void* positions, int32_t position_bytes, float eps, int64_t tokens, int32_t q_heads, int32_t k_heads,
                   int64_t d, int32_t dtype) {
    if (w_q == nullptr || w_k == nullptr || !dtype_ok(dtype)) return GALORE_ERR_INVALID_ARG;
    if (!is_aligned(w_q, 4) || !is_aligned(w_k, 4) || !is_aligned(table, 4)) return GALORE_ERR_INVALID_ARG;
    if (table == nullptr && rot > 0 && table_rows > 0) return GALORE_ERR_INVALID_ARG;
    if (positions != nullptr && (!index_ok(position_bytes) || !is_aligned(positions, position_bytes)))
        return GALORE_ERR_INVALID_ARG;
    if (!finite_f(eps) || eps <= 0.0f) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, 1) || d > kHeadMaxWidth) return GALORE_ERR_SHAPE;
    if (q_heads < 1 || k_heads < 1 || q_heads > kMaxHeads || k_heads > kMaxHeads) return GALORE_ERR_SHAPE;
    if (rot < 0 || rot % 2 != 0 || rot > d || table_rows < 0 || table_rows > kMaxSide || ld_table < rot || !pitch_ok(ld_table, table_rows))
        return GALORE_ERR_SHAPE;
    return GALORE_OK;
}

HeadNormArgs rotation_args(const float* w_q, const float* w_k, const float* table, int64_t table_rows, int64_t ld_table,
                           int64_t rot, const void* positions, int32_t position_bytes, int32_t interleaved, float eps,
                           int64_t tokens, int64_t d) {
    HeadNormArgs a{};
    a.w[0] = w_q;
    a.w[1] = w_k;
    a.table = table;
    a.table_rows = table_rows;
    a.ld_table = ld_table;
    a.rot = static_cast<int>(rot);
    a.positions = {positions, position_bytes == 8};
    a.interleaved = interleaved != 0;
    a.eps = eps;
    a.tokens = tokens;
    a.d = static_cast<int>(d);
    return a;
}

// a matrix of activations (tokens x d, `batch` of them)
int check_rows(const void* p, int32_t dtype, int64_t tokens, int64_t d, int64_t ld, int64_t stride, int32_t batch) {
    if ((p == nullptr && tokens > 0) || !elements_ok(p, dtype)) return GALORE_ERR_INVALID_ARG;
    if (!pitch_ok(ld, tokens) || !stride_ok(stride, batch)) return GALORE_ERR_SHAPE;
    return matrix_ok(tokens, d, ld, stride, batch) ? GALORE_OK : GALORE_ERR_SHAPE;
}

// its 8-bit checkpoint
int check_codes(const galore_mx_t* q, int64_t tokens, int64_t d, int32_t batch) {
    const int e = check_mx(q, tokens, d, kBytes8, batch);
    if (e != GALORE_OK) return e;
    const bool ok = pitch_ok(q->ldq, tokens) && pitch_ok(q->lds, tokens) && stride_ok(q->stride_q, batch) &&
                    stride_ok(q->stride_s, batch);
    return ok ? GALORE_OK : GALORE_ERR_SHAPE;
}

int check_sequences(const void* offsets, int32_t offset_bytes, int64_t sequences, int64_t tokens, int64_t d, int32_t dtype,
                    int32_t batch) {
    if (!dtype_ok(dtype)) return GALORE_ERR_INVALID_ARG;
    if (offsets != nullptr && (!index_ok(offset_bytes) || !is_aligned(offsets, offset_bytes))) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, batch)) return GALORE_ERR_SHAPE;
    if (offsets != nullptr && (batch != 1 || sequences < 1 || sequences > kMaxSide)) return GALORE_ERR_SHAPE;
    return GALORE_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need > 0 && (workspace == nullptr || !is_aligned(workspace, kAlign) || bytes < need)) return GALORE_ERR_WORKSPACE;
    return GALORE_OK;
}

}  // namespace

extern "C" {

// ---- embedding ----------------------------------------------------------------

int galore_embedding(const void* ids, int32_t id_bytes, int64_t tokens, const void* W, int32_t w_dtype, int64_t vocab,
                     int64_t d, int64_t ldw, float scale, void* out, int32_t out_dtype, int64_t ldo, hipStream_t stream) {
    if ((ids == nullptr && tokens > 0) || !index_ok(id_bytes) || !is_aligned(ids, id_bytes)) return GALORE_ERR_INVALID_ARG;
    if (W == nullptr || !dtype_ok(w_dtype) || !dtype_ok(out_dtype) || !finite_f(scale)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, 1) || d > kMaxWidth || vocab < 1 || vocab > kMaxSide) return GALORE_ERR_SHAPE;
    int e = check_rows(W, w_dtype, vocab, d, ldw, 0, 1);
    if (e == GALORE_OK) e = check_rows(out, out_dtype, tokens, d, ldo, 0, 1);
    if (e != GALORE_OK) return e;
    const LookupArgs a{{ids, id_bytes == 8}, W, out, tokens, vocab, d, ldw, ldo, scale};
    GALORE_TRY(launch_lookup(a, w_dtype == GALORE_BF16, out_dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

size_t galore_embedding_grad_workspace_size(int64_t tokens, int64_t vocab, int64_t d) {
    if (!sides_ok(tokens, d, 1) || d > kMaxWidth || vocab < 1 || vocab > kMaxSide) return 0;
    return align_up(embedding_grad_bytes(tokens, vocab, d));
}

int galore_embedding_grad(const void* ids, int32_t id_bytes, int64_t tokens, const void* dY, int32_t dy_dtype, int64_t lddy,
                          int64_t vocab, int64_t d, float scale, void* G, int32_t g_dtype, int64_t ldg, int32_t accumulate,
                          void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if ((ids == nullptr && tokens > 0) || !index_ok(id_bytes) || !is_aligned(ids, id_bytes)) return GALORE_ERR_INVALID_ARG;
    if (G == nullptr || !dtype_ok(dy_dtype) || !dtype_ok(g_dtype) || !finite_f(scale)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, d, 1) || d > kMaxWidth || vocab < 1 || vocab > kMaxSide) return GALORE_ERR_SHAPE;
    int e = check_rows(dY, dy_dtype, tokens, d, lddy, 0, 1);
    if (e == GALORE_OK) e = check_rows(G, g_dtype, vocab, d, ldg, 0, 1);
    if (e == GALORE_OK)
        e = check_workspace(workspace, workspace_bytes, galore_embedding_grad_workspace_size(tokens, vocab, d));
    if (e != GALORE_OK) return e;
    const EmbeddingGradArgs a{{ids, id_bytes == 8}, dY, G, tokens, vocab, d, lddy, ldg, scale, accumulate != 0, workspace};
    GALORE_TRY(launch_embedding_grad(a, dy_dtype == GALORE_BF16, g_dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

// ---- dropout --------------------------------------------------------------------

int galore_dropout(const void* X, int64_t ldx, int64_t stride_x, int32_t dtype, const void* R, int64_t ldr, int64_t stride_r,
                   int64_t tokens, int64_t cols, float p, uint64_t seed, uint32_t index, void* Y, int64_t ldy,
                   int64_t stride_y, const galore_mx_t* y8, int32_t batch, hipStream_t stream) {
    if (!dtype_ok(dtype) || !(p >= 0.0f && p <= 1.0f)) return GALORE_ERR_INVALID_ARG;
    if (!sides_ok(tokens, cols, batch) || cols > kMaxWidth) return GALORE_ERR_SHAPE;
    int e = check_rows(X, dtype, tokens, cols, ldx, stride_x, batch);
    if (e == GALORE_OK && R != nullptr) e = check_rows(R, dtype, tokens, cols, ldr, stride_r, batch);
    if (e == GALORE_OK) e = check_rows(Y, dtype, tokens, cols, ldy, stride_y, batch);
    if (e == GALORE_OK && y8 != nullptr) e = check_codes(y8, tokens, cols, batch);
    if (e != GALORE_OK) return e;
    DropoutArgs a{};
    a.X = X;
    a.R = R;
    a.Y = Y;
    a.ldx = ldx;
    a.strideX = batch > 1 ? stride_x : 0;
    a.ldr = ldr;
    a.strideR = batch > 1 ? stride_r : 0;
    a.ldy = ldy;
    a.strideY = batch > 1 ? stride_y : 0;
    if (y8 != nullptr) a.y8 = matrix_of(y8, batch);
    a.rows = tokens;
    a.cols = cols;
    a.cut = static_cast<uint32_t>(lrint(65536.0 * static_cast<double>(p)));
    a.scale = a.cut < 65536 ? static_cast<float>(65536.0 / (65536.0 - a.cut)) : 0.0f;
    a.key0 = static_cast<uint32_t>(seed);
    a.key1 = static_cast<uint32_t>(seed >> 32);
    a.index = index;
    GALORE_TRY(launch_dropout(a, dtype == GALORE_BF16, batch, stream));
    return GALORE_OK;
}

// ---- norms of heads with their rotation -------------------------------------------

int galore_head_norm(const galore_heads_t* Q, int32_t q_heads, const galore_heads_t* K, int32_t k_heads, int32_t dtype,
                     int64_t tokens, int64_t d, const float* w_q, const float* w_k, const float* table, int64_t table_rows,
                     int64_t ld_table, int64_t rot, const void* positions, int32_t position_bytes, int32_t interleaved,
                     float eps, const galore_heads_t* Q_out, const galore_heads_t* K_out, hipStream_t stream) {
    int e = check_rotation(w_q, w_k, table, table_rows, ld_table, rot, positions, position_bytes, eps, tokens, q_heads, k_heads,
                           d, dtype);
    if (e == GALORE_OK) e = check_heads(Q, q_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(K, k_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(Q_out, q_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(K_out, k_heads, tokens, d, dtype);
    if (e != GALORE_OK) return e;
    HeadNormArgs a = rotation_args(w_q, w_k, table, table_rows, ld_table, rot, positions, position_bytes, interleaved, eps,
                                   tokens, d);
    a.in[0] = heads_of(Q, q_heads);
    a.in[1] = heads_of(K, k_heads);
    a.out[0] = heads_of(Q_out, q_heads);
    a.out[1] = heads_of(K_out, k_heads);
    GALORE_TRY(launch_head_norm(a, dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

size_t galore_head_norm_backward_workspace_size(int64_t tokens, int32_t q_heads, int32_t k_heads, int64_t d) {
    if (!sides_ok(tokens, d, 1) || d > kHeadMaxWidth || q_heads < 1 || k_heads < 1 || q_heads > kMaxHeads ||
        k_heads > kMaxHeads)
        return 0;
    return align_up(sizeof(float) * 2 * static_cast<size_t>(d) * head_norm_groups(tokens));
}

int galore_head_norm_backward(const galore_heads_t* dQ, int32_t q_heads, const galore_heads_t* dK, int32_t k_heads,
                              int32_t dtype, int64_t tokens, int64_t d, const galore_heads_t* Q, const galore_heads_t* K,
                              const galore_mx_t* q8, const galore_mx_t* k8, const float* w_q, const float* w_k,
                              const float* table, int64_t table_rows, int64_t ld_table, int64_t rot, const void* positions,
                              int32_t position_bytes, int32_t interleaved, float eps, const galore_heads_t* dQ_in,
                              const galore_heads_t* dK_in, float* dw_q, float* dw_k, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
    const bool packed = q8 != nullptr;
    if (packed != (k8 != nullptr) || packed == (Q != nullptr) || packed == (K != nullptr)) return GALORE_ERR_INVALID_ARG;
    if (dw_q == nullptr || dw_k == nullptr || !is_aligned(dw_q, 4) || !is_aligned(dw_k, 4)) return GALORE_ERR_INVALID_ARG;
    int e = check_rotation(w_q, w_k, table, table_rows, ld_table, rot, positions, position_bytes, eps, tokens, q_heads, k_heads,
                           d, dtype);
    if (e == GALORE_OK) e = check_heads(dQ, q_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(dK, k_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = packed ? check_codes(q8, tokens, q_heads * d, 1) : check_heads(Q, q_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = packed ? check_codes(k8, tokens, k_heads * d, 1) : check_heads(K, k_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(dQ_in, q_heads, tokens, d, dtype);
    if (e == GALORE_OK) e = check_heads(dK_in, k_heads, tokens, d, dtype);
    if (e == GALORE_OK)
        e = check_workspace(workspace, workspace_bytes, galore_head_norm_backward_workspace_size(tokens, q_heads, k_heads, d));
    if (e != GALORE_OK) return e;
    HeadNormArgs a = rotation_args(w_q, w_k, table, table_rows, ld_table, rot, positions, position_bytes, interleaved, eps,
                                   tokens, d);
    a.in[0] = heads_of(dQ, q_heads);
    a.in[1] = heads_of(dK, k_heads);
    if (packed) {
        a.codes[0] = matrix_of(q8, 1);
        a.codes[1] = matrix_of(k8, 1);
    } else {
        a.saved[0] = heads_of(Q, q_heads);
        a.saved[1] = heads_of(K, k_heads);
    }
    a.out[0] = heads_of(dQ_in, q_heads);
    a.out[1] = heads_of(dK_in, k_heads);
    a.dw[0] = dw_q;
    a.dw[1] = dw_k;
    a.part = static_cast<float*>(workspace);
    GALORE_TRY(launch_head_norm_backward(a, dtype == GALORE_BF16, stream));
    return GALORE_OK;
}

// ---- gated linear recurrence ---------------------------------------------------------

int64_t galore_recurrence_states(int64_t tokens) {
    return tokens < 0 || tokens > kMaxSide ? 0 : (tokens + kScanStep - 1) / kScanStep;
}

size_t galore_recurrence_workspace_size(int64_t tokens, int64_t d, int32_t batch) {
    if (!sides_ok(tokens, d, batch)) return 0;
    return align_up(scan_bytes(tokens, d, batch));
}

int galore_recurrence(const void* X, int64_t ldx, int64_t stride_x, const void* F, int64_t ldf, int64_t stride_f,
                      int32_t dtype, int64_t tokens, int64_t d, const float* h0, const void* offsets, int32_t offset_bytes,
                      int64_t sequences, void* H, int64_t ldh, int64_t stride_h, float* last, float* states, int32_t batch,
                      void* workspace, size_t workspace_bytes, hipStream_t stream) {
    int e = check_sequences(offsets, offset_bytes, sequences, tokens, d, dtype, batch);
    if (e == GALORE_OK) e = check_rows(X, dtype, tokens, d, ldx, stride_x, batch);
    if (e == GALORE_OK) e = check_rows(F, dtype, tokens, d, ldf, stride_f, batch);
    if (e == GALORE_OK) e = check_rows(H, dtype, tokens, d, ldh, stride_h, batch);
    if (e == GALORE_OK && (last == nullptr || (offsets != nullptr && last == h0) || !is_aligned(last, 4) || !is_aligned(h0, 4) || !is_aligned(states, 4)))
        e = GALORE_ERR_INVALID_ARG;
    if (e == GALORE_OK) e = check_workspace(workspace, workspace_bytes, galore_recurrence_workspace_size(tokens, d, batch));
    if (e != GALORE_OK) return e;
    ScanArgs a{};
    a.X = X;
    a.ldx = ldx;
    a.strideX = batch > 1 ? stride_x : 0;
    a.F = F;
    a.ldf = ldf;
    a.strideF = batch > 1 ? stride_f : 0;
    a.H = H;
    a.ldh = ldh;
    a.strideH = batch > 1 ? stride_h : 0;
    a.h0 = h0;
    a.last = last;
    a.states = states;
    a.offsets = {offsets, offset_bytes == 8};
    a.sequences = sequences;
    a.T = tokens;
    a.d = d;
    a.workspace = workspace;
    GALORE_TRY(launch_scan(a, dtype == GALORE_BF16, batch, stream));
    return GALORE_OK;
}

int galore_recurrence_backward(const void* dH, int64_t lddh, int64_t stride_dh, const void* X, int64_t ldx, int64_t stride_x,
                               const void* F, int64_t ldf, int64_t stride_f, int32_t dtype, int64_t tokens, int64_t d,
                               const float* states, const float* h0, const float* dlast, const void* offsets,
                               int32_t offset_bytes, int64_t sequences, void* dX, int64_t lddx, int64_t stride_dx, void* dF,
                               int64_t lddf, int64_t stride_df, float* dh0, int32_t batch, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
    int e = check_sequences(offsets, offset_bytes, sequences, tokens, d, dtype, batch);
    if (e == GALORE_OK) e = check_rows(dH, dtype, tokens, d, lddh, stride_dh, batch);
    if (e == GALORE_OK) e = check_rows(X, dtype, tokens, d, ldx, stride_x, batch);
    if (e == GALORE_OK) e = check_rows(F, dtype, tokens, d, ldf, stride_f, batch);
    if (e == GALORE_OK) e = check_rows(dX, dtype, tokens, d, lddx, stride_dx, batch);
    if (e == GALORE_OK) e = check_rows(dF, dtype, tokens, d, lddf, stride_df, batch);
    if (e == GALORE_OK && (dh0 == nullptr || dh0 == dlast || (states == nullptr && tokens > 0) || !is_aligned(dh0, 4) || !is_aligned(h0, 4) ||
                           !is_aligned(dlast, 4) || !is_aligned(states, 4)))
        e = GALORE_ERR_INVALID_ARG;
    if (e == GALORE_OK) e = check_workspace(workspace, workspace_bytes, galore_recurrence_workspace_size(tokens, d, batch));
    if (e != GALORE_OK) return e;
    ScanArgs a{};
    a.dH = dH;
    a.lddh = lddh;
    a.strideDH = batch > 1 ? stride_dh : 0;
    a.X = X;
    a.ldx = ldx;
    a.strideX = batch > 1 ? stride_x : 0;
    a.F = F;
    a.ldf = ldf;
    a.strideF = batch > 1 ? stride_f : 0;
    a.dX = dX;
    a.lddx = lddx;
    a.strideDX = batch > 1 ? stride_dx : 0;
    a.dF = dF;
    a.lddf = lddf;
    a.strideDF = batch > 1 ? stride_df : 0;
    a.states = const_cast<float*>(states);
    a.h0 = h0;
    a.dlast = dlast;
    a.dh0 = dh0;
    a.offsets = {offsets, offset_bytes == 8};
    a.sequences = sequences;
    a.T = tokens;
    a.d = d;
    a.workspace = workspace;
    GALORE_TRY(launch_scan_backward(a, dtype == GALORE_BF16, batch, stream));
    return GALORE_OK;
}

}  // extern "C"
