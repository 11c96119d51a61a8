// Host-side validation for libbsr's C ABI: pure C++ with no HIP dependency.
//
// Every check here runs before anything is enqueued, so a rejected call launches nothing and
// leaves its outputs untouched.
#include <cmath>
#include <cstdint>
#include <cstring>

#include "bsr_internal.h"

namespace {

constexpr int64_t kMaxBlocks = (int64_t(1) << 31) - 1;   // block ids and indptr are int32
constexpr int64_t kMaxElems = int64_t(1) << 53;          // element offsets stay exact

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

bool tiles(int64_t N, int64_t K, int32_t R, int32_t C) {
    return N > 0 && K > 0 && R > 0 && C > 0 && N % R == 0 && K % C == 0;
}

}  // namespace

namespace bsr {

PruneWorkspace prune_workspace_layout(int64_t nb) {
    PruneWorkspace w{};
    w.key_offset = 0;
    w.key_bytes = size_t(nb) * sizeof(uint64_t);
    w.src_offset = align256(w.key_bytes);
    w.src_bytes = size_t(nb) * sizeof(int32_t);
    w.total = align256(w.src_offset + w.src_bytes);
    return w;
}

bsr_status check_prune(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t R, int32_t C,
                       int64_t k, const int32_t *indptr, const int32_t *indices,
                       const float *data, int64_t capacity_blocks, const void *workspace,
                       size_t ws_bytes) {
    if (!W || !indptr) return BSR_ERR_NULL;
    if (!tiles(N, K, R, C) || ldw < K) return BSR_ERR_SHAPE;
    const int64_t Nb = N / R, Kb = K / C;
    if (Nb > kMaxBlocks / Kb) return BSR_ERR_UNSUPPORTED;
    const int64_t nb = Nb * Kb;
    if (N > kMaxElems / ldw) return BSR_ERR_UNSUPPORTED;
    if (k < 0 || k > nb) return BSR_ERR_ARG;
    if (k > 0 && (!indices || !data)) return BSR_ERR_NULL;
    if (capacity_blocks < k) return BSR_ERR_CAPACITY;
    if (!workspace || ws_bytes < prune_workspace_layout(nb).total) return BSR_ERR_WORKSPACE;
    return BSR_OK;
}

bsr_status check_prune_noalloc(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t R,
                               int32_t C, int64_t k, const int32_t *indptr,
                               const int32_t *indices, const float *data,
                               int64_t capacity_blocks) {
    // The same checks as check_prune, with the library's fixed scratch array standing in for
    // the workspace: a matrix with more blocks than it holds is BSR_ERR_WORKSPACE.
    if (tiles(N, K, R, C)) {
        const int64_t Nb = N / R, Kb = K / C;
        if (Nb <= kMaxBlocks / Kb && Nb * Kb > BSR_NOALLOC_MAX_BLOCKS) {
            const bsr_status s = check_prune(W, N, K, ldw, R, C, k, indptr, indices, data,
                                             capacity_blocks, &kMaxBlocks, 0);
            return s == BSR_OK ? BSR_ERR_WORKSPACE : s;
        }
    }
    return check_prune(W, N, K, ldw, R, C, k, indptr, indices, data, capacity_blocks,
                       &kMaxBlocks, kNoallocScratchBytes);
}

bsr_status check_prune_options(const bsr_prune_options_t *opts, int64_t N, int32_t R,
                               int64_t k) {
    if (!opts) return BSR_OK;
    if (opts->norm != BSR_NORM_L2 && opts->norm != BSR_NORM_L1) return BSR_ERR_ARG;
    if (opts->select != BSR_SELECT_GLOBAL && opts->select != BSR_SELECT_PER_ROW)
        return BSR_ERR_ARG;
    if (opts->select == BSR_SELECT_PER_ROW && k % (N / R) != 0) return BSR_ERR_ARG;
    return BSR_OK;
}

bsr_status check_matrix(const bsr_matrix_t *W) {
    if (!W) return BSR_ERR_NULL;
    const int32_t dt = raw_enum(W->dtype);
    if (dt != BSR_F32 && dt != BSR_BF16) return BSR_ERR_ARG;
    if (!tiles(W->n_rows, W->n_cols, W->R, W->C)) return BSR_ERR_SHAPE;
    const int64_t Nb = W->n_rows / W->R, Kb = W->n_cols / W->C;
    if (Nb > kMaxBlocks / Kb) return BSR_ERR_UNSUPPORTED;
    if (W->nnzb < 0 || W->nnzb > Nb * Kb) return BSR_ERR_ARG;
    if (int64_t(W->R) * W->C > kMaxElems / (W->nnzb > 0 ? W->nnzb : 1))
        return BSR_ERR_UNSUPPORTED;
    if (!W->indptr) return BSR_ERR_NULL;
    if (W->nnzb > 0 && (!W->indices || !W->data)) return BSR_ERR_NULL;
    return BSR_OK;
}

namespace {

// Whether the byte ranges [a, a + na) and [b, b + nb) intersect (empty ranges never do).
bool overlaps(const void *a, int64_t na, const void *b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + uint64_t(nb) && pb < pa + uint64_t(na);
}

// Bytes spanned by the arrays of a valid matrix.
int64_t indptr_bytes(const bsr_matrix_t *W) { return (W->n_rows / W->R + 1) * 4; }
int64_t data_bytes(const bsr_matrix_t *W) {
    return W->nnzb * W->R * W->C * (W->dtype == BSR_BF16 ? 2 : 4);
}

}  // namespace

bsr_status check_spmm(const void *X, int x_dtype, int64_t T, int64_t ldx, const bsr_matrix_t *W,
                      const float *Y, int64_t ldy, const float *bias) {
    if (!W) return BSR_ERR_NULL;
    bsr_status s = check_matrix(W);
    if (s != BSR_OK) return s;
    if (x_dtype != BSR_F32 && x_dtype != BSR_BF16) return BSR_ERR_ARG;
    if (x_dtype != int(W->dtype)) return BSR_ERR_DTYPE;
    if (T < 0 || ldx < W->n_cols || ldy < W->n_rows) return BSR_ERR_SHAPE;
    if (T > 0 && (!X || !Y)) return BSR_ERR_NULL;
    if (T > kMaxElems / ldx || T > kMaxElems / ldy) return BSR_ERR_UNSUPPORTED;
    if (T > 0) {
        // Y must not overlap the product's inputs.
        const int64_t yb = ((T - 1) * ldy + W->n_rows) * 4;
        const int64_t xb = ((T - 1) * ldx + W->n_cols) * (x_dtype == BSR_BF16 ? 2 : 4);
        if (overlaps(Y, yb, X, xb) || overlaps(Y, yb, bias, W->n_rows * 4) ||
            overlaps(Y, yb, W->indptr, indptr_bytes(W)) ||
            overlaps(Y, yb, W->indices, W->nnzb * 4) || overlaps(Y, yb, W->data, data_bytes(W)))
            return BSR_ERR_ARG;
    }
    return BSR_OK;
}

bsr_status check_spmm_items(const bsr_spmm_item_t *items, int32_t n) {
    // Products of one call may run concurrently: each Y must be disjoint from every other
    // product's inputs and output (inputs may be shared).  Items are already checked one by
    // one, so every descriptor is valid here.
    auto y_bytes = [](const bsr_spmm_item_t &it) { return ((it.T - 1) * it.ldy + it.W->n_rows) * 4; };
    for (int32_t i = 0; i < n; ++i) {
        const bsr_spmm_item_t &a = items[i];
        if (a.T <= 0) continue;
        const int64_t yb = y_bytes(a);
        for (int32_t j = 0; j < n; ++j) {
            const bsr_spmm_item_t &b = items[j];
            if (j == i || b.T <= 0) continue;
            const bsr_matrix_t *W = b.W;
            const int64_t xb = ((b.T - 1) * b.ldx + W->n_cols) * (b.x_dtype == BSR_BF16 ? 2 : 4);
            if (overlaps(a.Y, yb, b.X, xb) || overlaps(a.Y, yb, b.bias, W->n_rows * 4) ||
                overlaps(a.Y, yb, W->indptr, indptr_bytes(W)) ||
                overlaps(a.Y, yb, W->indices, W->nnzb * 4) ||
                overlaps(a.Y, yb, W->data, data_bytes(W)) || overlaps(a.Y, yb, b.Y, y_bytes(b)))
                return BSR_ERR_ARG;
        }
    }
    return BSR_OK;
}

bsr_status check_plan_use(const bsr_spmm_item_t &it, const bsr_plan_t *plan,
                          int64_t layout_bytes) {
    // The plan must describe this product's matrix (the same arrays and shape) and fit its
    // recorded layout; its memory must not overlap the product's output.
    const bsr_matrix_t *W = it.W;
    if (!plan->mem) return BSR_ERR_NULL;
    if (plan->n_rows != W->n_rows || plan->n_cols != W->n_cols || plan->nnzb != W->nnzb ||
        plan->R != W->R || plan->C != W->C || plan->dtype != int(W->dtype) ||
        plan->indptr != W->indptr || plan->indices != W->indices || plan->data != W->data)
        return BSR_ERR_ARG;
    if (layout_bytes <= 0 || int64_t(plan->bytes) < layout_bytes) return BSR_ERR_ARG;
    if (it.T > 0 && overlaps(it.Y, ((it.T - 1) * it.ldy + W->n_rows) * 4, plan->mem,
                             int64_t(plan->bytes)))
        return BSR_ERR_ARG;
    return BSR_OK;
}

bsr_status check_plan_prepare(const bsr_matrix_t *W, const void *mem, size_t bytes,
                              int64_t layout_bytes) {
    // mem must hold the layout and not overlap the matrix it reads.
    if (!mem) return BSR_ERR_NULL;
    if (int64_t(bytes) < layout_bytes) return BSR_ERR_WORKSPACE;
    if (overlaps(mem, layout_bytes, W->indptr, indptr_bytes(W)) ||
        overlaps(mem, layout_bytes, W->indices, W->nnzb * 4) ||
        overlaps(mem, layout_bytes, W->data, data_bytes(W)))
        return BSR_ERR_ARG;
    return BSR_OK;
}

bsr_status check_to_dense(const bsr_matrix_t *W, const float *out, int64_t ldo) {
    if (!W || !out) return BSR_ERR_NULL;
    bsr_status s = check_matrix(W);
    if (s != BSR_OK) return s;
    if (W->dtype != BSR_F32) return BSR_ERR_DTYPE;
    if (ldo < W->n_cols) return BSR_ERR_SHAPE;
    if (W->n_rows > kMaxElems / ldo) return BSR_ERR_UNSUPPORTED;
    return BSR_OK;
}

bsr_status check_reblock(const bsr_matrix_t *W, int32_t R2, int32_t C2,
                         const int32_t *indptr_out, const int32_t *indices_out,
                         const void *data_out) {
    bsr_status s = check_matrix(W);
    if (s != BSR_OK) return s;
    if (R2 <= 0 || C2 <= 0 || W->R % R2 != 0 || W->C % C2 != 0) return BSR_ERR_SHAPE;
    if (!indptr_out) return BSR_ERR_NULL;
    if (W->nnzb > 0 && (!indices_out || !data_out)) return BSR_ERR_NULL;
    const int64_t pieces = int64_t(W->R / R2) * (W->C / C2);
    const int64_t Nb = W->n_rows / R2, Kb = W->n_cols / C2;
    if (Nb > kMaxBlocks / Kb) return BSR_ERR_UNSUPPORTED;
    if (W->nnzb > kMaxBlocks / pieces) return BSR_ERR_UNSUPPORTED;
    // Outputs must not overlap the inputs or each other.
    const int64_t n2 = W->nnzb * pieces;
    const int64_t outs[3] = {(Nb + 1) * 4, n2 * 4, data_bytes(W)};
    const void *optr[3] = {indptr_out, indices_out, data_out};
    const void *iptr[3] = {W->indptr, W->indices, W->data};
    const int64_t ins[3] = {indptr_bytes(W), W->nnzb * 4, data_bytes(W)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 3; ++j)
            if (overlaps(optr[i], outs[i], iptr[j], ins[j])) return BSR_ERR_ARG;
        for (int j = i + 1; j < 3; ++j)
            if (overlaps(optr[i], outs[i], optr[j], outs[j])) return BSR_ERR_ARG;
    }
    return BSR_OK;
}

bsr_status check_cast(const float *src, const uint16_t *dst, int64_t n) {
    if (n < 0) return BSR_ERR_SHAPE;
    if (n > 0 && (!src || !dst)) return BSR_ERR_NULL;
    if (n > kMaxElems) return BSR_ERR_UNSUPPORTED;
    return BSR_OK;
}

bsr_status check_iht_update(const float *W, int64_t ldw, const float *G, int64_t ldg,
                            const float *C0, int64_t ldc, float eta, int64_t N, int64_t K,
                            const float *V, int64_t ldv) {
    if (N < 0 || K < 0) return BSR_ERR_SHAPE;
    if (ldw < K || ldv < K || ldg < N || ldc < N) return BSR_ERR_SHAPE;
    if (!std::isfinite(eta)) return BSR_ERR_ARG;
    if (N == 0 || K == 0) return BSR_OK;
    if (!W || !G || !C0 || !V) return BSR_ERR_NULL;
    if (N > kMaxElems / ldw || N > kMaxElems / ldv || K > kMaxElems / ldg ||
        K > kMaxElems / ldc || N > (int64_t(1) << 37) || K > int64_t(65535) * 64)
        return BSR_ERR_UNSUPPORTED;
    // V may be W itself (each element is read before it is written, by the same thread), but
    // no other overlap of V with an input.
    const int64_t vb = ((N - 1) * ldv + K) * 4;
    if (overlaps(V, vb, G, ((K - 1) * ldg + N) * 4) || overlaps(V, vb, C0, ((K - 1) * ldc + N) * 4))
        return BSR_ERR_ARG;
    if (V != W && overlaps(V, vb, W, ((N - 1) * ldw + K) * 4)) return BSR_ERR_ARG;
    if (V == W && ldv != ldw) return BSR_ERR_ARG;
    return BSR_OK;
}

bsr_status check_attention(const float *Q, int64_t ldq, const float *K, int64_t ldk,
                           const float *V, int64_t ldv, const float *O, int64_t ldo,
                           int32_t batch, int32_t seq, int32_t heads, int32_t head_dim,
                           float scale) {
    if (batch < 0 || seq < 0 || heads < 1 || head_dim < 1) return BSR_ERR_SHAPE;
    const int64_t width = int64_t(heads) * head_dim;
    if (ldq < width || ldk < width || ldv < width || ldo < width) return BSR_ERR_SHAPE;
    if (!std::isfinite(scale)) return BSR_ERR_ARG;
    if (int64_t(batch) * seq == 0) return BSR_OK;
    if (!Q || !K || !V || !O) return BSR_ERR_NULL;
    if (head_dim != 64 || batch > 65535 || heads > 65535) return BSR_ERR_UNSUPPORTED;
    auto aligned = [](const void *p, int64_t ld) {
        return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 4 == 0;
    };
    if (!aligned(Q, ldq) || !aligned(K, ldk) || !aligned(V, ldv)) return BSR_ERR_UNSUPPORTED;
    const int64_t T = int64_t(batch) * seq;
    if (T > kMaxElems / ldq || T > kMaxElems / ldk || T > kMaxElems / ldv || T > kMaxElems / ldo)
        return BSR_ERR_UNSUPPORTED;
    return BSR_OK;
}

namespace {

// Rows that a call reads or writes: the bytes from the first to the end of the last, the pitch and
// the width of a row (an array without rows: its whole width).
struct Span {
    const void *p;
    int64_t bytes, pitch, width;
};

// `rows` rows of `width` elements of `size` bytes at pitch ld: sizes that are checked before, except
// the pitch of an array that is not given.
Span span(const void *p, int64_t rows, int64_t ld, int64_t width, int64_t size) {
    if (!p || rows <= 0) return Span{p, 0, 0, 0};
    return Span{p, ((rows - 1) * ld + width) * size, ld * size, width * size};
}

// Whether two arrays share bytes.  Columns of one buffer (the same pitch, such as G and U side by side)
// lie within each other's range without sharing any: their rows stay apart where the distance of
// their starts, modulo the pitch, leaves room for both.
bool overlaps(const Span &a, const Span &b) {
    if (!overlaps(a.p, a.bytes, b.p, b.bytes)) return false;
    if (a.pitch != b.pitch) return true;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
    const int64_t apart = int64_t(pb > pa ? pb - pa : pa - pb) % a.pitch;
    const int64_t first = pb > pa ? a.width : b.width, second = pb > pa ? b.width : a.width;
    return apart < first || apart + second > a.pitch;
}

// No output overlaps an input or another output.
template <size_t I, size_t O>
bool disjoint(const Span (&in)[I], const Span (&out)[O]) {
    for (size_t i = 0; i < O; ++i) {
        for (size_t j = 0; j < I; ++j)
            if (overlaps(out[i], in[j])) return false;
        for (size_t j = i + 1; j < O; ++j)
            if (overlaps(out[i], out[j])) return false;
    }
    return true;
}

bool known_dtype(int32_t d) { return d == BSR_F32 || d == BSR_BF16 || d == BSR_I8; }
int64_t dtype_size(int32_t d) { return d == BSR_F32 ? 4 : d == BSR_BF16 ? 2 : 1; }

// The block's own description, for a call whose operands are 8-bit or not; `T` bounds its outputs.
bsr_status check_gated_block(const bsr_gated_t *W, bool i8, int64_t T, int64_t ldx) {
    if (!W) return BSR_ERR_NULL;
    const int32_t dt = raw_enum(W->dtype);
    if (!known_dtype(dt) || W->act < BSR_ACT_SILU || W->act > BSR_ACT_RELU) return BSR_ERR_ARG;
    if ((dt == BSR_I8) != i8) return BSR_ERR_DTYPE;
    if (W->K < 1 || W->F < 1 || T < 0 || W->ldg < W->K || W->ldu < W->K || ldx < W->K)
        return BSR_ERR_SHAPE;
    if (W->K > kDenseMaxWidth || W->F > kDenseMaxWidth || W->ldg > kDenseMaxWidth ||
        W->ldu > kDenseMaxWidth || ldx > kDenseMaxWidth || T > kDenseMaxTokens ||
        W->F * T > kDenseMaxOut / 2 || (i8 && W->K > kI8MaxK))
        return BSR_ERR_UNSUPPORTED;
    if (!W->Wg || !W->Wu || (i8 && (!W->sg || !W->su))) return BSR_ERR_NULL;
    return BSR_OK;
}

}  // namespace

bsr_status check_quantize_rows(const void *X, int32_t x_dtype, int64_t T, int64_t K, int64_t ldx,
                               const int8_t *Q, int64_t ldq, const float *scale) {
    if (!known_dtype(x_dtype)) return BSR_ERR_ARG;
    if (x_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || ldx < K || ldq < K) return BSR_ERR_SHAPE;
    if (ldx > kDenseMaxWidth || ldq > kDenseMaxWidth || T > kDenseMaxTokens)
        return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!X || !Q || !scale) return BSR_ERR_NULL;
    const Span in[] = {span(X, T, ldx, K, dtype_size(x_dtype))};
    const Span out[] = {span(Q, T, ldq, K, 1), span(scale, 1, T, T, 4)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

bsr_status check_matmul_i8(const int8_t *Xq, int64_t T, int64_t K, int64_t ldx, const float *sx,
                           const int8_t *Wq, int64_t N, int64_t ldw, const float *sw,
                           const float *bias, const void *Y, int32_t y_dtype, int64_t ldy) {
    if (!known_dtype(y_dtype)) return BSR_ERR_ARG;
    if (y_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || N < 1 || ldx < K || ldw < K || ldy < N) return BSR_ERR_SHAPE;
    if (K > kI8MaxK || ldx > kDenseMaxWidth || ldw > kDenseMaxWidth || ldy > kDenseMaxWidth ||
        T > kDenseMaxTokens || T * N > kDenseMaxOut)
        return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!Xq || !sx || !Wq || !sw || !Y) return BSR_ERR_NULL;
    const Span in[] = {span(Xq, T, ldx, K, 1), span(Wq, N, ldw, K, 1), span(sx, 1, T, T, 4),
                       span(sw, 1, N, N, 4), span(bias, 1, N, N, 4)};
    const Span out[] = {span(Y, T, ldy, N, dtype_size(y_dtype))};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

bsr_status check_gated(const void *X, int64_t T, int64_t ldx, const bsr_gated_t *W, const void *H,
                       int64_t ldh, const float *G, const float *U, int64_t ldp) {
    const bsr_status s = check_gated_block(W, false, T, ldx);
    if (s != BSR_OK) return s;
    const bool keep = G || U;
    if (ldh < W->F || (keep && ldp < W->F)) return BSR_ERR_SHAPE;
    if (ldh > kDenseMaxWidth || (keep && ldp > kDenseMaxWidth)) return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!X || !H || (keep && (!G || !U))) return BSR_ERR_NULL;
    const int64_t e = dtype_size(raw_enum(W->dtype)), K = W->K, F = W->F;
    const Span in[] = {span(X, T, ldx, K, e), span(W->Wg, F, W->ldg, K, e),
                       span(W->Wu, F, W->ldu, K, e), span(W->bg, 1, F, F, 4),
                       span(W->bu, 1, F, F, 4)};
    const Span out[] = {span(H, T, ldh, F, e), span(G, T, ldp, F, 4), span(U, T, ldp, F, 4)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

bsr_status check_gated_i8(const int8_t *Xq, int64_t T, int64_t ldx, const float *sx,
                          const bsr_gated_t *W, const void *H, int32_t h_dtype, int64_t ldh) {
    const bsr_status s = check_gated_block(W, true, T, ldx);
    if (s != BSR_OK) return s;
    if (!known_dtype(h_dtype)) return BSR_ERR_ARG;
    if (h_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (ldh < W->F) return BSR_ERR_SHAPE;
    if (ldh > kDenseMaxWidth) return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!Xq || !sx || !H) return BSR_ERR_NULL;
    const int64_t K = W->K, F = W->F;
    const Span in[] = {span(Xq, T, ldx, K, 1), span(W->Wg, F, W->ldg, K, 1),
                       span(W->Wu, F, W->ldu, K, 1), span(sx, 1, T, T, 4),
                       span(W->sg, 1, F, F, 4), span(W->su, 1, F, F, 4),
                       span(W->bg, 1, F, F, 4), span(W->bu, 1, F, F, 4)};
    const Span out[] = {span(H, T, ldh, F, dtype_size(h_dtype))};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

GatedWorkspace gated_workspace_layout(int64_t T, int64_t K, int64_t F, int32_t dtype) {
    GatedWorkspace w{};
    const int64_t e = dtype_size(dtype), per = 16 / e;
    const int64_t blocks = (T + kGatedRowsPerPartial - 1) / kGatedRowsPerPartial;
    const bool bf16 = dtype == BSR_BF16;
    auto up = [](int64_t n, int64_t m) { return (n + m - 1) / m * m; };
    w.Fp = up(F, bf16 ? 32 : per);
    w.Kp = up(K, per);
    w.Tp = up(T, per);
    w.grad_offset = 0;
    w.gradt_offset = align256(size_t(T * 2 * w.Fp * e));
    w.x_offset = align256(w.gradt_offset + size_t((bf16 ? T * 2 * w.Fp : 2 * F * w.Tp) * e));
    w.w_offset = align256(w.x_offset + size_t(bf16 ? T * w.Kp * e : K * w.Tp * e));
    w.partial_offset = align256(w.w_offset + size_t(bf16 ? 2 * F * w.Kp * e : K * 2 * w.Fp * e));
    w.slice_offset = align256(w.partial_offset + size_t(blocks * 2 * F * 4));
    const int64_t dw_rows = bf16 ? 2 * w.Fp : 2 * F;
    w.x_slices = gated_slices(T, K, (2 * w.Fp + 31) / 32, bf16);
    w.w_slices = gated_slices(dw_rows, K, (T + 31) / 32, bf16);
    const int64_t xs = w.x_slices > 1 ? w.x_slices * T * K : 0;
    const int64_t ws = w.w_slices > 1 ? w.w_slices * dw_rows * K : 0;
    w.total = align256(w.slice_offset + size_t(xs > ws ? xs : ws) * 4);
    if (w.total == 0) w.total = 256;
    return w;
}

bsr_status check_gated_backward(const void *dH, int64_t lddh, const void *X, int64_t T,
                                int64_t ldx, const bsr_gated_t *W, const float *G, const float *U,
                                int64_t ldp, const void *dX, int64_t lddx, const void *dWg,
                                const void *dWu, int64_t lddw, const void *dbg, const void *dbu,
                                int32_t grad_dtype, const void *workspace, size_t ws_bytes) {
    const bsr_status s = check_gated_block(W, false, T, ldx);
    if (s != BSR_OK) return s;
    if (!known_dtype(grad_dtype)) return BSR_ERR_ARG;
    if (grad_dtype == BSR_I8) return BSR_ERR_DTYPE;
    const int64_t K = W->K, F = W->F;
    const bool dw = dWg || dWu;
    if (lddh < F || ldp < F || (dX && lddx < K) || (dw && lddw < K)) return BSR_ERR_SHAPE;
    if (T > kGatedMaxBackwardTokens || lddh > kDenseMaxWidth || ldp > kDenseMaxWidth ||
        (dX && lddx > kDenseMaxWidth) || (dw && lddw > kDenseMaxWidth) ||
        F > kGatedMaxBackwardWidth || F * K > kDenseMaxOut / 2 || T * K > kDenseMaxOut)
        return BSR_ERR_UNSUPPORTED;
    if (dw && (!dWg || !dWu)) return BSR_ERR_NULL;
    if (T > 0 && (!dH || !X || !G || !U)) return BSR_ERR_NULL;
    const int32_t dt = raw_enum(W->dtype);
    const int64_t e = dtype_size(dt), g = dtype_size(grad_dtype);
    const size_t need = gated_workspace_layout(T, K, F, dt).total;
    if (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0)
        return BSR_ERR_WORKSPACE;
    const Span in[] = {span(dH, T, lddh, F, e), span(X, T, ldx, K, e),
                       span(W->Wg, F, W->ldg, K, e), span(W->Wu, F, W->ldu, K, e),
                       span(G, T, ldp, F, 4), span(U, T, ldp, F, 4)};
    const Span out[] = {span(dX, T, lddx, K, e), span(dWg, F, lddw, K, g),
                        span(dWu, F, lddw, K, g), span(dbg, 1, F, F, g), span(dbu, 1, F, F, g),
                        span(workspace, 1, int64_t(need), int64_t(need), 1)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

// --- norms and 8-bit floating point -------------------------------------------------------------

bsr_status check_layer_norm(const void *X, int64_t ldx, const void *R, int64_t ldr, int64_t T, int64_t K,
                            int32_t dtype, const float *gamma, const float *beta, float eps,
                            const void *Y, int64_t ldy, const void *S, int64_t lds, const float *mean,
                            const float *rstd) {
    if (!known_dtype(dtype) || !std::isfinite(eps) || eps < 0.0f || (S && !R)) return BSR_ERR_ARG;
    if (dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || ldx < K || ldy < K || (R && ldr < K) || (S && lds < K)) return BSR_ERR_SHAPE;
    if (T > kDenseMaxTokens || K > kDenseMaxWidth || ldx > kDenseMaxWidth || ldy > kDenseMaxWidth ||
        (R && ldr > kDenseMaxWidth) || (S && lds > kDenseMaxWidth))
        return BSR_ERR_UNSUPPORTED;
    if (!mean != !rstd) return BSR_ERR_NULL;
    if (T == 0) return BSR_OK;
    if (!X || !Y) return BSR_ERR_NULL;
    const int64_t e = dtype_size(dtype);
    const Span in[] = {span(X, T, ldx, K, e), span(R, T, ldr, K, e), span(gamma, 1, K, K, 4),
                       span(beta, 1, K, K, 4)};
    const Span out[] = {span(Y, T, ldy, K, e), span(S, T, lds, K, e), span(mean, 1, T, T, 4),
                        span(rstd, 1, T, T, 4)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

bsr_status check_layer_norm_backward(const void *dY, int64_t lddy, const void *S, int64_t lds, int64_t T,
                                     int64_t K, int32_t dtype, const float *gamma, const float *mean,
                                     const float *rstd, const void *dS, int64_t ldds, const void *dX,
                                     int64_t lddx, const void *dgamma, const void *dbeta,
                                     int32_t grad_dtype, const void *workspace, size_t ws_bytes) {
    if (!known_dtype(dtype) || !known_dtype(grad_dtype)) return BSR_ERR_ARG;
    if (dtype == BSR_I8 || grad_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || lddy < K || lds < K || (dS && ldds < K) || (dX && lddx < K))
        return BSR_ERR_SHAPE;
    if (T > kDenseMaxTokens || K > kDenseMaxWidth || lddy > kDenseMaxWidth || lds > kDenseMaxWidth ||
        (dS && ldds > kDenseMaxWidth) || (dX && lddx > kDenseMaxWidth))
        return BSR_ERR_UNSUPPORTED;
    if (T > 0 && (!dY || !S || !mean || !rstd)) return BSR_ERR_NULL;
    const bool vectors = dgamma || dbeta;
    const size_t need = vectors ? layer_norm_workspace(T, K).bytes : 0;
    if (vectors &&
        (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0))
        return BSR_ERR_WORKSPACE;
    const int64_t e = dtype_size(dtype), g = dtype_size(grad_dtype);
    const Span in[] = {span(dY, T, lddy, K, e),   span(S, T, lds, K, e),   span(dS, T, ldds, K, e),
                       span(gamma, 1, K, K, 4), span(mean, 1, T, T, 4), span(rstd, 1, T, T, 4)};
    const Span out[] = {span(dX, T, lddx, K, e), span(dgamma, 1, K, K, g), span(dbeta, 1, K, K, g),
                        span(vectors ? workspace : nullptr, 1, int64_t(need), int64_t(need), 1)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

namespace {

bool known_f8(int32_t f) { return f == BSR_E4M3 || f == BSR_E5M2; }
int64_t blocks_of(int64_t n, int64_t rows) { return n / rows + (n % rows != 0); }

}  // namespace

bsr_status check_quantize_f8(const void *X, int32_t x_dtype, int64_t T, int64_t K, int64_t ldx,
                             int32_t block_rows, int32_t format, const void *Q, int64_t ldq,
                             const float *scale, int64_t ldscale, const void *QT, int64_t ldqt,
                             const float *scale_t, int64_t ldscale_t) {
    if (!known_dtype(x_dtype) || !known_f8(format) || (block_rows != 1 && block_rows != kF8Block))
        return BSR_ERR_ARG;
    if (x_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || ldx < K) return BSR_ERR_SHAPE;
    if (T > kDenseMaxTokens || ldx > kDenseMaxWidth) return BSR_ERR_UNSUPPORTED;
    const bool rows = Q || scale, columns = QT || scale_t;
    const int64_t kb = blocks_of(K, kF8Block), tb = blocks_of(T, kF8Block);
    const int64_t row_scales = blocks_of(T, block_rows), column_scales = blocks_of(K, block_rows);
    if ((rows && (ldq < K || ldscale < row_scales)) ||
        (columns && (ldqt < T || ldqt < 1 || ldscale_t < column_scales)))
        return BSR_ERR_SHAPE;
    if ((rows && (ldq > kDenseMaxWidth || ldscale > kDenseMaxTokens)) ||
        (columns && (ldqt > kDenseMaxWidth || ldscale_t > kDenseMaxTokens)))
        return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!X || !Q != !scale || !QT != !scale_t || (!Q && !QT)) return BSR_ERR_NULL;
    const Span in[] = {span(X, T, ldx, K, dtype_size(x_dtype))};
    const Span out[] = {span(Q, T, ldq, K, 1), span(scale, kb, ldscale, row_scales, 4),
                        span(QT, K, ldqt, T, 1), span(scale_t, tb, ldscale_t, column_scales, 4)};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

bsr_status check_matmul_f8(const void *Xq, int32_t x_format, int64_t T, int64_t K, int64_t ldx,
                           const float *sx, int64_t ldsx, const void *Wq, int64_t N, int64_t ldw,
                           const float *sw, int64_t ldsw, int32_t w_block_rows, const float *bias,
                           const void *Y, int32_t y_dtype, int64_t ldy) {
    if (!known_dtype(y_dtype) || !known_f8(x_format) || (w_block_rows != 1 && w_block_rows != kF8Block))
        return BSR_ERR_ARG;
    if (y_dtype == BSR_I8) return BSR_ERR_DTYPE;
    if (T < 0 || K < 1 || N < 1 || ldx < K || ldw < K || ldy < N || ldsx < T ||
        ldsw < blocks_of(N, w_block_rows))
        return BSR_ERR_SHAPE;
    if (ldx > kDenseMaxWidth || ldw > kDenseMaxWidth || ldy > kDenseMaxWidth || N > kDenseMaxWidth ||
        T > kDenseMaxTokens || ldsx > kDenseMaxTokens || ldsw > kDenseMaxTokens ||
        T * N > kDenseMaxOut)
        return BSR_ERR_UNSUPPORTED;
    if (T == 0) return BSR_OK;
    if (!Xq || !sx || !Wq || !sw || !Y) return BSR_ERR_NULL;
    const int64_t kb = blocks_of(K, kF8Block), wb = blocks_of(N, w_block_rows);
    const Span in[] = {span(Xq, T, ldx, K, 1), span(Wq, N, ldw, K, 1), span(sx, kb, ldsx, T, 4),
                       span(sw, kb, ldsw, wb, 4), span(bias, 1, N, N, 4)};
    const Span out[] = {span(Y, T, ldy, N, dtype_size(y_dtype))};
    return disjoint(in, out) ? BSR_OK : BSR_ERR_ARG;
}

}  // namespace bsr

extern "C" {

size_t bsr_layer_norm_workspace_bytes(int64_t T, int64_t K) {
    if (T < 0 || K < 1 || T > bsr::kDenseMaxTokens || K > bsr::kDenseMaxWidth) return 0;
    return bsr::layer_norm_workspace(T, K).bytes;
}

size_t bsr_gated_workspace_bytes(int64_t T, int64_t K, int64_t F, bsr_dtype dtype) {
    const int32_t dt = bsr::raw_enum(dtype);
    if (T < 0 || K < 1 || F < 1 || T > bsr::kGatedMaxBackwardTokens ||
        K > bsr::kDenseMaxWidth || F > bsr::kGatedMaxBackwardWidth ||
        (dt != BSR_F32 && dt != BSR_BF16))
        return 0;
    return bsr::gated_workspace_layout(T, K, F, dt).total;
}

bsr_status bsr_prune_count(int64_t N, int64_t K, int32_t R, int32_t C, double density,
                           int64_t *k) {
    if (!k) return BSR_ERR_NULL;
    if (!tiles(N, K, R, C)) return BSR_ERR_SHAPE;
    if (!(density >= 0.0 && density <= 1.0)) return BSR_ERR_ARG;  // rejects NaN too
    const int64_t Nb = N / R, Kb = K / C;
    if (Nb > kMaxBlocks / Kb) return BSR_ERR_UNSUPPORTED;
    const int64_t nb = Nb * Kb;
    double v = std::floor(density * double(nb) + 0.5);
    int64_t kk = int64_t(v);
    if (kk < 0) kk = 0;
    if (kk > nb) kk = nb;
    *k = kk;
    return BSR_OK;
}

bsr_status bsr_prune_count_ex(int64_t N, int64_t K, int32_t R, int32_t C, double density,
                              const bsr_prune_options_t *opts, int64_t *k) {
    const int32_t norm = opts ? opts->norm : BSR_NORM_L2;
    const int32_t select = opts ? opts->select : BSR_SELECT_GLOBAL;
    if (norm != BSR_NORM_L2 && norm != BSR_NORM_L1) return BSR_ERR_ARG;
    if (select != BSR_SELECT_GLOBAL && select != BSR_SELECT_PER_ROW) return BSR_ERR_ARG;
    if (select == BSR_SELECT_GLOBAL) return bsr_prune_count(N, K, R, C, density, k);
    if (!k) return BSR_ERR_NULL;
    if (!tiles(N, K, R, C)) return BSR_ERR_SHAPE;
    if (!(density >= 0.0 && density <= 1.0)) return BSR_ERR_ARG;
    const int64_t Nb = N / R, Kb = K / C;
    if (Nb > kMaxBlocks / Kb) return BSR_ERR_UNSUPPORTED;
    int64_t kr = int64_t(std::floor(density * double(Kb) + 0.5));
    if (kr < 0) kr = 0;
    if (kr > Kb) kr = Kb;
    *k = Nb * kr;
    return BSR_OK;
}

size_t bsr_prune_workspace_bytes(int64_t N, int64_t K, int32_t R, int32_t C) {
    if (!tiles(N, K, R, C)) return 0;
    const int64_t Nb = N / R, Kb = K / C;
    if (Nb > kMaxBlocks / Kb) return 0;
    return bsr::prune_workspace_layout(Nb * Kb).total;
}

const char *bsr_status_str(bsr_status s) {
    switch (s) {
        case BSR_OK: return "ok";
        case BSR_ERR_NULL: return "null pointer argument";
        case BSR_ERR_SHAPE: return "invalid shape or leading dimension";
        case BSR_ERR_ARG: return "invalid argument value";
        case BSR_ERR_DTYPE: return "dtype mismatch";
        case BSR_ERR_CAPACITY: return "output capacity too small";
        case BSR_ERR_WORKSPACE: return "workspace missing or too small";
        case BSR_ERR_HIP: return "HIP runtime error";
        case BSR_ERR_ARCH: return "device is not gfx950";
        case BSR_ERR_UNSUPPORTED: return "unsupported size";
    }
    return "unknown status";
}

}  // extern "C"
