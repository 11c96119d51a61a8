// Internal declarations shared by libbsr's translation units (not part of the C ABI).
#pragma once

#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include "../../include/libbsr.h"

namespace bsr {

// The integer in an enum-typed field or argument a caller passed (a C caller may store any
// int32 there), read as bytes: loading an enum lvalue that names no enumerator is undefined in
// C++, so validation reads enums this way before checking them.
template <class E>
inline int32_t raw_enum(const E &e) {
    static_assert(sizeof(E) == sizeof(int32_t), "the ABI's enums are 32-bit");
    int32_t v;
    memcpy(&v, &e, sizeof v);
    return v;
}

// Workspace layout of the pruning pipeline: fp64 key bits per block, then the source block id
// of every kept block.  Each region starts on a 256-byte boundary.
struct PruneWorkspace {
    size_t key_offset, key_bytes;
    size_t src_offset, src_bytes;
    size_t total;
};
PruneWorkspace prune_workspace_layout(int64_t nb);

// Host-side argument checks; pure C++ (no HIP), so they also run where no GPU exists.
bsr_status check_prune(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t R, int32_t C,
                       int64_t k, const int32_t *indptr, const int32_t *indices,
                       const float *data, int64_t capacity_blocks, const void *workspace,
                       size_t ws_bytes);
// bsr_prune_from_dense_noalloc: the workspace lives in a fixed device array of this many bytes,
// the prune workspace of BSR_NOALLOC_MAX_BLOCKS blocks (8-byte keys, then 4-byte source ids,
// each region a multiple of 256 bytes).
constexpr size_t kNoallocScratchBytes = size_t(BSR_NOALLOC_MAX_BLOCKS) * 8 +
                                        size_t(BSR_NOALLOC_MAX_BLOCKS) * 4;
static_assert(BSR_NOALLOC_MAX_BLOCKS % 64 == 0, "both regions stay 256-byte multiples");
bsr_status check_prune_noalloc(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t R,
                               int32_t C, int64_t k, const int32_t *indptr,
                               const int32_t *indices, const float *data,
                               int64_t capacity_blocks);
// Device address of this device's scratch array (found once per device, with it current).
bsr_status noalloc_scratch(void **ptr);
// Options of the _ex pruning entry point (after check_prune: N, R valid, k in [0, nb]).
bsr_status check_prune_options(const bsr_prune_options_t *opts, int64_t N, int32_t R, int64_t k);
bsr_status check_matrix(const bsr_matrix_t *W);
bsr_status check_spmm(const void *X, int x_dtype, int64_t T, int64_t ldx, const bsr_matrix_t *W,
                      const float *Y, int64_t ldy, const float *bias);
// A plan used by a product (after check_spmm): it describes the item's matrix, its recorded
// size covers `layout_bytes`, and it does not overlap the item's Y.
bsr_status check_plan_use(const bsr_spmm_item_t &it, const bsr_plan_t *plan,
                          int64_t layout_bytes);
// Plan memory for a matrix (after check_matrix): large enough, not overlapping the matrix.
bsr_status check_plan_prepare(const bsr_matrix_t *W, const void *mem, size_t bytes,
                              int64_t layout_bytes);
// Cross-product aliasing of a batched call (after check_spmm on every item).
bsr_status check_spmm_items(const bsr_spmm_item_t *items, int32_t n);
bsr_status check_to_dense(const bsr_matrix_t *W, const float *out, int64_t ldo);
bsr_status check_cast(const float *src, const uint16_t *dst, int64_t n);
bsr_status check_iht_update(const float *W, int64_t ldw, const float *G, int64_t ldg,
                            const float *C0, int64_t ldc, float eta, int64_t N, int64_t K,
                            const float *V, int64_t ldv);
bsr_status check_reblock(const bsr_matrix_t *W, int32_t R2, int32_t C2,
                         const int32_t *indptr_out, const int32_t *indices_out,
                         const void *data_out);
bsr_status check_attention(const float *Q, int64_t ldq, const float *K, int64_t ldk,
                           const float *V, int64_t ldv, const float *O, int64_t ldo,
                           int32_t batch, int32_t seq, int32_t heads, int32_t head_dim,
                           float scale);

// The dense products (8-bit and gated): limits that keep every tile's byte offsets in 32 bits (a
// tile spans at most 256 rows of at most 4 MiB) and every grid below 2^32 threads in x and 2^16
// workgroups in y (dense_plan.h, tests/host/dense_grids.cpp).
constexpr int64_t kDenseMaxWidth = int64_t(1) << 20;    // columns and pitches, elements
constexpr int64_t kDenseMaxTokens = int64_t(1) << 24;
constexpr int64_t kDenseMaxOut = int64_t(1) << 36;      // elements of all outputs of one tile grid
constexpr int64_t kGatedMaxBackwardTokens = int64_t(1) << 20;   // T is a pitch (fp32 transposes)
constexpr int64_t kGatedMaxBackwardWidth = kDenseMaxWidth / 2 - 32;   // F: 2 F, padded, is a pitch
constexpr int64_t kI8MaxK = 131071;                     // 2^14 * K stays below 2^31
bsr_status check_quantize_rows(const void *X, int32_t x_dtype, int64_t T, int64_t K, int64_t ldx,
                               const int8_t *Q, int64_t ldq, const float *scale);
bsr_status check_matmul_i8(const int8_t *Xq, int64_t T, int64_t K, int64_t ldx, const float *sx,
                           const int8_t *Wq, int64_t N, int64_t ldw, const float *sw,
                           const float *bias, const void *Y, int32_t y_dtype, int64_t ldy);
bsr_status check_gated(const void *X, int64_t T, int64_t ldx, const bsr_gated_t *W, const void *H,
                       int64_t ldh, const float *G, const float *U, int64_t ldp);
bsr_status check_gated_i8(const int8_t *Xq, int64_t T, int64_t ldx, const float *sx,
                          const bsr_gated_t *W, const void *H, int32_t h_dtype, int64_t ldh);
bsr_status check_gated_backward(const void *dH, int64_t lddh, const void *X, int64_t T,
                                int64_t ldx, const bsr_gated_t *W, const float *G, const float *U,
                                int64_t ldp, const void *dX, int64_t lddx, const void *dWg,
                                const void *dWu, int64_t lddw, const void *dbg, const void *dbu,
                                int32_t grad_dtype, const void *workspace, size_t ws_bytes);
// Workspace of bsr_gated_backward: byte offsets of its regions, each on a 256-byte boundary.
struct GatedWorkspace {
    int64_t Fp;              // F rounded up to whole steps of 32 (bf16) or 16-byte chunks (fp32)
    int64_t Kp;              // bf16: K rounded up to whole 16-byte chunks
    int64_t Tp;              // fp32: T rounded up to whole 16-byte chunks
    size_t grad_offset;      // [T][2 Fp]: dG | dU, of the block's dtype
    size_t gradt_offset;     // fp32: [2 F][Tp], its transpose; bf16: [T][2 Fp], what its rounding dropped
    size_t x_offset;         // bf16: [T][Kp], a copy of an unaligned X; fp32: [K][Tp], X's transpose
    size_t w_offset;         // bf16: [2][F][Kp], copies; fp32: [K][2 Fp], the weights' transposes
    size_t partial_offset;   // fp32 [row blocks][2 F]: partial bias gradients
    int x_slices, w_slices;  // of dX's and of the weight gradients' product
    size_t slice_offset;     // fp32: the slices' sums, of one product at a time
    size_t total;
};
// Slices that a gradient product of M x N outputs and `steps` steps of its contraction (32 of it each)
// is cut into where 64 x 64 tiles leave CUs idle (of 256; bf16: where they do not give two workgroups
// to each, fp32 gains nothing from the second); a slice keeps at least 64 steps in bf16 (10 us) and 16
// in fp32 (8 us).  Each writes fp32 sums, which are added in order.
inline int gated_slices(int64_t M, int64_t N, int64_t steps, bool bf16) {
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    int64_t n = (bf16 ? 512 : 256) / (tiles > 0 ? tiles : 1);
    if (n > steps / (bf16 ? 64 : 16)) n = steps / (bf16 ? 64 : 16);
    if (n > 16) n = 16;
    return n > 1 ? int(n) : 1;
}
constexpr int kGatedRowsPerPartial = 64;
GatedWorkspace gated_workspace_layout(int64_t T, int64_t K, int64_t F, int32_t dtype);

// Device-side entry points (implemented in the .hip files).  Arguments are already validated.
bsr_status ensure_device();  // current device is gfx950; caches its properties
int device_cu_count();
int auto_slices(const int64_t *tiles, int n, int cu_count);  // token tiles per product
size_t device_lds_per_block();

bsr_status launch_prune(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t R, int32_t C,
                        int64_t k, int32_t *indptr, int32_t *indices, float *data,
                        void *workspace, int norm, int select, void *stream);
bsr_status launch_to_dense(const bsr_matrix_t *W, float *out, int64_t ldo, void *stream);
bsr_status launch_cast(const float *src, uint16_t *dst, int64_t n, void *stream);
bsr_status launch_iht_update(const float *W, int64_t ldw, const float *G, int64_t ldg,
                             const float *C0, int64_t ldc, float eta, int64_t N, int64_t K,
                             float *V, int64_t ldv, void *stream);
bsr_status launch_reblock(const bsr_matrix_t *W, int32_t R2, int32_t C2, int32_t *indptr_out,
                          int32_t *indices_out, void *data_out, void *stream);
// Optional event pair recorded at a product kernel's start and end (hipExtLaunchKernel).
struct LaunchEvents {
    void *start = nullptr;
    void *stop = nullptr;
};

bsr_status launch_spmm_generic(const void *X, int64_t T, int64_t ldx, const bsr_matrix_t *W,
                               const float *bias, float *Y, int64_t ldy, void *stream,
                               const LaunchEvents &ev);

bsr_status launch_attention(const float *Q, int64_t ldq, const float *K, int64_t ldk,
                            const float *V, int64_t ldv, float *O, int64_t ldo, int batch,
                            int seq, int heads, float scale, void *stream);

bsr_status launch_quantize_rows(const void *X, int x_dtype, int64_t T, int64_t K, int64_t ldx,
                                int8_t *Q, int64_t ldq, float *scale, void *stream);
bsr_status launch_matmul_i8(const int8_t *Xq, int64_t T, int64_t K, int64_t ldx, const float *sx,
                            const int8_t *Wq, int64_t N, int64_t ldw, const float *sw,
                            const float *bias, void *Y, int y_dtype, int64_t ldy, void *stream);
bsr_status launch_gated(const void *X, int64_t T, int64_t ldx, const bsr_gated_t &W, void *H,
                        int64_t ldh, float *G, float *U, int64_t ldp, void *stream);
bsr_status launch_gated_i8(const int8_t *Xq, int64_t T, int64_t ldx, const float *sx,
                           const bsr_gated_t &W, void *H, int h_dtype, int64_t ldh, void *stream);
bsr_status launch_gated_backward(const void *dH, int64_t lddh, const void *X, int64_t T,
                                 int64_t ldx, const bsr_gated_t &W, const float *G,
                                 const float *U, int64_t ldp, void *dX, int64_t lddx, void *dWg,
                                 void *dWu, int64_t lddw, void *dbg, void *dbu, int grad_dtype,
                                 void *workspace, void *stream);

void set_last_hip_error(const char *msg);

}  // namespace bsr
