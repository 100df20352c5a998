// Matmuls in 8-bit integers and tokens sorted by expert: what their entry points ask of arguments (no device needed; the CPU build of the
// host logic makes the same checks) and what host and kernels share.
#pragma once
#include <stdint.h>

#include "ftuner.h"

namespace ftk {

inline uint32_t i8_pitch(uint32_t k) { return (k + 15u) / 16u * 16u; }
inline bool aligned_to(const void *p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

constexpr uint32_t kMaxExperts = 1024, kMaxTopK = 32, kMaxCols = 1u << 20, kMaxK = 131071;

// A launch has fewer than 2^32 threads: rows, `per` of them to a workgroup of `threads`, that one can take.  More rows are several launches.
constexpr uint32_t kMostThreads = 0xffffffffu;
constexpr uint32_t launch_rows(uint32_t per, uint32_t threads) { return kMostThreads / threads * per; }

// ---- quantised rows ----
struct QuantArgs {
    const void *X;
    int8_t *Q;
    float *scale;
    uint32_t rows, cols, ldx, ldq;
};
// *launch: whether there is anything to do
inline ft_status quant_check(const ft_quant_desc *d, uint32_t rows, const void *X, int8_t *Q, float *scale, QuantArgs *a, bool *launch) {
    *launch = false;
    if (!d || d->struct_size != sizeof(*d) || d->dtype > FT_F32 || d->act > FT_ACT_SILU_MUL || d->cols == 0) return FT_ERR_INVALID_ARG;
    if (d->cols > kMaxCols || rows > 0x7fffffffu) return FT_ERR_UNSUPPORTED;
    const uint32_t width = d->act == FT_ACT_SILU_MUL ? 2u * d->cols : d->cols;
    a->rows = rows;
    a->cols = d->cols;
    a->ldx = d->ldx ? d->ldx : width;
    a->ldq = d->ldq ? d->ldq : i8_pitch(d->cols);
    if (a->ldx < width || a->ldq < d->cols || a->ldq % 16u) return FT_ERR_INVALID_ARG;
    if (a->ldx > 4u * kMaxCols || a->ldq > 4u * kMaxCols) return FT_ERR_UNSUPPORTED;
    if (rows == 0) return FT_OK;
    if (!X || !Q || !scale || !aligned_to(X, d->dtype == FT_F32 ? 4 : 2) || !aligned_to(Q, 16) || !aligned_to(scale, 4)) return FT_ERR_INVALID_ARG;
    a->X = X; a->Q = Q; a->scale = scale;
    *launch = true;
    return FT_OK;
}

// ---- products ----
struct I8Args {
    const int8_t *A, *B;
    const float *scale_a, *scale_b, *bias;
    void *C;
    const int32_t *offsets, *a_row;      // grouped launches
    uint32_t m, n, k;                    // m: rows of C
    uint32_t lda, ldb, ldc;
    uint32_t experts, a_rows;
    uint32_t gated;                      // C has n / 2 columns, silu(gate) * value
    uint32_t out_kind;                   // 0 fp32, 1 fp16, 2 bf16
    uint32_t vec;                        // rows of C can be written 16 bytes (8 where C has 16 bits) at a time
    uint32_t through;                    // rows of C lie on 64-byte blocks, and there are many: they are streamed and written through the L2
    uint32_t row_tiles, col_tiles;       // grid of the body that was chosen (grouped: the most row tiles there can be)
    uint32_t group;
    uint32_t cus;                        // compute units of the device
};
inline ft_status i8_check(const ft_i8_desc *d, bool grouped, uint32_t m, const int32_t *offsets, const int8_t *A, const float *scale_a, uint32_t a_rows,
                          const int32_t *a_row, const int8_t *B, const float *scale_b, const float *bias, void *C, I8Args *a, bool *launch) {
    *launch = false;
    if (!d || d->struct_size != sizeof(*d) || d->n == 0 || d->k == 0 || d->dtype > FT_BF16 || d->out_dtype > FT_OUT_SAME || d->epilogue > FT_EPI_SILU_MUL) return FT_ERR_INVALID_ARG;
    if (grouped ? d->experts == 0 : d->experts != 0) return FT_ERR_INVALID_ARG;
    a->gated = d->epilogue == FT_EPI_SILU_MUL;
    if (a->gated && d->n % 2u) return FT_ERR_INVALID_ARG;
    const uint32_t columns = a->gated ? d->n / 2u : d->n;
    if (d->n >= (1u << 20) || d->k > kMaxK || d->experts > kMaxExperts || m > 0x7fffffffu) return FT_ERR_UNSUPPORTED;
    a->m = m; a->n = d->n; a->k = d->k;
    a->lda = d->lda ? d->lda : i8_pitch(d->k);
    a->ldb = d->ldb ? d->ldb : i8_pitch(d->k);
    a->ldc = d->ldc ? d->ldc : columns;
    if (a->lda < d->k || a->ldb < d->k || a->ldc < columns || a->lda % 16u || a->ldb % 16u) return FT_ERR_INVALID_ARG;
    if (a->lda > (1u << 20) || a->ldb > (1u << 20) || a->ldc > (1u << 22)) return FT_ERR_UNSUPPORTED;
    if (grouped && (uint64_t)a_rows * a->lda >= 0x80000000ull) return FT_ERR_UNSUPPORTED;
    if ((d->epilogue == FT_EPI_BIAS) != (bias != nullptr)) return FT_ERR_INVALID_ARG;
    if (m == 0) return FT_OK;
    a->out_kind = d->out_dtype == FT_OUT_F32 ? 0u : d->dtype == FT_F16 ? 1u : 2u;
    const uint32_t es = a->out_kind ? 2u : 4u;
    if (!A || !scale_a || !B || !scale_b || !C || !aligned_to(A, 16) || !aligned_to(B, 16) || !aligned_to(scale_a, 4) || !aligned_to(scale_b, 4) ||
        !aligned_to(bias, 4) || !aligned_to(C, es))
        return FT_ERR_INVALID_ARG;
    if (grouped && (!offsets || !aligned_to(offsets, 4) || !aligned_to(a_row, 4) || a_rows == 0)) return FT_ERR_INVALID_ARG;
    a->A = A; a->B = B; a->scale_a = scale_a; a->scale_b = scale_b; a->bias = bias; a->C = C;
    a->offsets = offsets; a->a_row = a_row;
    a->experts = d->experts; a->a_rows = a_rows;
    // (256 rows within a buffer's 2 GB)
    a->vec = aligned_to(C, 16) && (uint64_t)a->ldc * es % 16u == 0 && columns % (16u / es) == 0 && (uint64_t)a->ldc * es <= (4u << 20);
    // Streamed and written through the L2 (64 x 128 tiles: 1024 x 2304 x 768 bf16, 4.7 MB, 8.1 us kept, 7.5 streamed; 4096 x 11008 x 768 58.8 and 50.9) or, where
    // little is written, kept: the launch then ends a memory's latency earlier (128 x 4096 x 4096, 1 MB, 9.45 us kept, 9.7 streamed).
    a->through = aligned_to(C, 64) && (uint64_t)a->ldc * es % 64u == 0 && (uint64_t)m * columns * es >= (4u << 20);
    *launch = true;
    return FT_OK;
}

// ---- tokens by expert ----
// The sort: blocks of 1024 entries, each of which counts all entries itself, up to kSortRecount of them; beyond, at most kSortBlocks blocks,
// whose counts for each expert are the workspace of a launch before.
constexpr uint32_t kSortRecount = 16384, kSortSmall = 1024, kSortBlock = 2048, kSortBlocks = 256;
inline uint32_t sort_blocks(uint64_t entries) {
    const uint64_t blocks = entries <= kSortRecount ? (entries + kSortSmall - 1) / kSortSmall : (entries + kSortBlock - 1) / kSortBlock;
    return blocks < 1 ? 1u : blocks < kSortBlocks ? (uint32_t)blocks : kSortBlocks;
}

inline ft_status expert_shape(const ft_expert_desc *d, uint32_t tokens) {
    if (!d || d->struct_size != sizeof(*d) || d->experts == 0 || d->top_k == 0) return FT_ERR_INVALID_ARG;
    if (d->experts > kMaxExperts || d->top_k > kMaxTopK || (uint64_t)tokens * d->top_k > 0x7fffffffull) return FT_ERR_UNSUPPORTED;
    return FT_OK;
}
inline ft_status expert_workspace(const ft_expert_desc *d, uint32_t tokens, uint64_t *bytes) {
    if (!bytes) return FT_ERR_INVALID_ARG;
    const ft_status st = expert_shape(d, tokens);
    if (st != FT_OK) return st;
    const uint64_t entries = (uint64_t)tokens * d->top_k;
    *bytes = entries > kSortRecount ? (uint64_t)sort_blocks(entries) * d->experts * 4u : 0u;
    return FT_OK;
}
inline ft_status sort_check(const ft_expert_desc *d, uint32_t tokens, const int32_t *expert_of, int32_t *offsets, int32_t *row_token, int32_t *row_of, void *workspace,
                            uint64_t workspace_bytes) {
    uint64_t need = 0;
    const ft_status st = expert_workspace(d, tokens, &need);
    if (st != FT_OK) return st;
    if (!offsets || !aligned_to(offsets, 4)) return FT_ERR_INVALID_ARG;
    if (tokens && (!expert_of || !row_token || !row_of || !aligned_to(expert_of, 4) || !aligned_to(row_token, 4) || !aligned_to(row_of, 4))) return FT_ERR_INVALID_ARG;
    if (need && (!workspace || !aligned_to(workspace, 16) || workspace_bytes < need)) return FT_ERR_INVALID_ARG;
    return FT_OK;
}

struct MoveArgs {
    const void *src, *other;             // rows of tokens or entries; combine_grad: dOut and Y
    void *dst;
    const int32_t *row_of;
    const float *weights;
    float *dweights;
    uint32_t tokens, top_k, cols, ld_token, ld_row;
    uint32_t entries;                    // of all launches of a call: rows of Y and dY
};
// Rows beyond what the last-level cache holds (256 MB) are streamed: 8192 tokens x 8 of 4096 bf16, all moves of a training step 640 us kept, 566
// streamed; 1234 x 6 of 1001 fp16 the rows stay for the next call: combine 7.0 us kept, 8.4 streamed.
constexpr uint64_t kStreamBytes = 256ull << 20;
inline bool move_streams(const MoveArgs &a, uint32_t bytes) { return (uint64_t)a.entries * a.cols * bytes > kStreamBytes; }
// what the three calls share; the caller has set the pointers of `a`
inline ft_status move_check(const ft_expert_desc *d, uint32_t tokens, bool need_other, MoveArgs *a, bool *launch) {
    *launch = false;
    const ft_status st = expert_shape(d, tokens);
    if (st != FT_OK) return st;
    if (d->cols == 0 || d->dtype > FT_F32) return FT_ERR_INVALID_ARG;
    if (d->cols > kMaxCols) return FT_ERR_UNSUPPORTED;
    a->tokens = tokens; a->top_k = d->top_k; a->cols = d->cols;
    a->entries = tokens * d->top_k;
    a->ld_token = d->ld_token ? d->ld_token : d->cols;
    a->ld_row = d->ld_row ? d->ld_row : d->cols;
    if (a->ld_token < d->cols || a->ld_row < d->cols) return FT_ERR_INVALID_ARG;
    if (a->ld_token > 4u * kMaxCols || a->ld_row > 4u * kMaxCols) return FT_ERR_UNSUPPORTED;
    if (tokens == 0) return FT_OK;
    const uint32_t es = d->dtype == FT_F32 ? 4u : 2u;
    if (!a->src || !a->dst || !a->row_of || !aligned_to(a->src, es) || !aligned_to(a->dst, es) || !aligned_to(a->row_of, 4)) return FT_ERR_INVALID_ARG;
    if (need_other && (!a->other || !aligned_to(a->other, es))) return FT_ERR_INVALID_ARG;
    if (!aligned_to(a->weights, 4) || !aligned_to(a->dweights, 4)) return FT_ERR_INVALID_ARG;
    *launch = true;
    return FT_OK;
}

}  // namespace ftk
