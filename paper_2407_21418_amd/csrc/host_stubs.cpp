// Device half of the library replaced by stubs, for a CPU-only build of the host logic (generator,
// planner, plan cache) under AddressSanitizer / UBSan: every call that would need a GPU reports
// FT_ERR_UNSUPPORTED; host-only plans (FT_PLAN_HOST_ONLY) work as in the real library.
#include "ft_internal.h"
#include "i8_ops.h"

ft_status ftd_upload(ft_plan *) { return FT_ERR_UNSUPPORTED; }
void ftd_release(ft_plan *) {}

extern "C" {
ft_status ft_hw_query(int32_t, ft_hw_model *) { return FT_ERR_UNSUPPORTED; }
// (the argument checks that need no device are those of the real entry points)
ft_status ft_launch_epilogue(const ft_plan *plan, const void *A, const void *B, void *C, const float *bias, void *) {
    if (!plan) return FT_ERR_INVALID_ARG;
    if ((plan->op.epilogue == FT_EPI_BIAS) != (bias != nullptr)) return FT_ERR_INVALID_ARG;
    if (plan->st.n_tiles == 0) return FT_OK;
    if (!A || !B || !C || !plan->d_descs) return FT_ERR_INVALID_ARG;
    return FT_ERR_UNSUPPORTED;
}
ft_status ft_launch(const ft_plan *plan, const void *A, const void *B, void *C, void *s) { return ft_launch_epilogue(plan, A, B, C, nullptr, s); }
ft_status ft_launch_noalloc(const ft_plan *, const void *, const void *, void *, const float *, void *) { return FT_ERR_UNSUPPORTED; }
ft_status ft_stream_rate(const void *, void *, uint64_t, uint32_t, void *, float *, float *, float *) { return FT_ERR_UNSUPPORTED; }
ft_status ft_launch_timed(const ft_plan *, const void *const *, const void *const *, void *const *, uint32_t, void *, uint32_t,
                          float *) { return FT_ERR_UNSUPPORTED; }
ft_status ft_launch_timed_graph(const ft_plan *, const void *const *, const void *const *, void *const *, uint32_t, void *,
                                uint32_t, float *) { return FT_ERR_UNSUPPORTED; }

ft_status ft_i8_quantize(const ft_quant_desc *desc, uint32_t rows, const void *X, int8_t *Q, float *scale, void *) {
    ftk::QuantArgs a = {};
    bool go;
    const ft_status st = ftk::quant_check(desc, rows, X, Q, scale, &a, &go);
    return st != FT_OK || !go ? st : FT_ERR_UNSUPPORTED;
}
ft_status ft_i8_matmul(const ft_i8_desc *desc, uint32_t m, const int8_t *A, const float *scale_a, const int8_t *B, const float *scale_b, const float *bias, void *C, void *) {
    ftk::I8Args a = {};
    bool go;
    const ft_status st = ftk::i8_check(desc, false, m, nullptr, A, scale_a, 0, nullptr, B, scale_b, bias, C, &a, &go);
    return st != FT_OK || !go ? st : FT_ERR_UNSUPPORTED;
}
ft_status ft_i8_matmul_experts(const ft_i8_desc *desc, uint32_t rows, const int32_t *offsets, const int8_t *A, const float *scale_a, const int32_t *a_row, uint32_t a_rows,
                               const int8_t *B, const float *scale_b, const float *bias, void *C, void *) {
    ftk::I8Args a = {};
    bool go;
    const ft_status st = ftk::i8_check(desc, true, rows, offsets, A, scale_a, a_rows, a_row, B, scale_b, bias, C, &a, &go);
    return st != FT_OK || !go ? st : FT_ERR_UNSUPPORTED;
}
ft_status ft_expert_workspace(const ft_expert_desc *desc, uint32_t tokens, uint64_t *bytes) { return ftk::expert_workspace(desc, tokens, bytes); }
ft_status ft_expert_sort(const ft_expert_desc *desc, uint32_t tokens, const int32_t *expert_of, int32_t *offsets, int32_t *row_token, int32_t *row_of, void *workspace,
                         uint64_t workspace_bytes, void *) {
    const ft_status st = ftk::sort_check(desc, tokens, expert_of, offsets, row_token, row_of, workspace, workspace_bytes);
    return st != FT_OK ? st : FT_ERR_UNSUPPORTED;
}
static ft_status move_stub(const ft_expert_desc *desc, uint32_t tokens, const void *src, const void *other, bool need_other, const int32_t *row_of, const float *weights, void *dst,
                           float *dweights) {
    ftk::MoveArgs a = {};
    a.src = src; a.other = other; a.dst = dst; a.row_of = row_of; a.weights = weights; a.dweights = dweights;
    bool go;
    const ft_status st = ftk::move_check(desc, tokens, need_other, &a, &go);
    return st != FT_OK || !go ? st : FT_ERR_UNSUPPORTED;
}
ft_status ft_expert_gather(const ft_expert_desc *desc, uint32_t tokens, const void *X, const int32_t *row_of, void *Y, void *) {
    return move_stub(desc, tokens, X, nullptr, false, row_of, nullptr, Y, nullptr);
}
ft_status ft_expert_combine(const ft_expert_desc *desc, uint32_t tokens, const void *Y, const int32_t *row_of, const float *weights, void *Out, void *) {
    return move_stub(desc, tokens, Y, nullptr, false, row_of, weights, Out, nullptr);
}
ft_status ft_expert_combine_grad(const ft_expert_desc *desc, uint32_t tokens, const void *dOut, const void *Y, const int32_t *row_of, const float *weights, void *dY,
                                 float *dweights, void *) {
    return move_stub(desc, tokens, dOut, Y, dweights != nullptr, row_of, weights, dY, dweights);
}
}
