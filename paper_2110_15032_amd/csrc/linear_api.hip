// Host side of the product with bias, activation and residual, and of its epilogue's gradient: every check runs before anything is enqueued.
#include "sbp_buffers.h"

using namespace sbp;

namespace {

// where a vector over the columns of an activation lies
sbp_t along_columns(sbp_t s) { return s == SBP_S(1) ? SBP_S(0) : SBP_B; }

int32_t check_like(const sbp_tensor_t* t, sbp_t s, int32_t k, const sbp_tensor_t* y) {
    const int32_t st = check_block8(t, nullptr, s, k, false);
    if (st != SBP_OK) return st;
    if (t->rows != y->rows || t->cols != y->cols) return SBP_ERR_SHAPE;
    return t->trans ? SBP_ERR_UNSUPPORTED : SBP_OK;
}

}  // namespace

extern "C" {

int32_t sbp_linear(const sbp_tensor_t* x, sbp_t sx, const sbp_tensor_t* w, sbp_t sw, const sbp_tensor_t* bias, const sbp_tensor_t* residual, const sbp_tensor_t* pre,
                   const sbp_tensor_t* y, sbp_t sy, int32_t k, void* stream, int32_t epilogue) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    if (!x || !w || !y) return SBP_ERR_NULL;
    if (!is_sbp(sx) || !is_sbp(sw)) return SBP_ERR_AXIS;
    sbp_t deduced;
    int32_t st = sbp_infer_matmul(sx, sw, &deduced);
    if (st != SBP_OK) return st;
    if (sy == SBP_AUTO) sy = deduced;
    if (!is_sbp(sy)) return SBP_ERR_AXIS;
    if (sy != deduced || is_partial(sy)) return SBP_ERR_SIGNATURE;   // what follows the product is not linear, or would count k times
    if ((st = check_block8(x, nullptr, sx, k, false)) != SBP_OK) return st;
    if ((st = check_block8(w, nullptr, sw, k, false)) != SBP_OK) return st;
    if ((st = check_block8(y, nullptr, sy, k, false)) != SBP_OK) return st;
    if (x->dtype != w->dtype) return SBP_ERR_DTYPE;
    if (x->cols != w->rows || y->rows != x->rows || y->cols != w->cols) return SBP_ERR_SHAPE;
    if (y->trans) return SBP_ERR_UNSUPPORTED;
    if (bias && (st = check_column(bias, y->cols, along_columns(sy), k, true)) != SBP_OK) return st;
    if (residual && (st = check_like(residual, sy, k, y)) != SBP_OK) return st;
    if (pre && (st = check_like(pre, sy, k, y)) != SBP_OK) return st;
    if (epilogue != SBP_EPI_NONE && epilogue != SBP_EPI_GELU) return SBP_ERR_UNSUPPORTED;
    Buffers b;
    b.add(false, x, sx, k);
    b.add(false, w, sw, k);
    if (bias) b.add(false, bias, along_columns(sy), k);
    if (residual) b.add(false, residual, sy, k);
    if (pre) b.add(true, pre, sy, k);
    b.add(true, y, sy, k);
    if ((st = b.check()) != SBP_OK) return st;
    GemmBlockPlan plan{};
    plan.in_dtype = x->dtype;
    plan.a_kc = x->trans ? 0 : 1;
    plan.b_kc = w->trans ? 1 : 0;
    plan.flags = (bias && bias->dtype == SBP_BF16 ? GB_BIAS_BF16 : 0) | (residual && residual->dtype == SBP_BF16 ? GB_RESIDUAL_BF16 : 0) | (pre && pre->dtype == SBP_BF16 ? GB_PRE_BF16 : 0) |
                 (y->dtype == SBP_BF16 ? GB_OUT_BF16 : 0) | (epilogue == SBP_EPI_GELU ? y->dtype == SBP_BF16 ? GB_GELU : GB_GELU_ERF : 0);
    for (int32_t first = 0; first < k; first += GEMM_BLOCK_SHARDS) {
        plan.groups = std::min(k - first, GEMM_BLOCK_SHARDS);
        for (int32_t j = 0; j < plan.groups; ++j) {
            const int32_t i = first + j;
            const Local lx = local_of(x->rows, x->cols, sx, k, i), lw = local_of(w->rows, w->cols, sw, k, i), ly = local_of(y->rows, y->cols, sy, k, i);
            plan.s[j] = {x->shard[i], w->shard[i], y->shard[i], nullptr, (int32_t)ly.rows, (int32_t)ly.cols, (int32_t)lx.cols, (int32_t)pitch_of(x, lx), (int32_t)pitch_of(w, lw),
                         (int32_t)pitch_of(y, ly)};
            plan.x[j] = {bias ? bias->shard[i] : nullptr, residual ? residual->shard[i] : nullptr, pre ? pre->shard[i] : nullptr, residual ? (int32_t)pitch_of(residual, ly) : 0,
                         pre ? (int32_t)pitch_of(pre, ly) : 0};
        }
        if ((st = launch_linear(plan, static_cast<hipStream_t>(stream))) != SBP_OK) return st;
    }
    return SBP_OK;
}

int32_t sbp_linear_grad_workspace(int64_t rows, int64_t cols, sbp_t s, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    if (rows < 0 || cols < 0) return SBP_ERR_SHAPE;
    const int32_t st = check_whole(s);
    if (st != SBP_OK) return st;
    if (rows > INT32_MAX - 256 || cols > INT32_MAX - 256) return SBP_ERR_UNSUPPORTED;
    *bytes = 0;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(rows, cols, s, k, i);
        const int64_t blocks = linear_grad_blocks(l.rows, l.cols, k);
        if (blocks > 1) *bytes += (blocks * l.cols * 4 + 15) / 16 * 16;
    }
    return SBP_OK;
}

int32_t sbp_linear_grad(const sbp_tensor_t* dy, sbp_t s, const sbp_tensor_t* pre, const sbp_scales_t* pre_scales, const sbp_tensor_t* da, const sbp_tensor_t* dbias, void* workspace,
                        int64_t workspace_bytes, int32_t k, void* stream, int32_t epilogue) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    int32_t st;
    if ((st = check_whole(s)) != SBP_OK) return st;
    if ((st = check_block8(dy, nullptr, s, k, false)) != SBP_OK) return st;
    if (dy->trans) return SBP_ERR_UNSUPPORTED;
    if (epilogue != SBP_EPI_NONE && epilogue != SBP_EPI_GELU) return SBP_ERR_UNSUPPORTED;
    const bool gelu = epilogue == SBP_EPI_GELU;
    if (gelu) {
        if ((st = check_block8(pre, pre_scales, s, k)) != SBP_OK) return st;
        if (pre->rows != dy->rows || pre->cols != dy->cols) return SBP_ERR_SHAPE;
        if (pre->trans) return SBP_ERR_UNSUPPORTED;
        if ((st = check_like(da, s, k, dy)) != SBP_OK) return st;
        if (da->dtype != dy->dtype) return SBP_ERR_DTYPE;
    } else if (pre || pre_scales || da) {
        return SBP_ERR_UNSUPPORTED;   // the gradient in front of the bias is dy itself
    }
    const sbp_t sb = along_columns(s);
    if ((st = check_column(dbias, dy->cols, sb, k, false)) != SBP_OK) return st;
    int64_t room;
    if ((st = sbp_linear_grad_workspace(dy->rows, dy->cols, s, k, &room)) != SBP_OK) return st;
    if (room) {
        if (!workspace) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 15u) return SBP_ERR_ALIGN;
        if (workspace_bytes < room) return SBP_ERR_SHAPE;
    }
    Buffers b;
    b.add(false, dy, s, k);
    if (gelu) {
        b.add(false, pre, pre_scales, s, k);
        b.add(true, da, s, k);
    }
    b.add(true, dbias, sb, k);
    b.add(true, workspace, 1, room, room, 1);
    if ((st = b.check()) != SBP_OK) return st;
    if (dy->cols == 0) return SBP_OK;
    char* part = static_cast<char*>(workspace);
    return each_group<LINEAR_GRAD_SHARDS>(k, [&](auto shards, int32_t first, int32_t n) {
        LinearGradPlan<shards()> plan{};
        for (int32_t j = 0; j < n; ++j) {
            const int32_t i = first + j;
            const Local l = local_of(dy->rows, dy->cols, s, k, i);
            const int32_t blocks = linear_grad_blocks(l.rows, l.cols, k);
            const bool f8 = gelu && is_f8(pre->dtype);
            plan.s[j] = {dy->shard[i], gelu ? pre->shard[i] : nullptr, f8 ? pre_scales->shard[i] : nullptr, gelu ? da->shard[i] : nullptr, static_cast<float*>(dbias->shard[i]),
                         reinterpret_cast<float*>(part), (int32_t)l.rows, (int32_t)l.cols, (int32_t)pitch_of(dy, l), gelu ? (int32_t)pitch_of(pre, l) : 0,
                         f8 ? (int32_t)scale_pitch(pre_scales, l.cols) : 0, gelu ? (int32_t)pitch_of(da, l) : 0, blocks};
            if (blocks > 1) part += ((int64_t)blocks * l.cols * 4 + 15) / 16 * 16;
        }
        return launch_linear_grad(plan, n, dy->dtype, gelu ? pre->dtype : SBP_BF16, gelu, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
