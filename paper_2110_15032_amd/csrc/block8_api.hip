// Host side of the operators on 8-bit tensors and of layer normalisation: every check runs before anything is enqueued.
#include "sbp_buffers.h"

using namespace sbp;

extern "C" {

int32_t sbp_quantize(const sbp_tensor_t* x, sbp_t sx, const sbp_tensor_t* q, const sbp_scales_t* q_scales, int32_t k, void* stream, int32_t epilogue) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    int32_t st;
    if ((st = check_whole(sx)) != SBP_OK) return st;
    if ((st = check_block8(x, nullptr, sx, k, false)) != SBP_OK) return st;
    if (q && !is_f8(q->dtype)) return SBP_ERR_DTYPE;
    if ((st = check_block8(q, q_scales, sx, k)) != SBP_OK) return st;
    if (x->rows != q->rows || x->cols != q->cols) return SBP_ERR_SHAPE;
    if (x->trans) return SBP_ERR_UNSUPPORTED;
    if (epilogue != SBP_EPI_NONE && epilogue != SBP_EPI_GELU) return SBP_ERR_UNSUPPORTED;
    Buffers b;
    b.add(false, x, sx, k);
    b.add(true, q, q_scales, sx, k);
    if ((st = b.check()) != SBP_OK) return st;
    if (x->rows == 0 || x->cols == 0) return SBP_OK;
    Block8Plan plan{};
    plan.k = k;
    plan.f8 = q->dtype;
    plan.dtype = x->dtype;
    plan.trans = q->trans;
    plan.gelu = epilogue == SBP_EPI_GELU;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(x->rows, x->cols, sx, k, i);
        plan.s[i] = {x->shard[i], q_scales->shard[i], nullptr, q->shard[i], (int32_t)l.rows, (int32_t)l.cols, (int32_t)pitch_of(x, l),
                     (int32_t)scale_pitch(q_scales, stored_cols(q, l)), 0, (int32_t)pitch_of(q, l)};
    }
    return launch_quantize(plan, static_cast<hipStream_t>(stream));
}

int32_t sbp_dequantize(const sbp_tensor_t* q, const sbp_scales_t* q_scales, sbp_t sq, const sbp_tensor_t* x, int32_t k, void* stream, int32_t epilogue) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    int32_t st;
    if ((st = check_whole(sq)) != SBP_OK) return st;
    if (q && !is_f8(q->dtype)) return SBP_ERR_DTYPE;
    if ((st = check_block8(q, q_scales, sq, k)) != SBP_OK) return st;
    if ((st = check_block8(x, nullptr, sq, k, false)) != SBP_OK) return st;
    if (x->rows != q->rows || x->cols != q->cols) return SBP_ERR_SHAPE;
    if (x->trans) return SBP_ERR_UNSUPPORTED;
    if (epilogue != SBP_EPI_NONE && epilogue != SBP_EPI_GELU) return SBP_ERR_UNSUPPORTED;
    Buffers b;
    b.add(false, q, q_scales, sq, k);
    b.add(true, x, sq, k);
    if ((st = b.check()) != SBP_OK) return st;
    if (x->rows == 0 || x->cols == 0) return SBP_OK;
    Block8Plan plan{};
    plan.k = k;
    plan.f8 = q->dtype;
    plan.dtype = x->dtype;
    plan.trans = q->trans;
    plan.gelu = epilogue == SBP_EPI_GELU;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(x->rows, x->cols, sq, k, i);
        plan.s[i] = {q->shard[i], q_scales->shard[i], nullptr, x->shard[i], (int32_t)l.rows, (int32_t)l.cols, (int32_t)pitch_of(q, l),
                     (int32_t)scale_pitch(q_scales, stored_cols(q, l)), 0, (int32_t)pitch_of(x, l)};
    }
    return launch_dequantize(plan, static_cast<hipStream_t>(stream));
}

int32_t sbp_gelu_grad(const sbp_tensor_t* a, const sbp_scales_t* a_scales, sbp_t sa, const sbp_tensor_t* dh, const sbp_tensor_t* da, int32_t k, void* stream) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    int32_t st;
    if ((st = check_whole(sa)) != SBP_OK) return st;
    if ((st = check_block8(a, a_scales, sa, k)) != SBP_OK) return st;
    if ((st = check_block8(dh, nullptr, sa, k, false)) != SBP_OK) return st;
    if ((st = check_block8(da, nullptr, sa, k, false)) != SBP_OK) return st;
    if (a->rows != dh->rows || a->cols != dh->cols || a->rows != da->rows || a->cols != da->cols) return SBP_ERR_SHAPE;
    if (dh->dtype != da->dtype) return SBP_ERR_DTYPE;
    if (a->trans || dh->trans || da->trans) return SBP_ERR_UNSUPPORTED;
    Buffers b;
    b.add(false, a, a_scales, sa, k);
    b.add(false, dh, sa, k);
    b.add(true, da, sa, k);
    if ((st = b.check()) != SBP_OK) return st;
    if (a->rows == 0 || a->cols == 0) return SBP_OK;
    Block8Plan plan{};
    plan.k = k;
    plan.f8 = a->dtype;
    plan.dtype = da->dtype;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(a->rows, a->cols, sa, k, i);
        plan.s[i] = {a->shard[i], is_f8(a->dtype) ? a_scales->shard[i] : nullptr, dh->shard[i], da->shard[i], (int32_t)l.rows, (int32_t)l.cols,
                     (int32_t)pitch_of(a, l), is_f8(a->dtype) ? (int32_t)scale_pitch(a_scales, l.cols) : 0, (int32_t)pitch_of(dh, l), (int32_t)pitch_of(da, l)};
    }
    return launch_gelu_grad(plan, static_cast<hipStream_t>(stream));
}

// what sbp_layernorm and its gradient have in common
static int32_t check_norm(const sbp_tensor_t* x, sbp_t sx, int32_t k) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    const int32_t st = check_whole(sx);
    if (st != SBP_OK) return st;
    if (sx == SBP_S(1) || k > NORM_MAX_K) return SBP_ERR_UNSUPPORTED;   // the statistics of a row need all of it
    if (!x) return SBP_ERR_NULL;
    if (x->trans || x->cols > NORM_MAX_COLS) return SBP_ERR_UNSUPPORTED;
    return SBP_OK;
}

int32_t sbp_layernorm(const sbp_tensor_t* x, sbp_t sx, const sbp_tensor_t* gamma, const sbp_tensor_t* beta, float eps, const sbp_tensor_t* y,
                      const sbp_scales_t* y_scales, const sbp_tensor_t* mean, const sbp_tensor_t* rstd, int32_t k, void* stream) {
    int32_t st;
    if ((st = check_norm(x, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(x, nullptr, sx, k, false)) != SBP_OK) return st;
    if ((st = check_block8(y, y_scales, sx, k)) != SBP_OK) return st;
    if (x->rows != y->rows || x->cols != y->cols) return SBP_ERR_SHAPE;
    if (y->trans) return SBP_ERR_UNSUPPORTED;
    if (!(eps >= 0.0f)) return SBP_ERR_UNSUPPORTED;
    if (gamma && (st = check_column(gamma, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if (beta && (st = check_column(beta, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if (gamma && beta && gamma->dtype != beta->dtype) return SBP_ERR_DTYPE;
    if (!mean != !rstd) return SBP_ERR_NULL;
    if (mean && x->rows != 0 && x->cols == 0) return SBP_ERR_SHAPE;   // a row of nothing has none
    if (mean && (st = check_column(mean, x->rows, sx, k, false)) != SBP_OK) return st;
    if (rstd && (st = check_column(rstd, x->rows, sx, k, false)) != SBP_OK) return st;
    Buffers b;
    b.add(false, x, sx, k);
    if (gamma) b.add(false, gamma, SBP_B, k);
    if (beta) b.add(false, beta, SBP_B, k);
    b.add(true, y, y_scales, sx, k);
    if (mean) b.add(true, mean, sx, k);
    if (rstd) b.add(true, rstd, sx, k);
    if ((st = b.check()) != SBP_OK) return st;
    if (x->rows == 0 || x->cols == 0) return SBP_OK;
    NormPlan plan{};
    plan.k = k;
    plan.cols = (int32_t)x->cols;
    plan.x_dtype = x->dtype;
    plan.y_dtype = y->dtype;
    plan.w_dtype = gamma ? gamma->dtype : beta ? beta->dtype : SBP_F32;
    plan.eps = eps;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(x->rows, x->cols, sx, k, i);
        plan.s[i] = {x->shard[i], gamma ? gamma->shard[i] : nullptr, beta ? beta->shard[i] : nullptr, y->shard[i], y_scales ? y_scales->shard[i] : nullptr,
                     mean ? static_cast<float*>(mean->shard[i]) : nullptr, rstd ? static_cast<float*>(rstd->shard[i]) : nullptr, (int32_t)l.rows,
                     (int32_t)pitch_of(x, l), (int32_t)pitch_of(y, l), y_scales ? (int32_t)scale_pitch(y_scales, l.cols) : 0};
    }
    return launch_norm(plan, static_cast<hipStream_t>(stream));
}

int32_t sbp_layernorm_grad_workspace(int64_t rows, int64_t cols, sbp_t sx, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    if (rows < 0 || cols < 0) return SBP_ERR_SHAPE;
    sbp_tensor_t x{};
    x.rows = rows;
    x.cols = cols;
    const int32_t st = check_norm(&x, sx, k);
    if (st != SBP_OK) return st;
    if (rows > INT32_MAX) return SBP_ERR_UNSUPPORTED;
    *bytes = 0;
    for (int32_t i = 0; i < k; ++i) {
        const int64_t blocks = norm_grad_blocks(local_of(rows, cols, sx, k, i).rows, cols, k);
        if (blocks > 1) *bytes += blocks * 2 * cols * 4;
    }
    return SBP_OK;
}

int32_t sbp_layernorm_grad(const sbp_tensor_t* x, const sbp_scales_t* x_scales, sbp_t sx, const sbp_tensor_t* gamma, const sbp_tensor_t* mean,
                           const sbp_tensor_t* rstd, const sbp_tensor_t* dy, const sbp_tensor_t* dx, const sbp_tensor_t* dgamma, const sbp_tensor_t* dbeta,
                           void* workspace, int64_t workspace_bytes, int32_t k, void* stream) {
    int32_t st;
    if ((st = check_norm(x, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(x, x_scales, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(dy, nullptr, sx, k, false)) != SBP_OK) return st;
    if ((st = check_block8(dx, nullptr, sx, k, false)) != SBP_OK) return st;
    if (x->rows != dy->rows || x->cols != dy->cols || x->rows != dx->rows || x->cols != dx->cols) return SBP_ERR_SHAPE;
    if (dy->dtype != dx->dtype) return SBP_ERR_DTYPE;
    if (dy->trans || dx->trans) return SBP_ERR_UNSUPPORTED;
    if (gamma && (st = check_column(gamma, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if ((st = check_column(mean, x->rows, sx, k, false)) != SBP_OK) return st;
    if ((st = check_column(rstd, x->rows, sx, k, false)) != SBP_OK) return st;
    if (!dgamma != !dbeta) return SBP_ERR_NULL;
    // every device has its own sums: P(sum) of an S(0) activation, B of a B one, whole vectors either way
    if (dgamma && (st = check_column(dgamma, x->cols, SBP_B, k, false)) != SBP_OK) return st;
    if (dbeta && (st = check_column(dbeta, x->cols, SBP_B, k, false)) != SBP_OK) return st;
    int64_t room = 0;
    if (dgamma && (st = sbp_layernorm_grad_workspace(x->rows, x->cols, sx, k, &room)) != SBP_OK) return st;
    if (room) {
        if (!workspace) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 15u) return SBP_ERR_ALIGN;
        if (workspace_bytes < room) return SBP_ERR_SHAPE;
    }
    Buffers b;
    b.add(false, x, x_scales, sx, k);
    if (gamma) b.add(false, gamma, SBP_B, k);
    b.add(false, mean, sx, k);
    b.add(false, rstd, sx, k);
    b.add(false, dy, sx, k);
    b.add(true, dx, sx, k);
    if (dgamma) {
        b.add(true, dgamma, SBP_B, k);
        b.add(true, dbeta, SBP_B, k);
    }
    b.add(true, workspace, 1, room, room, 1);
    if ((st = b.check()) != SBP_OK) return st;
    if (x->cols == 0 || (x->rows == 0 && !dgamma)) return SBP_OK;
    NormGradPlan plan{};
    plan.k = k;
    plan.cols = (int32_t)x->cols;
    plan.x_dtype = x->dtype;
    plan.dy_dtype = dy->dtype;
    plan.w_dtype = gamma ? gamma->dtype : SBP_F32;
    float* part = static_cast<float*>(workspace);
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(x->rows, x->cols, sx, k, i);
        const int32_t blocks = norm_grad_blocks(l.rows, l.cols, k);
        plan.s[i] = {x->shard[i], x_scales ? x_scales->shard[i] : nullptr, gamma ? gamma->shard[i] : nullptr, static_cast<const float*>(mean->shard[i]),
                     static_cast<const float*>(rstd->shard[i]), dy->shard[i], dx->shard[i], dgamma ? static_cast<float*>(dgamma->shard[i]) : nullptr,
                     dbeta ? static_cast<float*>(dbeta->shard[i]) : nullptr, part, (int32_t)l.rows, (int32_t)pitch_of(x, l),
                     x_scales ? (int32_t)scale_pitch(x_scales, l.cols) : 0, (int32_t)pitch_of(dy, l), (int32_t)pitch_of(dx, l), blocks};
        if (dgamma && blocks > 1) part += (int64_t)blocks * 2 * l.cols;
    }
    return launch_norm_grad(plan, static_cast<hipStream_t>(stream));
}

int32_t sbp_matmul_f8(const sbp_tensor_t* x, const sbp_scales_t* x_scales, sbp_t sx, const sbp_tensor_t* w, const sbp_scales_t* w_scales, sbp_t sw,
                      const sbp_tensor_t* y, sbp_t sy, int32_t k, void* stream, int32_t epilogue) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    if (!x || !w || !y) return SBP_ERR_NULL;
    if (!is_sbp(sx) || !is_sbp(sw)) return SBP_ERR_AXIS;
    sbp_t deduced;
    int32_t st = sbp_infer_matmul(sx, sw, &deduced);
    if (st != SBP_OK) return st;
    if (sy == SBP_AUTO) sy = deduced;
    if (!is_sbp(sy)) return SBP_ERR_AXIS;
    if (sy != deduced) return SBP_ERR_SIGNATURE;
    if (!is_f8(x->dtype) || !is_f8(w->dtype)) return SBP_ERR_DTYPE;
    if (is_partial(sx) || is_partial(sw)) return SBP_ERR_DTYPE;   // an un-reduced partial is fp32
    if (k > GEMM_F8_MAX_K) return SBP_ERR_UNSUPPORTED;
    if ((st = check_block8(x, x_scales, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(w, w_scales, sw, k)) != SBP_OK) return st;
    if ((st = check_block8(y, nullptr, sy, k, false)) != SBP_OK) return st;
    if (x->cols != w->rows || y->rows != x->rows || y->cols != w->cols) return SBP_ERR_SHAPE;
    if (is_partial(sy) && y->dtype != SBP_F32) return SBP_ERR_DTYPE;
    if (x->trans != 0 || w->trans != 1 || y->trans != 0) return SBP_ERR_UNSUPPORTED;   // blocks run along the reduction
    if (epilogue != SBP_EPI_NONE && epilogue != SBP_EPI_GELU) return SBP_ERR_UNSUPPORTED;
    if (epilogue == SBP_EPI_GELU && is_partial(sy)) return SBP_ERR_SIGNATURE;
    Buffers b;
    b.add(false, x, x_scales, sx, k);
    b.add(false, w, w_scales, sw, k);
    b.add(true, y, sy, k);
    if ((st = b.check()) != SBP_OK) return st;
    GemmF8Plan plan{};
    plan.groups = k;
    plan.a_dtype = x->dtype;
    plan.b_dtype = w->dtype;
    plan.out_dtype = y->dtype;
    plan.epilogue = epilogue;
    for (int32_t i = 0; i < k; ++i) {
        const Local lx = local_of(x->rows, x->cols, sx, k, i), lw = local_of(w->rows, w->cols, sw, k, i), ly = local_of(y->rows, y->cols, sy, k, i);
        if (lx.cols != lw.rows || ly.rows != lx.rows || ly.cols != lw.cols) return SBP_ERR_SHAPE;
        GemmF8Shard& g = plan.s[i];
        g.a = static_cast<const uint8_t*>(x->shard[i]);
        g.a_scales = static_cast<const uint8_t*>(x_scales->shard[i]);
        g.b = static_cast<const uint8_t*>(w->shard[i]);
        g.b_scales = static_cast<const uint8_t*>(w_scales->shard[i]);
        g.c = y->shard[i];
        g.m = (int32_t)ly.rows;
        g.n = (int32_t)ly.cols;
        g.kk = (int32_t)lx.cols;
        g.lda = (int32_t)pitch_of(x, lx);
        g.ldas = (int32_t)scale_pitch(x_scales, lx.cols);
        g.ldb = (int32_t)pitch_of(w, lw);
        g.ldbs = (int32_t)scale_pitch(w_scales, lw.rows);
        g.ldc = (int32_t)pitch_of(y, ly);
    }
    return launch_gemm_f8(plan, static_cast<hipStream_t>(stream));
}

}  // extern "C"
