// Host side of the norms behind and in front of a block: every check runs before anything is enqueued.
#include "sbp_buffers.h"

using namespace sbp;

namespace {

constexpr int MAX_K = 32;   // as layer normalisation

int32_t check_activation(const sbp_tensor_t* t, sbp_t s, int32_t k, const sbp_tensor_t* like) {
    const int32_t st = check_block8(t, nullptr, s, k, false);
    if (st != SBP_OK) return st;
    if (t->rows != like->rows || t->cols != like->cols) return SBP_ERR_SHAPE;
    return t->trans ? SBP_ERR_UNSUPPORTED : SBP_OK;
}

// A norm's weights and statistics.  grad: the statistics are inputs, and the weights' gradients count.
int32_t check_norm_of(const sbp_norm_t* m, const sbp_tensor_t* x, sbp_t sx, int32_t k, bool grad) {
    if (!m) return SBP_OK;
    if (m->kind != SBP_NORM_LAYER && m->kind != SBP_NORM_RMS) return SBP_ERR_UNSUPPORTED;
    const bool layer = m->kind == SBP_NORM_LAYER;
    if (!(m->eps >= 0.0f)) return SBP_ERR_UNSUPPORTED;
    if (!layer && (m->beta || m->mean || (grad && m->dbeta))) return SBP_ERR_UNSUPPORTED;   // it has none
    int32_t st;
    if (m->gamma && (st = check_column(m->gamma, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if (m->beta && (st = check_column(m->beta, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if (grad ? !m->rstd || (layer && !m->mean) : layer && !m->mean != !m->rstd) return SBP_ERR_NULL;
    if (!grad && m->rstd && x->rows != 0 && x->cols == 0) return SBP_ERR_SHAPE;   // a row of nothing has none
    if (m->mean && (st = check_column(m->mean, x->rows, sx, k, false)) != SBP_OK) return st;
    if (m->rstd && (st = check_column(m->rstd, x->rows, sx, k, false)) != SBP_OK) return st;
    if (grad && m->dgamma && (st = check_column(m->dgamma, x->cols, SBP_B, k, false)) != SBP_OK) return st;
    if (grad && m->dbeta && (st = check_column(m->dbeta, x->cols, SBP_B, k, false)) != SBP_OK) return st;
    return SBP_OK;
}

// One type for all weights that there are.
int32_t weights_type(const sbp_norm_t* post, const sbp_tensor_t* gate, const sbp_norm_t* pre, int32_t& dtype) {
    const sbp_tensor_t* const all[5] = {gate, post ? post->gamma : nullptr, post ? post->beta : nullptr, pre ? pre->gamma : nullptr, pre ? pre->beta : nullptr};
    dtype = -1;
    for (const sbp_tensor_t* t : all) {
        if (!t) continue;
        if (dtype >= 0 && t->dtype != dtype) return SBP_ERR_DTYPE;
        dtype = t->dtype;
    }
    return SBP_OK;
}

int32_t check_shape(const sbp_tensor_t* x, sbp_t sx, int32_t k) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    const int32_t st = check_whole(sx);
    if (st != SBP_OK) return st;
    if (sx == SBP_S(1) || k > MAX_K) return SBP_ERR_UNSUPPORTED;   // the statistics of a row need all of it
    if (!x) return SBP_ERR_NULL;
    if (x->trans || x->cols > NORM_MAX_COLS) return SBP_ERR_UNSUPPORTED;
    return SBP_OK;
}

int32_t flags_of(const sbp_norm_t* post, const sbp_norm_t* pre, int32_t weights) {
    return (post ? RN_POST | (post->kind == SBP_NORM_LAYER ? RN_POST_LAYER : 0) : 0) | (pre ? RN_PRE | (pre->kind == SBP_NORM_LAYER ? RN_PRE_LAYER : 0) : 0) |
           (weights == SBP_BF16 ? RN_BF16_WEIGHTS : 0);
}
const void* at(const sbp_tensor_t* t, int32_t i) { return t ? t->shard[i] : nullptr; }
float* out_at(const sbp_tensor_t* t, int32_t i) { return t ? static_cast<float*>(t->shard[i]) : nullptr; }
void add_if(Buffers& b, bool out, const sbp_tensor_t* t, sbp_t s, int32_t k) {
    if (t) b.add(out, t, s, k);
}

}  // namespace

extern "C" {

int32_t sbp_residual_norm(const sbp_tensor_t* x, sbp_t sx, const sbp_norm_t* post, const sbp_tensor_t* gate, const sbp_tensor_t* r, float alpha, const sbp_tensor_t* h,
                          const sbp_norm_t* pre, const sbp_tensor_t* y, const sbp_scales_t* y_scales, int32_t k, void* stream) {
    int32_t st, weights;
    if ((st = check_shape(x, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(x, nullptr, sx, k, false)) != SBP_OK) return st;
    if ((st = check_activation(r, sx, k, x)) != SBP_OK) return st;
    if ((st = check_activation(h, sx, k, x)) != SBP_OK) return st;
    if (r->dtype != h->dtype) return SBP_ERR_DTYPE;
    if (!pre != !y) return SBP_ERR_NULL;
    if (!y && y_scales) return SBP_ERR_NULL;
    if (y) {
        if ((st = check_block8(y, y_scales, sx, k)) != SBP_OK) return st;
        if (y->rows != x->rows || y->cols != x->cols) return SBP_ERR_SHAPE;
        if (y->trans) return SBP_ERR_UNSUPPORTED;
    }
    if (gate && (st = check_column(gate, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if ((st = check_norm_of(post, x, sx, k, false)) != SBP_OK) return st;
    if ((st = check_norm_of(pre, x, sx, k, false)) != SBP_OK) return st;
    if ((st = weights_type(post, gate, pre, weights)) != SBP_OK) return st;
    Buffers b;
    b.add(false, x, sx, k);
    b.add(false, r, sx, k);
    add_if(b, false, gate, SBP_B, k);
    b.add(true, h, sx, k);
    if (y) b.add(true, y, y_scales, sx, k);
    for (const sbp_norm_t* m : {post, pre}) {
        if (!m) continue;
        add_if(b, false, m->gamma, SBP_B, k);
        add_if(b, false, m->beta, SBP_B, k);
        add_if(b, true, m->mean, sx, k);
        add_if(b, true, m->rstd, sx, k);
    }
    if ((st = b.check()) != SBP_OK) return st;
    if (x->rows == 0 || x->cols == 0) return SBP_OK;
    return each_group<RESNORM_SHARDS>(k, [&](auto shards, int32_t first, int32_t n) {
        ResNormPlan<shards()> plan{};
        plan.cols = (int32_t)x->cols;
        plan.flags = flags_of(post, pre, weights);
        plan.alpha = alpha;
        plan.eps1 = post ? post->eps : 0.0f;
        plan.eps2 = pre ? pre->eps : 0.0f;
        for (int32_t j = 0; j < n; ++j) {
            const int32_t i = first + j;
            const Local l = local_of(x->rows, x->cols, sx, k, i);
            ResNormShard& s = plan.s[j];
            s = {x->shard[i], r->shard[i], h->shard[i], y ? y->shard[i] : nullptr, y && is_f8(y->dtype) ? y_scales->shard[i] : nullptr,
                 post ? out_at(post->mean, i) : nullptr, post ? out_at(post->rstd, i) : nullptr, pre ? out_at(pre->mean, i) : nullptr, pre ? out_at(pre->rstd, i) : nullptr,
                 at(gate, i), post ? at(post->gamma, i) : nullptr, post ? at(post->beta, i) : nullptr, pre ? at(pre->gamma, i) : nullptr, pre ? at(pre->beta, i) : nullptr,
                 (int32_t)l.rows, (int32_t)pitch_of(x, l), (int32_t)pitch_of(r, l), (int32_t)pitch_of(h, l), y ? (int32_t)pitch_of(y, l) : 0,
                 y && is_f8(y->dtype) ? (int32_t)scale_pitch(y_scales, l.cols) : 0};
        }
        return launch_residual_norm(plan, n, x->dtype, r->dtype, y ? y->dtype : SBP_BF16, static_cast<hipStream_t>(stream));
    });
}

int32_t sbp_residual_norm_grad_workspace(int64_t rows, int64_t cols, sbp_t sx, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    if (rows < 0 || cols < 0) return SBP_ERR_SHAPE;
    sbp_tensor_t x{};
    x.rows = rows;
    x.cols = cols;
    const int32_t st = check_shape(&x, sx, k);
    if (st != SBP_OK) return st;
    if (rows > INT32_MAX - 256) return SBP_ERR_UNSUPPORTED;
    *bytes = 0;
    for (int32_t i = 0; i < k; ++i) *bytes += residual_norm_grad_blocks(local_of(rows, cols, sx, k, i).rows, cols, k) * 4 * cols * 4;
    return SBP_OK;
}

int32_t sbp_residual_norm_grad(const sbp_tensor_t* x, sbp_t sx, const sbp_norm_t* post, const sbp_tensor_t* gate, float alpha, const sbp_tensor_t* h, const sbp_norm_t* pre,
                               const sbp_tensor_t* dh, const sbp_tensor_t* dy, const sbp_tensor_t* dx, const sbp_tensor_t* dr, const sbp_tensor_t* dgate, void* workspace,
                               int64_t workspace_bytes, int32_t k, void* stream) {
    int32_t st, weights;
    if ((st = check_shape(x, sx, k)) != SBP_OK) return st;
    if ((st = check_block8(x, nullptr, sx, k, false)) != SBP_OK) return st;
    if (!pre != !h || !pre != !dy || (!pre && !dh)) return SBP_ERR_NULL;
    if (h && (st = check_activation(h, sx, k, x)) != SBP_OK) return st;
    if (dy && (st = check_activation(dy, sx, k, x)) != SBP_OK) return st;
    if (dh && (st = check_activation(dh, sx, k, x)) != SBP_OK) return st;
    if ((st = check_activation(dx, sx, k, x)) != SBP_OK) return st;
    if ((st = check_activation(dr, sx, k, x)) != SBP_OK) return st;
    if (dx->dtype != x->dtype || (h && h->dtype != dr->dtype) || (dh && dh->dtype != dr->dtype)) return SBP_ERR_DTYPE;
    if (gate && (st = check_column(gate, x->cols, SBP_B, k, true)) != SBP_OK) return st;
    if (dgate && (st = check_column(dgate, x->cols, SBP_B, k, false)) != SBP_OK) return st;
    if ((st = check_norm_of(post, x, sx, k, true)) != SBP_OK) return st;
    if ((st = check_norm_of(pre, x, sx, k, true)) != SBP_OK) return st;
    if ((st = weights_type(post, gate, pre, weights)) != SBP_OK) return st;
    const bool sums = dgate || (post && (post->dgamma || post->dbeta)) || (pre && (pre->dgamma || pre->dbeta));
    int64_t room = 0;
    if (sums && (st = sbp_residual_norm_grad_workspace(x->rows, x->cols, sx, k, &room)) != SBP_OK) return st;
    if (room) {
        if (!workspace) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 15u) return SBP_ERR_ALIGN;
        if (workspace_bytes < room) return SBP_ERR_SHAPE;
    }
    Buffers b;
    b.add(false, x, sx, k);
    add_if(b, false, gate, SBP_B, k);
    add_if(b, false, h, sx, k);
    add_if(b, false, dh, sx, k);
    add_if(b, false, dy, sx, k);
    b.add(true, dx, sx, k);
    b.add(true, dr, sx, k);
    add_if(b, true, dgate, SBP_B, k);
    for (const sbp_norm_t* m : {post, pre}) {
        if (!m) continue;
        add_if(b, false, m->gamma, SBP_B, k);
        add_if(b, false, m->beta, SBP_B, k);
        add_if(b, false, m->mean, sx, k);
        add_if(b, false, m->rstd, sx, k);
        add_if(b, true, m->dgamma, SBP_B, k);
        add_if(b, true, m->dbeta, SBP_B, k);
    }
    b.add(true, workspace, 1, room, room, 1);
    if ((st = b.check()) != SBP_OK) return st;
    if (x->cols == 0 || (x->rows == 0 && !sums)) return SBP_OK;
    float* const part = static_cast<float*>(workspace);
    int64_t used = 0;
    float* parts[MAX_K] = {};
    int32_t blocks[MAX_K];
    for (int32_t i = 0; i < k; ++i) {
        blocks[i] = residual_norm_grad_blocks(local_of(x->rows, x->cols, sx, k, i).rows, x->cols, k);
        if (sums) parts[i] = part + used;
        used += (int64_t)blocks[i] * 4 * x->cols;
    }
    const int32_t flags = flags_of(post, pre, weights) | (dh ? RN_DH : 0);
    st = each_group<RESNORM_SHARDS>(k, [&](auto shards, int32_t first, int32_t n) {
        ResNormGradPlan<shards()> plan{};
        plan.cols = (int32_t)x->cols;
        plan.flags = flags;
        plan.alpha = alpha;
        for (int32_t j = 0; j < n; ++j) {
            const int32_t i = first + j;
            const Local l = local_of(x->rows, x->cols, sx, k, i);
            plan.s[j] = {x->shard[i], at(h, i), at(dh, i), at(dy, i), dx->shard[i], dr->shard[i],
                         post ? out_at(post->mean, i) : nullptr, post ? out_at(post->rstd, i) : nullptr, pre ? out_at(pre->mean, i) : nullptr, pre ? out_at(pre->rstd, i) : nullptr,
                         at(gate, i), post ? at(post->gamma, i) : nullptr, pre ? at(pre->gamma, i) : nullptr, parts[i],
                         (int32_t)l.rows, (int32_t)pitch_of(x, l), h ? (int32_t)pitch_of(h, l) : 0, dh ? (int32_t)pitch_of(dh, l) : 0, dy ? (int32_t)pitch_of(dy, l) : 0,
                         (int32_t)pitch_of(dx, l), (int32_t)pitch_of(dr, l), blocks[i]};
        }
        return launch_residual_norm_grad(plan, n, x->dtype, dr->dtype, dy ? dy->dtype : SBP_BF16, static_cast<hipStream_t>(stream));
    });
    if (st != SBP_OK || !sums) return st;
    return each_group<RESNORM_SHARDS>(k, [&](auto shards, int32_t first, int32_t n) {
        ResNormJoin<shards()> join{};
        join.cols = (int32_t)x->cols;
        join.flags = flags;
        for (int32_t j = 0; j < n; ++j) {
            const int32_t i = first + j;
            join.s[j] = {parts[i], at(gate, i), post ? at(post->gamma, i) : nullptr, post ? at(post->beta, i) : nullptr, out_at(dgate, i),
                         post ? out_at(post->dgamma, i) : nullptr, post ? out_at(post->dbeta, i) : nullptr, pre ? out_at(pre->dgamma, i) : nullptr,
                         pre ? out_at(pre->dbeta, i) : nullptr, blocks[i]};
        }
        return launch_residual_norm_join(join, n, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
