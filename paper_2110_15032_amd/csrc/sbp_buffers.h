// Host side of the operators whose calls name many buffers: the buffers of a call, 8-bit tensors, activations and vectors.
#pragma once
#include <type_traits>

#include "sbp_check.h"

namespace sbp {

// The buffers of a call, in place (a C entry must not throw, and a vector may).
struct Buffers {
    static constexpr int MOST = 7 * SBP_MAX_K;   // inputs or outputs: up to 13 tensors of 32 devices, 6 of 64
    Span outs[MOST], ins[MOST];
    int n_out = 0, n_in = 0;

    void add(bool out, const void* p, int64_t rows, int64_t pitch, int64_t cols, int bytes) {
        if (rows * cols == 0) return;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        (out ? outs[n_out++] : ins[n_in++]) = {lo, lo + (uintptr_t)((rows - 1) * pitch + cols) * bytes};
    }
    void add(bool out, const sbp_tensor_t* t, sbp_t s, int32_t k) {
        for (int32_t i = 0; i < k; ++i) {
            const Local l = local_of(t->rows, t->cols, s, k, i);
            add(out, t->shard[i], t->trans ? l.cols : l.rows, pitch_of(t, l), t->trans ? l.rows : l.cols, elem_bytes(t->dtype));
        }
    }
    void add(bool out, const sbp_tensor_t* t, const sbp_scales_t* scales, sbp_t s, int32_t k);
    // outputs pairwise disjoint, and disjoint from every input
    int32_t check() {
        std::sort(outs, outs + n_out, [](const Span& a, const Span& b) { return a.lo < b.lo; });
        for (int i = 1; i < n_out; ++i)
            if (outs[i].lo < outs[i - 1].hi) return SBP_ERR_ALIAS;
        for (int i = 0; i < n_in; ++i)
            if (meets(ins[i])) return SBP_ERR_ALIAS;
        return SBP_OK;
    }
    // behind check(): does an output overlap it?
    bool meets(const Span& v) const {   // the first output that ends behind its start
        const Span* o = std::upper_bound(outs, outs + n_out, v.lo, [](uintptr_t lo, const Span& b) { return lo < b.hi; });
        return o != outs + n_out && o->lo < v.hi;
    }
};

inline int64_t stored_rows(const sbp_tensor_t* t, const Local& l) { return t->trans ? l.cols : l.rows; }
inline int64_t stored_cols(const sbp_tensor_t* t, const Local& l) { return t->trans ? l.rows : l.cols; }
inline int64_t scale_pitch(const sbp_scales_t* s, int64_t cols) { return s->ld ? s->ld : f8_blocks(cols); }

inline void Buffers::add(bool out, const sbp_tensor_t* t, const sbp_scales_t* scales, sbp_t s, int32_t k) {
    add(out, t, s, k);
    if (!is_f8(t->dtype)) return;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(t->rows, t->cols, s, k, i);
        const int64_t cols = stored_cols(t, l);
        add(out, scales->shard[i], stored_rows(t, l), scale_pitch(scales, cols), f8_blocks(cols), 1);
    }
}

// A tensor with its scales where it is in 8 bits, and none where it is not.
inline int32_t check_block8(const sbp_tensor_t* t, const sbp_scales_t* scales, sbp_t s, int32_t k, bool f8 = true) {
    if (!t) return SBP_ERR_NULL;
    // before anything is multiplied; kernels count up to the end of a tile of 256 behind a tensor's last row or column in 32 bits
    constexpr int64_t MOST = INT32_MAX - 256;
    if (t->rows > MOST || t->cols > MOST) return SBP_ERR_UNSUPPORTED;
    const int32_t st = check_tensor(t, s, k, true, f8);
    if (st != SBP_OK) return st;
    if (!is_f8(t->dtype)) return scales ? SBP_ERR_DTYPE : SBP_OK;
    if (!scales || !scales->shard) return SBP_ERR_NULL;
    if (scales->ld < 0) return SBP_ERR_SHAPE;
    if (scales->ld > INT32_MAX) return SBP_ERR_UNSUPPORTED;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(t->rows, t->cols, s, k, i);
        if (l.rows * l.cols == 0) continue;
        if (scales->ld && scales->ld < f8_blocks(stored_cols(t, l))) return SBP_ERR_SHAPE;
        if (!scales->shard[i]) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(scales->shard[i]) & 15u) return SBP_ERR_ALIGN;
    }
    return SBP_OK;
}

// an elementwise operator's or a norm's activation: whole values on every device
inline int32_t check_whole(sbp_t s) { return !is_sbp(s) ? SBP_ERR_AXIS : is_partial(s) ? SBP_ERR_SIGNATURE : SBP_OK; }

// a weight of `n` elements or a vector of `n` rows, a dense [n, 1]
inline int32_t check_column(const sbp_tensor_t* t, int64_t n, sbp_t s, int32_t k, bool bf16) {
    if (!t) return SBP_ERR_NULL;
    if (t->rows != n || t->cols != 1) return SBP_ERR_SHAPE;
    if (t->dtype != SBP_F32 && !(bf16 && t->dtype == SBP_BF16)) return SBP_ERR_DTYPE;
    if (t->trans) return SBP_ERR_UNSUPPORTED;
    return check_tensor(t, s, k);
}

// Devices dealt out over launches: one has a launch of its own size, more go MOST at a time, as an argument block costs about a microsecond a KB
// (a kernel that does nothing, us: 256 bytes 3.4, 1024 4.4, 4000 6.9).  F(integral constant: shards of the block, first shard, number of shards).
template <int MOST, typename F>
int32_t each_group(int32_t k, F&& f) {
    if (k == 1) return f(std::integral_constant<int, 1>{}, 0, 1);
    for (int32_t i = 0; i < k; i += MOST) {
        const int32_t st = f(std::integral_constant<int, MOST>{}, i, std::min(k - i, MOST));
        if (st != SBP_OK) return st;
    }
    return SBP_OK;
}

}  // namespace sbp
