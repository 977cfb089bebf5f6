// Host side of the C ABI, shared by its translation units: signatures, shard geometry, validation of descriptors and of
// overlapping buffers.
#pragma once
#include <algorithm>
#include <vector>

#include "sbp_internal.h"

namespace sbp {

inline bool is_sbp(sbp_t s) { return s == SBP_S(0) || s == SBP_S(1) || s == SBP_B || s == SBP_P_SUM || s == SBP_P_MAX; }
inline bool is_partial(sbp_t s) { return s == SBP_P_SUM || s == SBP_P_MAX; }
inline bool is_f8(int32_t dtype) { return dtype == SBP_F8E4M3 || dtype == SBP_F8E5M2; }
inline int elem_bytes(int32_t dtype) { return is_f8(dtype) ? 1 : dtype == SBP_BF16 ? 2 : 4; }

struct Local {
    int64_t rows, cols;
};
inline Local local_of(int64_t rows, int64_t cols, sbp_t s, int32_t k, int32_t i) {
    if (s == SBP_S(0)) return {split_len(rows, k, i), cols};
    if (s == SBP_S(1)) return {rows, split_len(cols, k, i)};
    return {rows, cols};
}

// row pitch of a stored local buffer in elements: the descriptor's, or the stored row length
inline int64_t pitch_of(const sbp_tensor_t* t, const Local& l) { return t->ld ? t->ld : (t->trans ? l.rows : l.cols); }

// with_ld: the entry point takes a row pitch (sbp_tensor_t::ld); the others want dense tensors.  f8: the 8-bit types are allowed as well
inline int32_t check_tensor(const sbp_tensor_t* t, sbp_t s, int32_t k, bool with_ld = false, bool f8 = false) {
    if (!t || !t->shard) return SBP_ERR_NULL;
    if (t->rows < 0 || t->cols < 0 || t->ld < 0) return SBP_ERR_SHAPE;
    if (t->dtype != SBP_F32 && t->dtype != SBP_BF16 && !(f8 && is_f8(t->dtype))) return SBP_ERR_DTYPE;
    if (t->trans != 0 && t->trans != 1) return SBP_ERR_SHAPE;
    if (!is_sbp(s)) return SBP_ERR_AXIS;
    if (t->ld && !with_ld) return SBP_ERR_UNSUPPORTED;
    if (t->ld > INT32_MAX) return SBP_ERR_UNSUPPORTED;
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(t->rows, t->cols, s, k, i);
        if (l.rows * l.cols == 0) continue;  // an empty local tensor needs no storage
        if (t->ld && (t->trans ? l.rows : l.cols) > t->ld) return SBP_ERR_SHAPE;
        if (!t->shard[i]) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(t->shard[i]) & 15u) return SBP_ERR_ALIGN;
    }
    return SBP_OK;
}

struct Span {
    uintptr_t lo, hi;
};
inline void spans_of(const sbp_tensor_t* t, sbp_t s, int32_t k, std::vector<Span>& v) {
    for (int32_t i = 0; i < k; ++i) {
        const Local l = local_of(t->rows, t->cols, s, k, i);
        if (l.rows * l.cols == 0) continue;
        // stored as nrow rows of ncol elements, pitch_of() apart: the span ends with the last row's last element
        const int64_t nrow = t->trans ? l.cols : l.rows, ncol = t->trans ? l.rows : l.cols;
        const uintptr_t bytes = (uintptr_t)((nrow - 1) * pitch_of(t, l) + ncol) * elem_bytes(t->dtype);
        const uintptr_t lo = reinterpret_cast<uintptr_t>(t->shard[i]);
        v.push_back({lo, lo + bytes});
    }
}
inline bool overlap(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }

// Two-dimensional signatures (Sec. 3.3): s[0] places the tensor on the k0 groups, s[1] each group's
// tensor on its k1 devices; device (a, b) is shard a * k1 + b.
inline Local local_of2(int64_t rows, int64_t cols, const sbp_t* s, int32_t k0, int32_t k1, int32_t a, int32_t b) {
    const Local n = local_of(rows, cols, s[0], k0, a);
    return local_of(n.rows, n.cols, s[1], k1, b);
}
inline int32_t check_grid(int32_t k0, int32_t k1) {
    if (k0 < 1 || k1 < 1 || (int64_t)k0 * k1 > SBP_MAX_K) return SBP_ERR_K;
    return SBP_OK;
}
inline int32_t check_tensor2(const sbp_tensor_t* t, const sbp_t* s, int32_t k0, int32_t k1, bool with_ld = false) {
    if (!t || !t->shard || !s) return SBP_ERR_NULL;
    if (t->rows < 0 || t->cols < 0 || t->ld < 0) return SBP_ERR_SHAPE;
    if (t->dtype != SBP_F32 && t->dtype != SBP_BF16) return SBP_ERR_DTYPE;
    if (t->trans != 0 || (t->ld != 0 && !with_ld) || t->ld > INT32_MAX) return SBP_ERR_UNSUPPORTED;
    if (!is_sbp(s[0]) || !is_sbp(s[1])) return SBP_ERR_AXIS;
    for (int32_t a = 0; a < k0; ++a)
        for (int32_t b = 0; b < k1; ++b) {
            const Local l = local_of2(t->rows, t->cols, s, k0, k1, a, b);
            if (l.rows * l.cols == 0) continue;
            if (t->ld && l.cols > t->ld) return SBP_ERR_SHAPE;
            void* p = t->shard[a * k1 + b];
            if (!p) return SBP_ERR_NULL;
            if (reinterpret_cast<uintptr_t>(p) & 15u) return SBP_ERR_ALIGN;
        }
    return SBP_OK;
}
inline void spans_of2(const sbp_tensor_t* t, const sbp_t* s, int32_t k0, int32_t k1, std::vector<Span>& v) {
    for (int32_t a = 0; a < k0; ++a)
        for (int32_t b = 0; b < k1; ++b) {
            const Local l = local_of2(t->rows, t->cols, s, k0, k1, a, b);
            if (l.rows * l.cols == 0) continue;
            const uintptr_t bytes = (uintptr_t)((l.rows - 1) * pitch_of(t, l) + l.cols) * elem_bytes(t->dtype);
            const uintptr_t lo = reinterpret_cast<uintptr_t>(t->shard[a * k1 + b]);
            v.push_back({lo, lo + bytes});
        }
}

// outputs must be pairwise disjoint and disjoint from every input
inline int32_t check_alias(const std::vector<Span>& outs, const std::vector<Span>& ins) {
    for (size_t a = 0; a < outs.size(); ++a) {
        for (size_t b = a + 1; b < outs.size(); ++b)
            if (overlap(outs[a], outs[b])) return SBP_ERR_ALIAS;
        for (const Span& in : ins)
            if (overlap(outs[a], in)) return SBP_ERR_ALIAS;
    }
    return SBP_OK;
}

// a vector [rows, 1], B (one device pointer per logical device; copies may share a buffer)
inline int32_t check_vector(const sbp_tensor_t* t, int64_t rows, int32_t dtype, int32_t k) {
    if (!t || !t->shard) return SBP_ERR_NULL;
    if (t->rows != rows || t->cols != 1) return SBP_ERR_SHAPE;
    if (t->dtype != dtype) return SBP_ERR_DTYPE;
    if (t->trans) return SBP_ERR_UNSUPPORTED;
    for (int32_t i = 0; i < k && rows > 0; ++i) {
        if (!t->shard[i]) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(t->shard[i]) & 15u) return SBP_ERR_ALIGN;
    }
    return SBP_OK;
}
inline void spans_of_vector(const sbp_tensor_t* t, int32_t k, std::vector<Span>& v) {
    for (int32_t i = 0; i < k; ++i) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(t->shard[i]);
        if (t->rows) v.push_back({lo, lo + (uintptr_t)t->rows * 4});
    }
}

}  // namespace sbp
