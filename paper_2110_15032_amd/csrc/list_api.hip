// Host side of the operators on lists of tensors: every check runs before anything is enqueued.
#include <cstdlib>

#include "sbp_buffers.h"

using namespace sbp;

namespace {

// A local tensor as it is stored.
struct Stored {
    int64_t rows, cols, pitch;
};
Stored stored_of(const sbp_tensor_t* t, sbp_t s, int32_t k, int32_t i) {
    const Local l = local_of(t->rows, t->cols, s, k, i);
    return {stored_rows(t, l), stored_cols(t, l), pitch_of(t, l)};
}
// one row where rows lie back to back
Stored as_rows(Stored s, bool dense) { return dense || s.rows == 1 ? Stored{1, s.rows * s.cols, 0} : s; }
int64_t chunks_of(const Stored& s) { return (s.rows * ((s.cols + 7) / 8) + LIST_CHUNK - 1) / LIST_CHUNK; }

int32_t check_list(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    if (n < 0) return SBP_ERR_SHAPE;
    if (n && (!t || !s)) return SBP_ERR_NULL;
    constexpr int64_t MOST = INT32_MAX;
    for (int32_t j = 0; j < n; ++j) {
        int32_t st;
        if ((st = check_whole(s[j])) != SBP_OK) return st;
        if (t[j].rows > MOST || t[j].cols > MOST) return SBP_ERR_UNSUPPORTED;   // before anything is multiplied
        if ((st = check_tensor(t + j, s[j], k, true)) != SBP_OK) return st;
    }
    return SBP_OK;
}
int32_t check_scalar(const sbp_tensor_t* t, int32_t k) { return check_column(t, 1, SBP_B, k, false); }

// What device i counts of tensor t.
struct Counted {
    const char* at;
    Stored s;
};
Counted counted(const sbp_tensor_t* t, sbp_t s, int32_t k, int32_t i) {
    Stored l = stored_of(t, s, k, i);
    const bool dense = l.pitch == l.cols;
    const char* at = static_cast<const char*>(t->shard[i]);
    if (s == SBP_B && l.rows * l.cols) {
        at += split_begin(l.rows, k, i) * l.pitch * elem_bytes(t->dtype);
        l.rows = split_len(l.rows, k, i);
    }
    return {at, as_rows(l, dense)};
}

// The launches of a sum of squares: devices in turn, parts of each in order, as many as a launch takes.  `blocks` workgroups for every
// device in every launch, each of which leaves a partial sum; device d's lie from d * turns * blocks on, launch by launch.
struct SquarePlan {
    int blocks;
    int32_t turns;
    int32_t used[SBP_MAX_K];   // launches that a device has parts in
};
template <typename F>   // F(plan, devices of the launch): a full launch
int32_t each_launch(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, SquarePlan& sq, ListPlan& plan, F&& launch) {
    for (int32_t d = 0; d < k; ++d) sq.used[d] = 0;
    int devices = 0;
    int64_t chunk = 0;
    plan.parts = 0;
    plan.chunk0[0] = 0;
    auto flush = [&]() {
        const int32_t st = devices ? launch(plan, devices) : SBP_OK;
        devices = 0;
        chunk = 0;
        plan.parts = 0;
        return st;
    };
    for (int32_t d = 0; d < k; ++d) {
        bool open = false;   // this device has its place in the launch being filled
        for (int32_t j = 0; j < n; ++j) {
            const Local l = local_of(t[j].rows, t[j].cols, s[j], k, d);
            if (l.rows * l.cols == 0) continue;
            const Counted c = counted(t + j, s[j], k, d);
            const int64_t chunks = chunks_of(c.s);
            if (chunks == 0) continue;
            if (chunks > INT32_MAX / 2) return SBP_ERR_UNSUPPORTED;
            if (plan.parts == LIST_PARTS || chunk + chunks > INT32_MAX / 2) {
                const int32_t st = flush();
                if (st != SBP_OK) return st;
                open = false;
            }
            if (!open) {
                plan.slot[devices] = d * sq.turns + sq.used[d]++;
                ++devices;
                open = true;
            }
            plan.first[plan.parts] = (int32_t)chunk;
            plan.s[plan.parts++] = {c.at, nullptr, c.s.cols, (int32_t)c.s.rows, (int32_t)c.s.pitch, 0, t[j].dtype == SBP_BF16 ? 1 : 0};
            chunk += chunks;
            plan.chunk0[devices] = (int32_t)chunk;
        }
    }
    return flush();
}
int32_t plan_squares(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, SquarePlan& sq, ListPlan& plan) {
    sq.turns = 0;
    int64_t most = 1;
    int devices_most = 1;
    const int32_t st = each_launch(t, s, n, k, sq, plan, [&](const ListPlan& p, int devices) {
        devices_most = std::max(devices_most, devices);
        for (int d = 0; d < devices; ++d) most = std::max<int64_t>(most, p.chunk0[d + 1] - p.chunk0[d]);
        return (int32_t)SBP_OK;
    });
    if (st != SBP_OK) return st;
    sq.blocks = (int)std::min<int64_t>(most, std::max(1, LIST_BLOCKS / devices_most));
    for (int32_t d = 0; d < k; ++d) sq.turns = std::max(sq.turns, sq.used[d]);
    return SBP_OK;
}

}  // namespace

extern "C" {

int32_t sbp_square_sum_workspace(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    int32_t st;
    if ((st = check_list(t, s, n, k)) != SBP_OK) return st;
    SquarePlan sq;
    ListPlan plan;
    if ((st = plan_squares(t, s, n, k, sq, plan)) != SBP_OK) return st;
    *bytes = (int64_t)k * sq.turns * sq.blocks * 8;
    return SBP_OK;
}

int32_t sbp_square_sum(const sbp_tensor_t* t, const sbp_t* s, int32_t n, const sbp_tensor_t* out, void* workspace, int64_t workspace_bytes, int32_t k, void* stream) {
    int32_t st;
    if ((st = check_list(t, s, n, k)) != SBP_OK) return st;
    if ((st = check_scalar(out, k)) != SBP_OK) return st;
    SquarePlan sq;
    ListPlan plan;
    if ((st = plan_squares(t, s, n, k, sq, plan)) != SBP_OK) return st;
    const int64_t room = (int64_t)k * sq.turns * sq.blocks * 8;
    if (room) {
        if (!workspace) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 15u) return SBP_ERR_ALIGN;
        if (workspace_bytes < room) return SBP_ERR_SHAPE;
    }
    Buffers b;
    b.add(true, out, SBP_B, k);
    b.add(true, workspace, 1, room, room, 1);
    if ((st = b.check()) != SBP_OK) return st;
    for (int32_t j = 0; j < n; ++j) {   // the outputs are in order now: the inputs against them, a few at a time
        b.n_in = 0;
        b.add(false, t + j, s[j], k);
        if ((st = b.check()) != SBP_OK) return st;
    }
    plan.partial = static_cast<double*>(workspace);
    st = each_launch(t, s, n, k, sq, plan, [&](const ListPlan& p, int devices) { return launch_square_sum(p, devices, sq.blocks, static_cast<hipStream_t>(stream)); });
    if (st != SBP_OK) return st;
    SquareJoin join{};
    join.partial = plan.partial;
    join.per_device = (int64_t)sq.turns * sq.blocks;
    for (int32_t d = 0; d < k; ++d) {
        join.count[d] = sq.used[d] * sq.blocks;
        join.out[d] = static_cast<float*>(out->shard[d]);
    }
    return launch_square_join(join, k, static_cast<hipStream_t>(stream));
}

int32_t sbp_clip(const sbp_tensor_t* in, const sbp_t* s, int32_t n, const sbp_tensor_t* squares, sbp_t sbp_squares, float max_norm, const sbp_tensor_t* out,
                 const sbp_tensor_t* norm, int32_t k, void* stream) {
    int32_t st;
    if ((st = check_list(in, s, n, k)) != SBP_OK) return st;
    if ((st = check_list(out, s, n, k)) != SBP_OK) return st;
    for (int32_t j = 0; j < n; ++j) {
        if (in[j].rows != out[j].rows || in[j].cols != out[j].cols) return SBP_ERR_SHAPE;
        if (in[j].trans != out[j].trans) return SBP_ERR_UNSUPPORTED;
        for (int32_t i = 0; i < k; ++i)
            if (chunks_of(stored_of(in + j, s[j], k, i)) > INT32_MAX / 2) return SBP_ERR_UNSUPPORTED;
    }
    if (!is_sbp(sbp_squares)) return SBP_ERR_AXIS;
    if (sbp_squares != SBP_P_SUM && sbp_squares != SBP_B) return SBP_ERR_SIGNATURE;
    if ((st = check_scalar(squares, k)) != SBP_OK) return st;
    if (norm && (st = check_scalar(norm, k)) != SBP_OK) return st;
    if (!(max_norm >= 0.0f)) return SBP_ERR_UNSUPPORTED;

    // outputs in the order of their addresses, each with its number; an input may meet its own output only, and only in place
    struct Out {
        Span span;
        int64_t id;
    };
    const int64_t most = ((int64_t)n + 1) * k;
    Out* const outs = static_cast<Out*>(std::malloc((size_t)most * sizeof(Out)));
    if (!outs) return SBP_ERR_UNSUPPORTED;
    int64_t n_out = 0;
    auto span = [&](const sbp_tensor_t* t, sbp_t sig, int32_t i) {
        const Stored l = stored_of(t, sig, k, i);
        const uintptr_t lo = reinterpret_cast<uintptr_t>(t->shard[i]);
        return l.rows * l.cols ? Span{lo, lo + (uintptr_t)((l.rows - 1) * l.pitch + l.cols) * elem_bytes(t->dtype)} : Span{0, 0};
    };
    auto clear = [&](const Span& v, int64_t id, bool in_place) {   // no output but its own, in place
        if (v.hi == 0) return true;
        const Out* o = std::upper_bound(outs, outs + n_out, v.lo, [](uintptr_t lo, const Out& b) { return lo < b.span.hi; });
        for (; o != outs + n_out && o->span.lo < v.hi; ++o)
            if (!in_place || o->id != id) return false;
        return true;
    };
    bool good = true;
    for (int32_t j = 0; j <= n; ++j)
        for (int32_t i = 0; i < k; ++i) {
            if (j == n && !norm) continue;
            const Span v = j < n ? span(out + j, s[j], i) : span(norm, SBP_B, i);
            if (v.hi) outs[n_out++] = {v, (int64_t)j * k + i};
        }
    auto before = [](const Out& a, const Out& b) { return a.span.lo < b.span.lo; };
    if (!std::is_sorted(outs, outs + n_out, before)) std::sort(outs, outs + n_out, before);
    for (int64_t i = 1; i < n_out; ++i) good = good && outs[i].span.lo >= outs[i - 1].span.hi;
    for (int32_t j = 0; good && j < n; ++j)
        for (int32_t i = 0; good && i < k; ++i) {
            const bool same = in[j].shard[i] == out[j].shard[i] && in[j].dtype == out[j].dtype && stored_of(in + j, s[j], k, i).pitch == stored_of(out + j, s[j], k, i).pitch;
            good = clear(span(in + j, s[j], i), (int64_t)j * k + i, same);
        }
    for (int32_t i = 0; good && i < k; ++i) good = clear(span(squares, SBP_B, i), -1, false);
    std::free(outs);
    if (!good) return SBP_ERR_ALIAS;

    ClipSum sums{};
    sums.most = max_norm;
    sums.k = k;
    sums.partial = sbp_squares == SBP_P_SUM;
    for (int32_t i = 0; i < k; ++i) {
        sums.sum[i] = static_cast<const float*>(squares->shard[i]);
        sums.norm[i] = norm ? static_cast<float*>(norm->shard[i]) : nullptr;
    }
    ListPlan plan{};
    int64_t chunk = 0;
    bool launched = false;
    auto flush = [&]() {
        plan.chunk0[1] = (int32_t)chunk;
        const int32_t status = launch_clip(plan, sums, static_cast<hipStream_t>(stream));
        for (int32_t i = 0; i < k; ++i) sums.norm[i] = nullptr;   // the first launch writes it
        plan.parts = 0;
        chunk = 0;
        launched = true;
        return status;
    };
    for (int32_t i = 0; i < k; ++i)
        for (int32_t j = 0; j < n; ++j) {
            const Stored a = stored_of(in + j, s[j], k, i), o = stored_of(out + j, s[j], k, i);
            if (a.rows * a.cols == 0) continue;
            const bool dense = a.pitch == a.cols && o.pitch == o.cols;
            const Stored l = as_rows(a, dense);
            const int64_t chunks = chunks_of(l);
            if (plan.parts == LIST_PARTS || chunk + chunks > INT32_MAX / 2)
                if ((st = flush()) != SBP_OK) return st;
            plan.first[plan.parts] = (int32_t)chunk;
            plan.s[plan.parts++] = {in[j].shard[i], out[j].shard[i], l.cols, (int32_t)l.rows, (int32_t)a.pitch, (int32_t)o.pitch,
                                    (in[j].dtype == SBP_BF16 ? 1 : 0) | (out[j].dtype == SBP_BF16 ? 2 : 0) | i << 2};
            chunk += chunks;
        }
    return plan.parts || (norm && !launched) ? flush() : SBP_OK;
}

}  // extern "C"
