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

// A local tensor of a list: what device i counts of it, or (clipping) holds of it.
struct Item {
    const char* in;
    char* out;
    Stored s;              // as_rows()
    int64_t ldo;
    int32_t what;          // without the device
    int64_t chunks;
};
bool counted(const sbp_tensor_t* t, sbp_t s, int32_t k, int32_t i, Item& to) {
    Stored l = stored_of(t, s, k, i);
    if (l.rows * l.cols == 0) return false;
    const bool dense = l.pitch == l.cols;
    const char* at = static_cast<const char*>(t->shard[i]);
    if (s == SBP_B) {   // its share of the stored rows
        at += split_begin(l.rows, k, i) * l.pitch * elem_bytes(t->dtype);
        l.rows = split_len(l.rows, k, i);
        if (l.rows == 0) return false;
    }
    const Stored r = as_rows(l, dense);
    to = {at, nullptr, r, 0, of_list(t->dtype == SBP_BF16, false, 0), chunks_of(r)};
    return true;
}
bool clipped(const sbp_tensor_t* in, const sbp_tensor_t* out, sbp_t s, int32_t k, int32_t i, Item& to) {
    const Stored a = stored_of(in, s, k, i), o = stored_of(out, s, k, i);
    if (a.rows * a.cols == 0) return false;
    const Stored r = as_rows(a, a.pitch == a.cols && o.pitch == o.cols);
    to = {static_cast<const char*>(in->shard[i]), static_cast<char*>(out->shard[i]), r, o.pitch, of_list(in->dtype == SBP_BF16, out->dtype == SBP_BF16, 0), chunks_of(r)};
    return true;
}

// Local tensors of one launch, in the order of their devices.
struct Batch {
    Item item[LIST_DENSE];
    int32_t device[LIST_DENSE];
    int32_t n, first_device, devices;
    int32_t turn;          // launches that the first device has parts in already
    int64_t chunks, most;  // all, and the most of a device
};
// F(batch) for the local tensors that lie in one row, or for those with rows at a pitch; ITEM(tensor, device, item): false where there is nothing.
// used: batches that a device has parts in.
template <typename ITEM, typename F>
int32_t each_batch(int32_t n, int32_t k, bool dense, Batch& b, int16_t* used, ITEM&& make, F&& f) {
    const int32_t cap = dense ? LIST_DENSE : LIST_PITCHED;
    b.n = 0;
    for (int32_t d = 0; d < k; ++d) {
        used[d] = 0;
        int64_t mine = 0;   // chunks of this device in the batch
        for (int32_t j = 0; j < n; ++j) {
            Item it;
            if (!make(j, d, it) || (it.s.rows == 1) != dense) continue;
            if (it.chunks > INT32_MAX / 2) return SBP_ERR_UNSUPPORTED;
            if (b.n && (b.n == cap || b.chunks + it.chunks > INT32_MAX / 2)) {
                const int32_t st = f(b);
                if (st != SBP_OK) return st;
                b.n = 0;
            }
            if (b.n == 0) {
                b.first_device = d;
                b.turn = used[d];
                b.chunks = b.most = mine = 0;
            }
            if (mine == 0) ++used[d];
            b.item[b.n] = it;
            b.device[b.n++] = d - b.first_device;
            b.devices = d - b.first_device + 1;
            b.chunks += it.chunks;
            mine += it.chunks;
            b.most = std::max(b.most, mine);
        }
    }
    return b.n ? f(b) : SBP_OK;
}
template <bool OUT>
DensePart<OUT> dense_part(const Item& it, int32_t device) {
    const uint64_t info = (uint64_t)it.s.cols | (uint64_t)(it.what | device << 2) << 48;
    if constexpr (OUT) return {it.in, it.out, info};
    else return {it.in, info};
}
template <bool OUT>
PitchedPart<OUT> pitched_part(const Item& it, int32_t device) {
    return {it.in, it.out, (int32_t)it.s.rows, (int32_t)it.s.cols, (int32_t)it.s.pitch, (int32_t)it.ldo, it.what | device << 2};
}

// How a sum of squares is dealt out.
struct SquareShape {
    int32_t blocks;                                    // workgroups of every device in every launch
    int32_t dense_turns, turns;                        // places of a device's partial sums, in units of them
    int16_t dense[SBP_MAX_K], pitched[SBP_MAX_K];      // launches that a device has parts in
    int64_t bytes(int32_t k) const { return (int64_t)k * turns * blocks * 8; }
};
int32_t square_shape(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, SquareShape& sq, Batch& b) {
    int64_t most = 1;
    int32_t devices = 1, st;
    auto make = [&](int32_t j, int32_t d, Item& it) { return counted(t + j, s[j], k, d, it); };
    auto look = [&](const Batch& b) {
        most = std::max(most, b.most);
        devices = std::max(devices, b.devices);
        return (int32_t)SBP_OK;
    };
    if ((st = each_batch(n, k, true, b, sq.dense, make, look)) != SBP_OK) return st;
    if ((st = each_batch(n, k, false, b, sq.pitched, make, look)) != SBP_OK) return st;
    sq.blocks = (int32_t)std::min<int64_t>(most, std::max(1, LIST_BLOCKS / devices));
    sq.dense_turns = *std::max_element(sq.dense, sq.dense + k);
    sq.turns = sq.dense_turns + *std::max_element(sq.pitched, sq.pitched + k);
    return SBP_OK;
}
template <template <bool> class PART, int CAP, typename MAKE>
int32_t square_batch(const Batch& b, const SquareShape& sq, int32_t base, double* partial, MAKE&& make, hipStream_t stream) {
    SquarePlan<PART, CAP> plan;
    for (int32_t i = 0; i < CAP; ++i) plan.s[i] = i < b.n ? make(b.item[i], b.device[i]) : PART<false>{};
    plan.partial = partial;
    plan.parts = b.n;
    plan.first_device = b.first_device;
    plan.turns = sq.turns;
    plan.first_turn = base + b.turn;
    plan.other_turn = base;
    return launch_square_sum(plan, b.devices, sq.blocks, stream);
}
template <int S>
int32_t square_join(const SquareShape& sq, const double* partial, const sbp_tensor_t* out, int32_t k, hipStream_t stream) {
    SquareJoin<S> join{};
    join.partial = partial;
    join.blocks = sq.blocks;
    join.turns = sq.turns;
    join.dense_turns = sq.dense_turns;
    for (int32_t d = 0; d < k; ++d) {
        join.dense[d] = sq.dense[d];
        join.pitched[d] = sq.pitched[d];
        join.out[d] = static_cast<float*>(out->shard[d]);
    }
    return launch_square_join(join, k, stream);
}
template <template <bool> class PART, int CAP, int S, typename MAKE>
int32_t clip_batch(const Batch& b, const sbp_tensor_t* squares, bool partial, float most, const sbp_tensor_t* norm, int32_t k, MAKE&& make, hipStream_t stream) {
    ClipPlan<PART, CAP, S> plan{};
    for (int32_t i = 0; i < b.n; ++i) plan.s[i] = make(b.item[i], b.device[i]);
    for (int32_t i = 0; i < k; ++i) {
        plan.sum[i] = static_cast<const float*>(squares->shard[i]);
        plan.norm[i] = norm ? static_cast<float*>(norm->shard[i]) : nullptr;
    }
    plan.most = most;
    plan.parts = b.n;
    plan.chunks = (int32_t)b.chunks;
    plan.k = k;
    plan.partial = partial;
    plan.first_device = b.first_device;
    return launch_clip(plan, stream);
}
template <template <bool> class PART, int CAP, typename MAKE>
int32_t clip_devices(const Batch& b, const sbp_tensor_t* squares, bool partial, float most, const sbp_tensor_t* norm, int32_t k, MAKE&& make, hipStream_t stream) {
    return k <= 8 ? clip_batch<PART, CAP, 8>(b, squares, partial, most, norm, k, make, stream) : clip_batch<PART, CAP, SBP_MAX_K>(b, squares, partial, most, norm, k, make, stream);
}

}  // namespace

extern "C" {

int32_t sbp_square_sum_workspace(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    int32_t st;
    if ((st = check_list(t, s, n, k)) != SBP_OK) return st;
    SquareShape sq;
    Batch batch;
    if ((st = square_shape(t, s, n, k, sq, batch)) != SBP_OK) return st;
    *bytes = sq.bytes(k);
    return SBP_OK;
}

int32_t sbp_square_sum(const sbp_tensor_t* t, const sbp_t* s, int32_t n, const sbp_tensor_t* out, void* workspace, int64_t workspace_bytes, int32_t k, void* stream) {
    int32_t st;
    if ((st = check_list(t, s, n, k)) != SBP_OK) return st;
    if ((st = check_scalar(out, k)) != SBP_OK) return st;
    SquareShape sq;
    Batch batch;
    if ((st = square_shape(t, s, n, k, sq, batch)) != SBP_OK) return st;
    const int64_t room = sq.bytes(k);
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
    double* const partial = static_cast<double*>(workspace);
    const hipStream_t on = static_cast<hipStream_t>(stream);
    auto make = [&](int32_t j, int32_t d, Item& it) { return counted(t + j, s[j], k, d, it); };
    int16_t used[SBP_MAX_K];
    st = each_batch(n, k, true, batch, used, make, [&](const Batch& b) {
        return b.n <= LIST_FEW ? square_batch<DensePart, LIST_FEW>(b, sq, 0, partial, dense_part<false>, on) : square_batch<DensePart, LIST_DENSE>(b, sq, 0, partial, dense_part<false>, on);
    });
    if (st != SBP_OK) return st;
    st = each_batch(n, k, false, batch, used, make, [&](const Batch& b) {
        return b.n <= LIST_FEW ? square_batch<PitchedPart, LIST_FEW>(b, sq, sq.dense_turns, partial, pitched_part<false>, on)
                               : square_batch<PitchedPart, LIST_PITCHED>(b, sq, sq.dense_turns, partial, pitched_part<false>, on);
    });
    if (st != SBP_OK) return st;
    return k <= 8 ? square_join<8>(sq, partial, out, k, on) : square_join<SBP_MAX_K>(sq, partial, out, k, on);
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

    const hipStream_t on = static_cast<hipStream_t>(stream);
    const bool partial = sbp_squares == SBP_P_SUM;
    auto make = [&](int32_t j, int32_t d, Item& it) { return clipped(in + j, out + j, s[j], k, d, it); };
    int16_t used[SBP_MAX_K];
    Batch batch;
    const sbp_tensor_t* to = norm;   // the first launch writes it
    st = each_batch(n, k, true, batch, used, make, [&](const Batch& b) {
        const int32_t status = b.n <= LIST_FEW ? clip_devices<DensePart, LIST_FEW>(b, squares, partial, max_norm, to, k, dense_part<true>, on)
                                               : clip_devices<DensePart, LIST_DENSE>(b, squares, partial, max_norm, to, k, dense_part<true>, on);
        to = nullptr;
        return status;
    });
    if (st != SBP_OK) return st;
    st = each_batch(n, k, false, batch, used, make, [&](const Batch& b) {
        const int32_t status = b.n <= LIST_FEW ? clip_devices<PitchedPart, LIST_FEW>(b, squares, partial, max_norm, to, k, pitched_part<true>, on)
                                               : clip_devices<PitchedPart, LIST_PITCHED>(b, squares, partial, max_norm, to, k, pitched_part<true>, on);
        to = nullptr;
        return status;
    });
    if (st != SBP_OK || !to) return st;
    batch.n = 0;   // nothing but the norm
    batch.chunks = batch.first_device = 0;
    return clip_devices<DensePart, LIST_FEW>(batch, squares, partial, max_norm, to, k, dense_part<true>, on);
}

}  // extern "C"
