// Host side of the operators on lists of tensors: every check runs before anything is enqueued.
#include <cstdlib>

#include "sbp_buffers.h"

using namespace sbp;

namespace {

// A local tensor as it is stored.
struct Stored {
    int64_t rows, cols, pitch;
    bool empty() const { return rows == 0 || cols == 0; }
    bool dense() const { return pitch == cols || rows == 1; }
};
// Those of a list, tensor j's on device i at [j * k + i], worked out once: a call goes through them several times, and 64-bit divisions are slow.
struct Locals {
    Stored* of = nullptr;
    ~Locals() { std::free(of); }
    bool room(int32_t n, int32_t k) {
        of = static_cast<Stored*>(std::malloc(((size_t)n * k + 1) * sizeof(Stored)));
        return of != nullptr;
    }
};
// one row where rows lie back to back
Stored as_rows(const Stored& s, bool dense) { return dense ? Stored{1, s.rows * s.cols, 0} : s; }
int64_t chunks_of(const Stored& s) { return (s.rows * ((s.cols + 7) / 8) + LIST_CHUNK - 1) / LIST_CHUNK; }
constexpr int64_t MOST_CHUNKS = INT32_MAX / 2;

// check_tensor's rules, with the local tensors noted
int32_t check_one(const sbp_tensor_t* t, sbp_t s, int32_t k, Stored* of) {
    const int32_t st = check_whole(s);
    if (st != SBP_OK) return st;
    if (!t->shard) return SBP_ERR_NULL;
    if (t->rows > INT32_MAX || t->cols > INT32_MAX) return SBP_ERR_UNSUPPORTED;   // before anything is multiplied
    if (t->rows < 0 || t->cols < 0 || t->ld < 0) return SBP_ERR_SHAPE;
    if (t->dtype != SBP_F32 && t->dtype != SBP_BF16) return SBP_ERR_DTYPE;
    if (t->trans != 0 && t->trans != 1) return SBP_ERR_SHAPE;
    if (t->ld > INT32_MAX) return SBP_ERR_UNSUPPORTED;
    const int64_t along = s == SBP_S(0) ? t->rows : t->cols, least = s == SBP_B ? 0 : along / k, more = s == SBP_B ? 0 : along % k;
    for (int32_t i = 0; i < k; ++i) {
        const int64_t part = least + (i < more ? 1 : 0), rows = s == SBP_S(0) ? part : t->rows, cols = s == SBP_S(1) ? part : t->cols;
        of[i] = t->trans ? Stored{cols, rows, t->ld ? t->ld : rows} : Stored{rows, cols, t->ld ? t->ld : cols};
        if (of[i].empty()) continue;
        if (of[i].cols > of[i].pitch) return SBP_ERR_SHAPE;
        if (!t->shard[i]) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(t->shard[i]) & 15u) return SBP_ERR_ALIGN;
        if (chunks_of(of[i]) > MOST_CHUNKS) return SBP_ERR_UNSUPPORTED;
    }
    return SBP_OK;
}
int32_t check_list(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, Locals& locals) {
    if (k < 1 || k > SBP_MAX_K) return SBP_ERR_K;
    if (n < 0) return SBP_ERR_SHAPE;
    if (n && (!t || !s)) return SBP_ERR_NULL;
    if (n > 1 << 20) return SBP_ERR_UNSUPPORTED;   // a device's launches are counted in 16 bits
    if (!locals.room(n, k)) return SBP_ERR_UNSUPPORTED;
    for (int32_t j = 0; j < n; ++j) {
        const int32_t st = check_one(t + j, s[j], k, locals.of + (int64_t)j * k);
        if (st != SBP_OK) return st;
    }
    return SBP_OK;
}
int32_t check_scalar(const sbp_tensor_t* t, int32_t k) { return check_column(t, 1, SBP_B, k, false); }
Span span_of(const sbp_tensor_t* t, const Stored& l, int32_t i) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(t->shard[i]);
    return l.empty() ? Span{0, 0} : Span{lo, lo + (uintptr_t)((l.rows - 1) * l.pitch + l.cols) * elem_bytes(t->dtype)};
}

// A local tensor of a list: what device i counts of it, or (clipping) holds of it.
struct Item {
    const char* in;
    char* out;
    Stored s;              // as_rows()
    int64_t ldo;
    int32_t what;          // without the device
    int64_t chunks;
};
bool counted(const sbp_tensor_t* t, sbp_t s, Stored l, int32_t k, int32_t i, Item& to) {
    if (l.empty()) return false;
    const bool dense = l.pitch == l.cols;
    const char* at = static_cast<const char*>(t->shard[i]);
    if (s == SBP_B) {   // its share of the stored rows
        at += split_begin(l.rows, k, i) * l.pitch * elem_bytes(t->dtype);
        l.rows = split_len(l.rows, k, i);
        if (l.rows == 0) return false;
    }
    const Stored r = as_rows(l, dense || l.rows == 1);
    to = {at, nullptr, r, 0, of_list(t->dtype == SBP_BF16, false, 0), chunks_of(r)};
    return true;
}
bool clipped(const sbp_tensor_t* in, const Stored& a, const sbp_tensor_t* out, const Stored& o, int32_t i, Item& to) {
    if (a.empty()) return false;
    const Stored r = as_rows(a, a.dense() && o.dense());
    to = {static_cast<const char*>(in->shard[i]), static_cast<char*>(out->shard[i]), r, o.pitch, of_list(in->dtype == SBP_BF16, out->dtype == SBP_BF16, 0), chunks_of(r)};
    return true;
}
// Two local tensors that lie back to back, results as well, are one.
bool joins(const Item& a, const Item& b) {
    return a.what == b.what && a.in + a.s.cols * (a.what & 1 ? 2 : 4) == b.in && (!a.out || a.out + a.s.cols * (a.what & 2 ? 2 : 4) == b.out);
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
            if (it.chunks > MOST_CHUNKS) return SBP_ERR_UNSUPPORTED;
            if (dense && mine && b.chunks + it.chunks <= MOST_CHUNKS && joins(b.item[b.n - 1], it)) {
                Item& last = b.item[b.n - 1];
                last.s.cols += it.s.cols;
                const int64_t more = chunks_of(last.s) - last.chunks;
                last.chunks += more;
                b.chunks += more;
                mine += more;
                b.most = std::max(b.most, mine);
                continue;
            }
            if (b.n && (b.n == cap || b.chunks + it.chunks > MOST_CHUNKS)) {
                const int32_t st = f(b);
                if (st != SBP_OK) return st;
                b.n = 0;
                mine = 0;
            }
            if (b.n == 0) {
                b.first_device = d;
                b.turn = used[d];
                b.chunks = b.most = 0;
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

// Past the caches go the sum of squares of more than the memory-side cache (256 MB) keeps for the clipping that follows, and the clipping of what
// moves more than a good part of it.  us for both calls, neither / both past the caches: 2^28 elements from bf16 to fp32 390 / 352, 100 M in bf16 (200 MB)
// 119 / 104, with the sum of squares cached 98; 67 M 82 / 71 / 68; 34 M (67 MB, 134 moved) 44.0 / 41.4; 17 M 23.7 / 26.4.
constexpr int64_t KEPT = (int64_t)192 << 20, MOVED = (int64_t)96 << 20;

// How a sum of squares is dealt out.
struct SquareShape {
    int32_t blocks;                                    // workgroups of every device in every launch
    int32_t dense_turns, turns;                        // places of a device's partial sums, in units of them
    int16_t dense[SBP_MAX_K], pitched[SBP_MAX_K];      // launches that a device has parts in
    int64_t bytes;                                     // for the workspace
    int32_t stream;                                    // what is read goes past the caches
};
// The workspace goes by the sizes alone, and not by which tensors lie back to back: a device has parts in at most so many launches, and at most so many
// workgroups there.
int32_t square_shape(const sbp_tensor_t* t, const sbp_t* s, const Locals& locals, int32_t n, int32_t k, SquareShape& sq, Batch& b) {
    int64_t most = 1, all = 0, read = 0;
    int32_t devices = 1, st;
    for (int32_t d = 0; d < k; ++d) {
        int64_t mine = 0;
        for (int32_t j = 0; j < n; ++j) {
            const Stored& l = locals.of[(int64_t)j * k + d];
            mine += l.empty() ? 0 : chunks_of(l);
            read += l.rows * l.cols * elem_bytes(t[j].dtype);
        }
        all = std::max(all, mine);
    }
    sq.stream = read > KEPT;
    auto make = [&](int32_t j, int32_t d, Item& it) { return counted(t + j, s[j], locals.of[(int64_t)j * k + d], k, d, it); };
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
    const int64_t turns = (n + LIST_DENSE - 1) / LIST_DENSE + (n + LIST_PITCHED - 1) / LIST_PITCHED + 2;
    if (sq.turns > turns) return SBP_ERR_UNSUPPORTED;   // tensors that no memory holds
    sq.bytes = (all ? k * turns * std::min<int64_t>(all, LIST_BLOCKS) : 0) * 8;
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
    plan.stream = sq.stream;
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
int32_t clip_batch(const Batch& b, const sbp_tensor_t* squares, bool partial, bool past, float most, const sbp_tensor_t* norm, int32_t k, MAKE&& make, hipStream_t stream) {
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
    plan.stream = past;
    return launch_clip(plan, stream);
}
template <template <bool> class PART, int CAP, typename MAKE>
int32_t clip_devices(const Batch& b, const sbp_tensor_t* squares, bool partial, bool past, float most, const sbp_tensor_t* norm, int32_t k, MAKE&& make, hipStream_t stream) {
    return k <= 8 ? clip_batch<PART, CAP, 8>(b, squares, partial, past, most, norm, k, make, stream) : clip_batch<PART, CAP, SBP_MAX_K>(b, squares, partial, past, most, norm, k, make, stream);
}

}  // namespace

extern "C" {

int32_t sbp_square_sum_workspace(const sbp_tensor_t* t, const sbp_t* s, int32_t n, int32_t k, int64_t* bytes) {
    if (!bytes) return SBP_ERR_NULL;
    int32_t st;
    Locals locals;
    if ((st = check_list(t, s, n, k, locals)) != SBP_OK) return st;
    SquareShape sq;
    Batch batch;
    if ((st = square_shape(t, s, locals, n, k, sq, batch)) != SBP_OK) return st;
    *bytes = sq.bytes;
    return SBP_OK;
}

int32_t sbp_square_sum(const sbp_tensor_t* t, const sbp_t* s, int32_t n, const sbp_tensor_t* out, void* workspace, int64_t workspace_bytes, int32_t k, void* stream) {
    int32_t st;
    Locals locals;
    if ((st = check_list(t, s, n, k, locals)) != SBP_OK) return st;
    if ((st = check_scalar(out, k)) != SBP_OK) return st;
    SquareShape sq;
    Batch batch;
    if ((st = square_shape(t, s, locals, n, k, sq, batch)) != SBP_OK) return st;
    if (sq.bytes) {
        if (!workspace) return SBP_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 15u) return SBP_ERR_ALIGN;
        if (workspace_bytes < sq.bytes) return SBP_ERR_SHAPE;
    }
    Buffers b;
    b.add(true, out, SBP_B, k);
    b.add(true, workspace, 1, sq.bytes, sq.bytes, 1);
    if ((st = b.check()) != SBP_OK) return st;
    for (int32_t j = 0; j < n; ++j)   // the outputs are in order now
        for (int32_t i = 0; i < k; ++i)
            if (b.meets(span_of(t + j, locals.of[(int64_t)j * k + i], i))) return SBP_ERR_ALIAS;
    double* const partial = static_cast<double*>(workspace);
    const hipStream_t on = static_cast<hipStream_t>(stream);
    auto make = [&](int32_t j, int32_t d, Item& it) { return counted(t + j, s[j], locals.of[(int64_t)j * k + d], k, d, it); };
    int16_t used[SBP_MAX_K];
    st = each_batch(n, k, true, batch, used, make, [&](const Batch& b) {
        if (b.n <= LIST_FEW) return square_batch<DensePart, LIST_FEW>(b, sq, 0, partial, dense_part<false>, on);
        if (b.n <= LIST_SOME) return square_batch<DensePart, LIST_SOME>(b, sq, 0, partial, dense_part<false>, on);
        return square_batch<DensePart, LIST_DENSE>(b, sq, 0, partial, dense_part<false>, on);
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
    Locals from, to;
    if ((st = check_list(in, s, n, k, from)) != SBP_OK) return st;
    if ((st = check_list(out, s, n, k, to)) != SBP_OK) return st;
    for (int32_t j = 0; j < n; ++j) {
        if (in[j].rows != out[j].rows || in[j].cols != out[j].cols) return SBP_ERR_SHAPE;
        if (in[j].trans != out[j].trans) return SBP_ERR_UNSUPPORTED;
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
    auto clear = [&](const Span& v, int64_t id, bool in_place) {   // no output but its own, in place
        if (v.hi == 0) return true;
        const Out* o = std::upper_bound(outs, outs + n_out, v.lo, [](uintptr_t lo, const Out& b) { return lo < b.span.hi; });
        for (; o != outs + n_out && o->span.lo < v.hi; ++o)
            if (!in_place || o->id != id) return false;
        return true;
    };
    bool good = true;
    constexpr Stored SCALAR = {1, 1, 1};
    for (int32_t i = 0; i < k; ++i)
        for (int32_t j = 0; j <= n; ++j) {
            if (j == n && !norm) continue;
            const Span v = j < n ? span_of(out + j, to.of[(int64_t)j * k + i], i) : span_of(norm, SCALAR, i);
            if (v.hi) outs[n_out++] = {v, (int64_t)j * k + i};
        }
    auto before = [](const Out& a, const Out& b) { return a.span.lo < b.span.lo; };
    if (!std::is_sorted(outs, outs + n_out, before)) std::sort(outs, outs + n_out, before);
    for (int64_t i = 1; i < n_out; ++i) good = good && outs[i].span.lo >= outs[i - 1].span.hi;
    for (int32_t j = 0; good && j < n; ++j)
        for (int32_t i = 0; good && i < k; ++i) {
            const int64_t id = (int64_t)j * k + i;
            const bool same = in[j].shard[i] == out[j].shard[i] && in[j].dtype == out[j].dtype && from.of[id].pitch == to.of[id].pitch;
            good = clear(span_of(in + j, from.of[id], i), id, same);
        }
    for (int32_t i = 0; good && i < k; ++i) good = clear(span_of(squares, SCALAR, i), -1, false);
    std::free(outs);
    if (!good) return SBP_ERR_ALIAS;

    const hipStream_t on = static_cast<hipStream_t>(stream);
    const bool partial = sbp_squares == SBP_P_SUM;
    int64_t moved = 0;
    for (int32_t j = 0; j < n; ++j)
        for (int32_t i = 0; i < k; ++i) moved += from.of[(int64_t)j * k + i].rows * from.of[(int64_t)j * k + i].cols * (elem_bytes(in[j].dtype) + elem_bytes(out[j].dtype));
    const bool past = moved > MOVED;
    auto make = [&](int32_t j, int32_t d, Item& it) { return clipped(in + j, from.of[(int64_t)j * k + d], out + j, to.of[(int64_t)j * k + d], d, it); };
    int16_t used[SBP_MAX_K];
    Batch batch;
    const sbp_tensor_t* write = norm;   // the first launch does
    st = each_batch(n, k, true, batch, used, make, [&](const Batch& b) {
        const int32_t status = b.n <= LIST_FEW ? clip_devices<DensePart, LIST_FEW>(b, squares, partial, past, max_norm, write, k, dense_part<true>, on)
                             : b.n <= LIST_SOME ? clip_devices<DensePart, LIST_SOME>(b, squares, partial, past, max_norm, write, k, dense_part<true>, on)
                                               : clip_devices<DensePart, LIST_DENSE>(b, squares, partial, past, max_norm, write, k, dense_part<true>, on);
        write = nullptr;
        return status;
    });
    if (st != SBP_OK) return st;
    st = each_batch(n, k, false, batch, used, make, [&](const Batch& b) {
        const int32_t status = b.n <= LIST_FEW ? clip_devices<PitchedPart, LIST_FEW>(b, squares, partial, past, max_norm, write, k, pitched_part<true>, on)
                                               : clip_devices<PitchedPart, LIST_PITCHED>(b, squares, partial, past, max_norm, write, k, pitched_part<true>, on);
        write = nullptr;
        return status;
    });
    if (st != SBP_OK || !write) return st;
    batch.n = 0;   // nothing but the norm
    batch.chunks = batch.first_device = 0;
    return clip_devices<DensePart, LIST_FEW>(batch, squares, partial, past, max_norm, write, k, dense_part<true>, on);
}

}  // extern "C"
