// The sum of squares of many tensors, and all of them times one factor: the norm of all gradients and their clipping.
//
//   s_i = sum over the tensors of x^2 over what device i counts,  norm = sqrt(sum of s_i),  out = x min(1, max_norm / norm)
//
// Both are bound by HBM.  The argument block of a launch names local tensors (parts); their vectors of eight elements are numbered
// through, a workgroup takes 1024 of them at a time (a chunk, of one part).  Where a part's chunks start is summed up over the lanes of every wave, so that the
// argument block need not hold it.  2^28 elements from bf16 to fp32 on 8 devices: 80 us for the sum (537 MB, 6.7 TB/s), 265 for the clipping (1.61 GB, 6.1 TB/s), 353 in
// all; 72 small tensors on two devices 22, of which the device works 11 in three launches.
#include "block8_device.h"

namespace sbp {
namespace {

constexpr int NT = 256, PER = LIST_CHUNK / NT;
constexpr uint64_t ELEMENTS = ((uint64_t)1 << 48) - 1;

// Waves a SIMD: eight, for all of a launch's workgroups at once (seven, with the rest in a second turn, took 117 us where eight take 109, 2^28 bf16
// elements); rows at a pitch need more registers.
template <template <bool> class PART>
constexpr int waves_with(int pitched) { return std::is_same_v<PART<false>, DensePart<false>> ? 8 : pitched; }

// A part as the kernels see it: `count` elements in one row (rows 1), or rows of `cols` at a pitch.
struct Shape {
    int64_t cols;
    int32_t rows, ldi, ldo, what;
};
template <bool OUT>
__device__ inline Shape shape_of(const DensePart<OUT>& s) { return {(int64_t)(s.info & ELEMENTS), 1, 0, 0, (int32_t)(s.info >> 48)}; }
template <bool OUT>
__device__ inline Shape shape_of(const PitchedPart<OUT>& s) { return {s.cols, s.rows, s.ldi, s.ldo, s.what}; }
__device__ inline int chunks_of(const Shape& s) {
    const int64_t vectors = s.rows == 1 ? (s.cols + 7) / 8 : s.rows * ((s.cols + 7) / 8);
    return (int)((vectors + LIST_CHUNK - 1) / LIST_CHUNK);
}

// First chunk of every part: lane l holds those of parts l, l + 64, l + 128.
template <int CAP>
struct Starts {
    static constexpr int N = (CAP + 63) / 64;
    int32_t start[N], total;
    int32_t device[N];   // of a part, behind the last one a number that is none
    template <typename PART>
    __device__ Starts(const PART (&s)[CAP], int parts) {
        const int lane = threadIdx.x & 63;
        total = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = i * 64 + lane;
            int mine = 0;
            device[i] = INT32_MAX;
            if (at < parts) {
                const Shape h = shape_of(s[at]);
                mine = chunks_of(h);
                device[i] = h.what >> 2;
            }
            int sum = mine;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int other = __shfl_up(sum, off, 64);
                sum += lane >= off ? other : 0;
            }
            start[i] = at < parts ? total + sum - mine : INT32_MAX;
            total += __shfl(sum, 63, 64);
        }
    }
    // parts of devices before the d-th
    __device__ int parts_before(int d) const {
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(device[i] < d));
        return n;
    }
    __device__ int start_of(int part) const {   // part is uniform; behind the last one the number of chunks
        int v = total;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (part >> 6 == i) v = __builtin_amdgcn_readlane(start[i], part & 63);
        return v == INT32_MAX ? total : v;
    }
    __device__ int part_of(int chunk) const {
        int n = -1;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(start[i] <= chunk));
        return n;
    }
};

// F(turn, row, first column that the pointer stands for, column from there on, length of the row from there on) of the chunk's vectors.  The first
// column counts from the row's start in 64 bits, as a dense tensor may be longer than 2^31.
template <typename F>
__device__ inline void each_vector(const Shape& s, int chunk, F&& f) {
    const int64_t first = (int64_t)chunk * LIST_CHUNK;
    if (s.rows == 1) {
        const int64_t left = s.cols - first * 8;
#pragma unroll
        for (int u = 0; u < PER; ++u) f(u, (int64_t)0, first * 8, (u * NT + (int)threadIdx.x) * 8, (int)(left < LIST_CHUNK * 8 + 8 ? left : LIST_CHUNK * 8 + 8));
        return;
    }
    const int32_t per_row = (int32_t)((s.cols + 7) / 8);
    const int64_t row0 = first / per_row;
    const uint32_t vector0 = (uint32_t)(first - row0 * per_row);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        uint32_t v = vector0 + (uint32_t)(u * NT) + threadIdx.x, r = 0;
        if (per_row > LIST_CHUNK) {
            if (v >= (uint32_t)per_row) {
                v -= (uint32_t)per_row;
                r = 1;
            }
        } else {
            r = v / (uint32_t)per_row;
            v -= r * (uint32_t)per_row;
        }
        const int64_t row = row0 + r;
        f(u, row, (int64_t)0, (int)v * 8, row < s.rows ? (int)s.cols : 0);
    }
}
// settle8 of rows that may be as long as 2^31 - 1
template <int T>
__device__ inline Raw8<T> settle_any8(const Raw8<T> r, int c, int cols) {
    const int left = cols - c;
    return left >= 8 || left <= 0 || cols < 8 ? r : without_front<T>(r, 8 - left);
}
// all of the chunk's vectors are whole ones of one row
__device__ inline bool whole_chunk(const Shape& s, int chunk) { return s.rows == 1 && ((int64_t)chunk + 1) * (LIST_CHUNK * 8) <= s.cols; }
// Whole chunks: G consecutive elements a lane and load, so that the loads and stores of a wave are of consecutive bytes where the wider side has 16 of a lane.  At an element's
// alignment: a device's share of a copy starts at any row.
template <int T, int G>
struct Group;   // G elements as they are stored
template <>
struct Group<T_F32, 4> {
    typedef f32x4_any type;
};
template <>
struct Group<T_BF16, 4> {
    typedef u32x2_half type;
};
template <>
struct Group<T_BF16, 8> {
    typedef u32x4_any type;
};
template <int T, int G>
__device__ inline void widen_group(const typename Group<T, G>::type r, float (&v)[G]) {
#pragma unroll
    for (int e = 0; e < G; ++e) {
        if constexpr (T == T_F32) v[e] = r[e];
        else v[e] = __uint_as_float(e & 1 ? r[e >> 1] & 0xFFFF0000u : r[e >> 1] << 16);
    }
}
template <int T, int G>
__device__ inline typename Group<T, G>::type narrow_group(const float (&v)[G]) {
    typename Group<T, G>::type r;
#pragma unroll
    for (int e = 0; e < G; ++e) {
        if constexpr (T == T_F32) r[e] = v[e];
        else if (e & 1) r[e >> 1] = f32_to_bf16x2(v[e - 1], v[e]);
    }
    return r;
}
template <int T, int G>
__device__ inline const typename Group<T, G>::type* group_at(const void* p, int chunk) {
    return reinterpret_cast<const typename Group<T, G>::type*>(static_cast<const char*>(p) + (int64_t)chunk * (LIST_CHUNK * 8 * bytes_of<T>)) + threadIdx.x;
}
// STREAM: past the caches (a template argument, as the compiler takes the two forms of a load in two branches for one)
template <bool STREAM, int T, int G, int N>
__device__ inline void load_whole(const void* in, int chunk, typename Group<T, G>::type (&raw)[N]) {
    const auto* const from = group_at<T, G>(in, chunk);
#pragma unroll
    for (int u = 0; u < N; ++u) {
        if constexpr (STREAM) raw[u] = __builtin_nontemporal_load(from + u * NT);
        else raw[u] = from[u * NT];
    }
}

// Squares are summed in 64 bits: neither the number of elements nor their size loses anything before the sum is rounded to fp32.  Lane, wave and workgroup
// sums in an order of the sizes alone.
__device__ inline double sum_block(double v, double* waves) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    v = waves[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v += waves[w];
    return v;
}
template <int G>
__device__ inline void add_squares(const float (&v)[G], double (&acc)[2]) {
#pragma unroll
    for (int e = 0; e < G; ++e) acc[e & 1] = fma((double)v[e], (double)v[e], acc[e & 1]);
}

template <bool STREAM, int T>
__device__ inline void square_chunk(const void* in, const Shape& s, int chunk, double (&acc)[2]) {
    if (whole_chunk(s, chunk)) {
        constexpr int G = T == T_F32 ? 4 : 8, N = LIST_CHUNK * 8 / NT / G;
        typename Group<T, G>::type raw[N];
        load_whole<STREAM, T, G>(in, chunk, raw);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float v[G];
            widen_group<T, G>(raw[u], v);
            add_squares(v, acc);
        }
        return;
    }
    Raw8<T> raw[PER];
    float v[8];
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) { raw[u] = load8<T>(static_cast<const char*>(in) + (row * s.ldi + from) * bytes_of<T>, c, cols); });
    each_vector(s, chunk, [&](int u, int64_t, int64_t, int c, int cols) {
        widen<T>(settle_any8<T>(raw[u], c, cols), 1.0f, v);
        add_squares(v, acc);
    });
}

template <bool STREAM, template <bool> class PART, int CAP>
__global__ __launch_bounds__(NT, waves_with<PART>(5)) void square_sum_kernel(SquarePlan<PART, CAP> p) {
    __shared__ double waves[NT / 64];
    const Starts<CAP> starts(p.s, p.parts);
    const int d = blockIdx.y, end = starts.start_of(starts.parts_before(d + 1));
    double acc[2] = {0.0, 0.0};
    for (int c = starts.start_of(starts.parts_before(d)) + blockIdx.x; c < end; c += gridDim.x) {
        const int part = __builtin_amdgcn_readfirstlane(starts.part_of(c));
        const Shape s = shape_of(p.s[part]);
        const int chunk = c - starts.start_of(part);
        if (s.what & 1) square_chunk<STREAM, T_BF16>(p.s[part].in, s, chunk, acc);
        else square_chunk<STREAM, T_F32>(p.s[part].in, s, chunk, acc);
    }
    const double sum = sum_block(acc[0] + acc[1], waves);
    if (threadIdx.x == 0) p.partial[((int64_t)(p.first_device + d) * p.turns + (d ? p.other_turn : p.first_turn)) * gridDim.x + blockIdx.x] = sum;
}

// The partial sums of every device, joined in order and rounded once.
template <int S>
__global__ __launch_bounds__(NT) void square_join_kernel(SquareJoin<S> p) {
    __shared__ double waves[NT / 64];
    const int d = blockIdx.x;
    const double* const part = p.partial + (int64_t)d * p.turns * p.blocks;
    double v = 0.0;
    for (int i = threadIdx.x; i < p.dense[d] * p.blocks; i += NT) v += part[i];
    for (int i = threadIdx.x; i < p.pitched[d] * p.blocks; i += NT) v += part[p.dense_turns * p.blocks + i];
    v = sum_block(v, waves);
    if (threadIdx.x == 0) *p.out[d] = (float)v;
}

template <typename PLAN>
__device__ inline float sum_of(const PLAN& p, int d) {
    if (!p.partial) return *p.sum[d];
    float v = *p.sum[0];
    for (int i = 1; i < p.k; ++i) v += *p.sum[i];   // in the order of the devices, as boxing adds
    return v;
}
// A norm that is no number makes the factor NaN, an infinite one 0.
__device__ inline float factor_of(float sum, float most) {
    const float norm = sqrtf(sum);
    return norm <= most ? 1.0f : most / norm;
}

template <bool STREAM, int T, int U>
__device__ inline void clip_chunk(const void* in, void* out, const Shape& s, int chunk, float factor) {
    if (whole_chunk(s, chunk)) {
        constexpr int G = T == T_BF16 && U == T_BF16 ? 8 : 4, N = LIST_CHUNK * 8 / NT / G;
        typename Group<T, G>::type raw[N];
        load_whole<STREAM, T, G>(in, chunk, raw);
        auto* const to = const_cast<typename Group<U, G>::type*>(group_at<U, G>(out, chunk));
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float v[G];
            widen_group<T, G>(raw[u], v);
#pragma unroll
            for (int e = 0; e < G; ++e) v[e] *= factor;
            if constexpr (STREAM) __builtin_nontemporal_store(narrow_group<U, G>(v), to + u * NT);
            else to[u * NT] = narrow_group<U, G>(v);
        }
        return;
    }
    Raw8<T> raw[PER];
    float v[8];
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) { raw[u] = load8<T>(static_cast<const char*>(in) + (row * s.ldi + from) * bytes_of<T>, c, cols); });
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) {
        widen<T>(settle_any8<T>(raw[u], c, cols), 1.0f, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= factor;
        store8<U>(static_cast<char*>(out) + (row * s.ldo + from + c) * bytes_of<U>, narrow<U>(v), cols - c);   // none of them where cols - c is not positive
    });
}

template <bool STREAM, template <bool> class PART, int CAP, int S>
__global__ __launch_bounds__(NT, waves_with<PART>(6)) void clip_kernel(ClipPlan<PART, CAP, S> p) {
    const Starts<CAP> starts(p.s, p.parts);
    for (int c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const int part = __builtin_amdgcn_readfirstlane(starts.part_of(c));
        const Shape s = shape_of(p.s[part]);
        const int chunk = c - starts.start_of(part);
        const float factor = factor_of(sum_of(p, p.first_device + (s.what >> 2)), p.most);
        const void* const in = p.s[part].in;
        void* const out = p.s[part].out;
        switch (s.what & 3) {
            case 0: clip_chunk<STREAM, T_F32, T_F32>(in, out, s, chunk, factor); break;
            case 1: clip_chunk<STREAM, T_BF16, T_F32>(in, out, s, chunk, factor); break;
            case 2: clip_chunk<STREAM, T_F32, T_BF16>(in, out, s, chunk, factor); break;
            default: clip_chunk<STREAM, T_BF16, T_BF16>(in, out, s, chunk, factor);
        }
    }
    if (p.norm[0] && blockIdx.x == 0 && (int)threadIdx.x < p.k) *p.norm[threadIdx.x] = sqrtf(sum_of(p, threadIdx.x));
}

}  // namespace

template <template <bool> class PART, int CAP>
int32_t launch_square_sum(const SquarePlan<PART, CAP>& plan, int devices, int blocks, hipStream_t stream) {
    const dim3 grid((uint32_t)blocks, (uint32_t)devices);
    if (plan.stream) hipLaunchKernelGGL((square_sum_kernel<true, PART, CAP>), grid, dim3(NT), 0, stream, plan);
    else hipLaunchKernelGGL((square_sum_kernel<false, PART, CAP>), grid, dim3(NT), 0, stream, plan);
    return launch_status(__func__);
}
template <int S>
int32_t launch_square_join(const SquareJoin<S>& join, int32_t k, hipStream_t stream) {
    hipLaunchKernelGGL(square_join_kernel<S>, dim3((uint32_t)k), dim3(NT), 0, stream, join);
    return launch_status(__func__);
}
template <template <bool> class PART, int CAP, int S>
int32_t launch_clip(const ClipPlan<PART, CAP, S>& plan, hipStream_t stream) {
    // a chunk a workgroup: they end at different times, and their stores drain beside others' loads (2^28 elements from bf16 to fp32, us a call with the sum
    // of squares: 2048 workgroups 411, 8192 403, 32768 386)
    const int blocks = std::max(1, std::min<int>(plan.chunks, 1 << 20));
    if (plan.stream) hipLaunchKernelGGL((clip_kernel<true, PART, CAP, S>), dim3((uint32_t)blocks), dim3(NT), 0, stream, plan);
    else hipLaunchKernelGGL((clip_kernel<false, PART, CAP, S>), dim3((uint32_t)blocks), dim3(NT), 0, stream, plan);
    return launch_status(__func__);
}

template int32_t launch_square_sum(const SquarePlan<DensePart, LIST_FEW>&, int, int, hipStream_t);
template int32_t launch_square_sum(const SquarePlan<DensePart, LIST_SOME>&, int, int, hipStream_t);
template int32_t launch_square_sum(const SquarePlan<DensePart, LIST_DENSE>&, int, int, hipStream_t);
template int32_t launch_square_sum(const SquarePlan<PitchedPart, LIST_FEW>&, int, int, hipStream_t);
template int32_t launch_square_sum(const SquarePlan<PitchedPart, LIST_PITCHED>&, int, int, hipStream_t);
template int32_t launch_square_join(const SquareJoin<8>&, int32_t, hipStream_t);
template int32_t launch_square_join(const SquareJoin<SBP_MAX_K>&, int32_t, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_FEW, 8>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_FEW, SBP_MAX_K>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_SOME, 8>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_SOME, SBP_MAX_K>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_DENSE, 8>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<DensePart, LIST_DENSE, SBP_MAX_K>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<PitchedPart, LIST_FEW, 8>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<PitchedPart, LIST_FEW, SBP_MAX_K>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<PitchedPart, LIST_PITCHED, 8>&, hipStream_t);
template int32_t launch_clip(const ClipPlan<PitchedPart, LIST_PITCHED, SBP_MAX_K>&, hipStream_t);

}  // namespace sbp
