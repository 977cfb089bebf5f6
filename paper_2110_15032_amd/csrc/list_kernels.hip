// The sum of squares of many tensors, and all of them times one factor: the norm of all gradients and their clipping.
//
//   s_i = sum over the tensors of x^2 over what device i counts,  norm = sqrt(sum of s_i),  out = x min(1, max_norm / norm)
//
// Both are bound by HBM.  A launch takes PARTS local tensors, which its argument block names; their vectors of eight elements are numbered
// through, a workgroup takes 1024 of them at a time (a chunk, of one tensor) and finds the tensor among the parts with one comparison a lane.
#include "block8_device.h"

namespace sbp {
namespace {

constexpr int NT = 256, PER = LIST_CHUNK / NT;

// A chunk's part: the last whose first chunk is not behind it.  Every lane looks at two of the first chunks (LIST_PARTS <= 128).
struct PartOf {
    int32_t a, b;
    __device__ PartOf(const ListPlan& p) {
        const int lane = threadIdx.x & 63;
        a = lane < p.parts ? p.first[lane] : INT32_MAX;
        b = lane + 64 < p.parts ? p.first[lane + 64] : INT32_MAX;
    }
    __device__ int operator()(int chunk) const {
        return __popcll(__builtin_amdgcn_ballot_w64(a <= chunk)) + __popcll(__builtin_amdgcn_ballot_w64(b <= chunk)) - 1;
    }
};

// Vector `off` of a chunk: row and first column, from the chunk's first vector on.
struct Place {
    int64_t row;     // of the chunk's first vector
    int64_t vector;  // in that row
    int32_t per_row;
    bool single;
    __device__ Place(const ListPart& s, int chunk) {
        const int64_t first = (int64_t)chunk * LIST_CHUNK;
        single = s.rows == 1;
        per_row = single ? 0 : (int32_t)((s.cols + 7) / 8);
        row = single ? 0 : first / per_row;
        vector = single ? first : first - row * per_row;
    }
};

// F(row, column, length of the row from the column that the pointer stands for on): of every vector of the chunk that exists.
template <typename F>
__device__ inline void each_vector(const ListPart& s, int chunk, F&& f) {
    const Place at(s, chunk);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int off = u * NT + (int)threadIdx.x;
        if (at.single) {   // columns counted from the chunk's start, as a row may be longer than 2^31
            const int64_t left = s.cols - at.vector * 8;
            f(u, (int64_t)0, at.vector * 8, off * 8, (int)(left < LIST_CHUNK * 8 + 8 ? left : LIST_CHUNK * 8 + 8));
        } else {
            uint32_t v = (uint32_t)at.vector + (uint32_t)off, r = 0;
            if (at.per_row > LIST_CHUNK) {
                if (v >= (uint32_t)at.per_row) {
                    v -= (uint32_t)at.per_row;
                    r = 1;
                }
            } else {
                r = v / (uint32_t)at.per_row;
                v -= r * (uint32_t)at.per_row;
            }
            const int64_t row = at.row + r;
            f(u, row, (int64_t)0, (int)v * 8, row < s.rows ? (int)s.cols : 0);
        }
    }
}

// Squares are summed in 64 bits: neither the number of elements nor their size loses anything before the sum is rounded to fp32, and
// the conversion and the fused product of eight elements cost less than loading them.  Lane, wave and workgroup sums in an order of the sizes alone.
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

template <int T>
__device__ inline void square_chunk(const ListPart& s, int chunk, double (&acc)[2]) {
    Raw8<T> raw[PER];
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) {
        raw[u] = load8<T>(static_cast<const char*>(s.in) + (row * s.ldi + from) * bytes_of<T>, c, cols);
    });
    each_vector(s, chunk, [&](int u, int64_t, int64_t, int c, int cols) {
        float v[8];
        widen<T>(settle8<T>(raw[u], c, cols), 1.0f, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e & 1] = fma((double)v[e], (double)v[e], acc[e & 1]);
    });
}

__global__ __launch_bounds__(NT) void square_sum_kernel(ListPlan p) {
    __shared__ double waves[NT / 64];
    const PartOf part_of(p);
    const int d = blockIdx.y;
    double acc[2] = {0.0, 0.0};
    for (int c = p.chunk0[d] + blockIdx.x; c < p.chunk0[d + 1]; c += gridDim.x) {
        const int part = __builtin_amdgcn_readfirstlane(part_of(c));
        const ListPart& s = p.s[part];
        const int chunk = c - p.first[part];
        if (s.types & 1) square_chunk<T_BF16>(s, chunk, acc);
        else square_chunk<T_F32>(s, chunk, acc);
    }
    const double sum = sum_block(acc[0] + acc[1], waves);
    if (threadIdx.x == 0) p.partial[(int64_t)p.slot[d] * gridDim.x + blockIdx.x] = sum;
}

// The partial sums of every device, joined in order and rounded once.
__global__ __launch_bounds__(NT) void square_join_kernel(SquareJoin p) {
    __shared__ double waves[NT / 64];
    const int d = blockIdx.x;
    const double* const part = p.partial + (int64_t)d * p.per_device;
    double v = 0.0;
    for (int i = threadIdx.x; i < p.count[d]; i += NT) v += part[i];
    v = sum_block(v, waves);
    if (threadIdx.x == 0) *p.out[d] = (float)v;
}

// The factor of a device's gradients.  A norm that is no number makes it NaN, an infinite one 0.
__device__ inline float sum_of(const ClipSum& p, int d) {
    if (!p.partial) return *p.sum[d];
    float v = *p.sum[0];
    for (int i = 1; i < p.k; ++i) v += *p.sum[i];   // in the order of the devices, as boxing adds
    return v;
}
__device__ inline float factor_of(float sum, float most) {
    const float norm = sqrtf(sum);
    return norm <= most ? 1.0f : most / norm;
}

template <int T, int U>
__device__ inline void clip_chunk(const ListPart& s, int chunk, float factor) {
    Raw8<T> raw[PER];
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) {
        raw[u] = load8<T>(static_cast<const char*>(s.in) + (row * s.ldi + from) * bytes_of<T>, c, cols);
    });
    each_vector(s, chunk, [&](int u, int64_t row, int64_t from, int c, int cols) {
        float v[8];
        widen<T>(settle8<T>(raw[u], c, cols), 1.0f, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= factor;
        if (c < cols) store8<U>(static_cast<char*>(s.out) + (row * s.ldo + from + c) * bytes_of<U>, narrow<U>(v), cols - c);
    });
}

__global__ __launch_bounds__(NT) void clip_kernel(ListPlan p, ClipSum sums) {
    const PartOf part_of(p);
    for (int c = blockIdx.x; c < p.chunk0[1]; c += gridDim.x) {
        const int part = __builtin_amdgcn_readfirstlane(part_of(c));
        const ListPart& s = p.s[part];
        const int chunk = c - p.first[part];
        const float factor = factor_of(sum_of(sums, s.types >> 2), sums.most);
        switch (s.types & 3) {
            case 0: clip_chunk<T_F32, T_F32>(s, chunk, factor); break;
            case 1: clip_chunk<T_BF16, T_F32>(s, chunk, factor); break;
            case 2: clip_chunk<T_F32, T_BF16>(s, chunk, factor); break;
            default: clip_chunk<T_BF16, T_BF16>(s, chunk, factor);
        }
    }
    if (sums.norm[0] && blockIdx.x == 0 && (int)threadIdx.x < sums.k) *sums.norm[threadIdx.x] = sqrtf(sum_of(sums, threadIdx.x));
}

}  // namespace

int32_t launch_square_sum(const ListPlan& plan, int devices, int blocks, hipStream_t stream) {
    hipLaunchKernelGGL(square_sum_kernel, dim3((uint32_t)blocks, (uint32_t)devices), dim3(NT), 0, stream, plan);
    return launch_status(__func__);
}
int32_t launch_square_join(const SquareJoin& join, int32_t k, hipStream_t stream) {
    hipLaunchKernelGGL(square_join_kernel, dim3((uint32_t)k), dim3(NT), 0, stream, join);
    return launch_status(__func__);
}
int32_t launch_clip(const ListPlan& plan, const ClipSum& sums, hipStream_t stream) {
    const int blocks = std::max(1, std::min<int>(plan.chunk0[1], LIST_BLOCKS));
    hipLaunchKernelGGL(clip_kernel, dim3((uint32_t)blocks), dim3(NT), 0, stream, plan, sums);
    return launch_status(__func__);
}

}  // namespace sbp
