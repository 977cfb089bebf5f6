// Rows of up to 16384 elements in the registers of TPR threads, V vectors of eight elements each, vector v of thread t from column
// 8 (v TPR + t) on; what lies behind a row's end is 0.
#pragma once
#include "block8_device.h"

namespace sbp {
namespace {

// Eight elements of a weight from column c on; `otherwise` where there is no weight.  bf16: its type (uniform).
__device__ inline void load_weight8(const void* w, bool bf16, int c, int cols, float otherwise, float (&out)[8]) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = c + e < cols ? otherwise : 0.0f;
    } else if (bf16) {
        widen<T_BF16>(settle8<T_BF16>(load8<T_BF16>(static_cast<const char*>(w), c, cols), c, cols), 1.0f, out);
    } else {
        widen<T_F32>(settle8<T_F32>(load8<T_F32>(static_cast<const char*>(w), c, cols), c, cols), 1.0f, out);
    }
}
// all of a lane's
template <int V, int TPR>
__device__ inline void load_column(const void* w, bool bf16, int t, int cols, float otherwise, float (&out)[V * 8]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float u[8];
        load_weight8(w, bf16, (v * TPR + t) * 8, cols, otherwise, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) out[v * 8 + e] = u[e];
    }
}

// 1 / sqrt: the hardware's, to a unit in the last place, which takes subnormal numbers for zero
__device__ inline float inverse_root(float v) {
    if (v < 1e-37f) {
        asm volatile("");
        return 1.0f / sqrtf(v);
    }
    return __builtin_amdgcn_rsqf(v);
}

// a / n, over = 1 / n: the product put right by its remainder, which gives the nearest number, so that the mean of equal values is their value
__device__ inline float quotient(float a, float n, float over) {
    const float q = a * over, r = fmaf(fmaf(-q, n, a), over, q);
    return fabsf(q) < INFINITY ? r : q;
}

// the sum of N neighbouring lanes' numbers (1, 2, 4, 8 or 16) on each of them
template <int N>
__device__ inline float sum_lanes(float v) {
    if constexpr (N > 1) v += dpp<0xB1>(v);
    if constexpr (N > 2) v += dpp<0x4E>(v);
    if constexpr (N > 4) v += dpp<0x141>(v);
    if constexpr (N > 8) v += dpp<0x140>(v);
    return v;
}

// Where a lane's part of a row lies.
template <int TPR, int V>
struct RowPart {
    static constexpr int NW = TPR / 64;
    int t, cols;
    bool whole;        // no lane is without elements
    bool even;         // no lane has fewer than eight of a vector without having none
    float of_wave, over_wave;   // elements of this lane's wave
    float elements;    // of wave t % NW
    float over;        // 1 / cols
    __device__ RowPart(int t_, int cols_) : t(t_), cols(cols_) {
        int have = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) have += min(max(cols - (v * TPR + t) * 8, 0), 8);
        whole = cols == TPR * V * 8;
        even = cols % 8 == 0;
        of_wave = sum_wave((float)have);
        over_wave = of_wave > 0.0f ? 1.0f / of_wave : 0.0f;
        over = 1.0f / (float)cols;
        elements = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) elements += (float)min(max(cols - (v * TPR + (t & (NW - 1)) * 64) * 8, 0), 512);
    }

    // 0 where no element is, which a row of `upto` elements ends in front of; not for `whole` ones.
    __device__ inline void clear(float (&x)[V * 8], int upto) const {
        if (even) {
            asm volatile("");   // or both would be worked out, and one chosen
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const bool is = (v * TPR + t) * 8 < upto;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v * 8 + e] = is ? x[v * 8 + e] : 0.0f;
            }
        } else {
            asm volatile("");
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int left = upto - (v * TPR + t) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v * 8 + e] = e < left ? x[v * 8 + e] : 0.0f;
            }
        }
    }

    // Mean and sum of the squares of the distances to it (RMS, layer = false: 0 and the sum of squares), exact to fp32 sums whatever the row's
    // offset: every wave sums its elements, then the squares of their distances from its own mean, and the waves' pairs are joined with the
    // distances of their means, a pair a lane.  One barrier; `part` is not written again before another one.
    __device__ inline void spread(const float (&x)[V * 8], bool layer, float2* part, float& mean, float& m2) const {
        float centre = 0.0f;
        if (layer) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V * 8; ++i) sum += x[i];
            centre = quotient(sum_wave(sum), of_wave, over_wave);
        }
        float sq = 0.0f;
        if (whole || !layer) {
#pragma unroll
            for (int i = 0; i < V * 8; ++i) {
                const float d = x[i] - centre;
                sq = fmaf(d, d, sq);
            }
        } else {
            float d[V * 8];
#pragma unroll
            for (int i = 0; i < V * 8; ++i) d[i] = x[i] - centre;
            clear(d, cols);
#pragma unroll
            for (int i = 0; i < V * 8; ++i) sq = fmaf(d[i], d[i], sq);
        }
        sq = sum_wave(sq);
        mean = centre;
        m2 = sq;
        if constexpr (NW > 1) {
            if ((t & 63) == 0) part[t >> 6] = float2{centre, sq};
            __syncthreads();
            const float2 of_one = part[t & (NW - 1)];
            mean = layer ? quotient(sum_lanes<NW>(of_one.x * elements), (float)cols, over) : 0.0f;
            const float d = of_one.x - mean;
            m2 = sum_lanes<NW>(fmaf(elements * d, d, of_one.y));
        }
    }

    // Two sums over the row at once.  One barrier, as above.
    __device__ inline void sums(float& a, float& b, float2* part) const {
        a = sum_wave(a);
        b = sum_wave(b);
        if constexpr (NW > 1) {
            if ((t & 63) == 0) part[t >> 6] = float2{a, b};
            __syncthreads();
            const float2 of_one = part[t & (NW - 1)];
            a = sum_lanes<NW>(of_one.x);
            b = sum_lanes<NW>(of_one.y);
        }
    }
};

template <typename F>
void with_wide_type(int32_t dtype, F&& f) {
    if (dtype == SBP_F32) f(std::integral_constant<int, T_F32>{});
    else f(std::integral_constant<int, T_BF16>{});
}
template <typename F>
void with_any_type(int32_t dtype, F&& f) {
    if (dtype == SBP_F8E4M3) f(std::integral_constant<int, T_E4M3>{});
    else if (dtype == SBP_F8E5M2) f(std::integral_constant<int, T_E5M2>{});
    else with_wide_type(dtype, f);
}
inline int bytes_of_type(int32_t dtype) { return dtype == SBP_F32 ? 4 : dtype == SBP_BF16 ? 2 : 1; }

}  // namespace
}  // namespace sbp
