// Layer normalisation over rows and its gradient.
//
//   y = (x - mean) rstd gamma + beta,  mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)
//   xhat = (x - mean) rstd,  g = dy gamma,  dx = rstd (g - sum g / n - xhat sum (g xhat) / n),  dgamma = sum over rows dy xhat,  dbeta = sum dy
//
// Both are bound by HBM: a row is read once and stays in registers, TPR threads a row with V vectors of eight elements each.  A workgroup
// walks over rows, so that gamma and beta are read once, and reads the next row before it works on this one.  Measured: 8192 x 4096 on eight devices
// from bf16 to 8 bits (101 MB) 22.7 us, 4.5 TB/s; the gradient of 16384 x 4096 on eight devices, x in 8 bits (336 MB), 74 us, 4.5 TB/s.
#include "block8_device.h"

namespace sbp {
namespace {

// Workgroups of 256 threads of a launch, so that every compute unit has several (8192 x 4096 in bf16 into 8 bits on one device, without statistics,
// us: 512 24.9, 1024 20.5, 2048 22.7; 2048 x 16384 38.6, 24.0, 27.5).
constexpr int NORM_BLOCKS = 1024;
constexpr int GRAD_NT = 512;

template <int WT, int V, int TPR>
__device__ inline void load_weight(const void* w, int t, int cols, float otherwise, float (&out)[V * 8]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * TPR + t) * 8;
        float u[8];
        if (w) {
            widen<WT>(settle8<WT>(load8<WT>(static_cast<const char*>(w), c, cols), c, cols), 1.0f, u);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = c + e < cols ? otherwise : 0.0f;   // zeros behind the row's end, as load8 gives
        }
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

// the sum of N neighbouring lanes' numbers (4, 8 or 16) on each of them
template <int N>
__device__ inline float sum_lanes(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    if constexpr (N > 4) v += dpp<0x141>(v);
    if constexpr (N > 8) v += dpp<0x140>(v);
    return v;
}

// The statistics are exact to fp32 sums whatever the row's offset: every wave sums its elements, then the squares of their distances from
// its own mean, and the waves' pairs are joined with the distances of their means (one exchange for both, and a pair a lane, as sixteen pairs in every
// lane's registers spilled).  y goes by the distance to the mean, as the gradient does: mean * rstd has a rounding that x * rstd does not take
// back, up to 2^-24 |mean| rstd.
template <int XT, int YT, int WT, int TPR, int V>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(NormPlan p) {
    constexpr int NT = TPR < 256 ? 256 : TPR, G = NT / TPR, NW = TPR / 64;
    const NormShard& s = p.s[blockIdx.y];
    const int t = threadIdx.x % TPR, group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0, wave = t >> 6, cols = p.cols;   // whole waves
    __shared__ float2 part[2][NW];
    float gamma[V * 8], beta[V * 8];
    load_weight<WT, V, TPR>(s.gamma, t, cols, 1.0f, gamma);
    load_weight<WT, V, TPR>(s.beta, t, cols, 0.0f, beta);
    int have = 0;   // elements of this lane
#pragma unroll
    for (int v = 0; v < V; ++v) have += min(max(cols - (v * TPR + t) * 8, 0), 8);
    const bool whole = cols == TPR * V * 8;   // no lane is without elements
    const float of_wave = sum_wave((float)have), over_wave = of_wave > 0.0f ? 1.0f / of_wave : 0.0f, over = 1.0f / (float)cols;
    float elements = 0.0f;   // of wave t % NW
#pragma unroll
    for (int v = 0; v < V; ++v) elements += (float)min(max(cols - (v * TPR + (t & (NW - 1)) * 64) * 8, 0), 512);

    // AHEAD rows on their way
    constexpr int AHEAD = XT == T_F32 ? 1 : 2;
    const int step = gridDim.x * G;
    Raw8<XT> next[AHEAD][V];
    auto fetch = [&](Raw8<XT> (&to)[V], int64_t row) {
        const char* const from = static_cast<const char*>(s.x) + row * s.ldx * bytes_of<XT>;
#pragma unroll
        for (int v = 0; v < V; ++v) to[v] = load8<XT>(from, (v * TPR + t) * 8, row < s.rows ? cols : 0);
    };
    int64_t row = (int64_t)blockIdx.x * G + group;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(next[a], row + a * step);
    int turn = 0;
    auto work = [&](Raw8<XT> (&raw)[V]) {   // one row of every group, and the row AHEAD of it on its way
        float x[V * 8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float u[8];
            const int c = (v * TPR + t) * 8;
            widen<XT>(whole ? raw[v] : settle8<XT>(raw[v], c, row < s.rows ? cols : 0), 1.0f, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[v * 8 + e] = u[e];
        }
        fetch(raw, row + AHEAD * step);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V * 8; ++i) sum += x[i];
        sum = sum_wave(sum);
        const float centre = quotient(sum, of_wave, over_wave);
        float sq = 0.0f;
        if (whole) {
#pragma unroll
            for (int i = 0; i < V * 8; ++i) {
                const float d = x[i] - centre;
                sq = fmaf(d, d, sq);
            }
        } else {
            asm volatile("");   // or both would be worked out, and one chosen
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int left = cols - (v * TPR + t) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float d = e < left ? x[v * 8 + e] - centre : 0.0f;
                    sq = fmaf(d, d, sq);
                }
            }
        }
        sq = sum_wave(sq);
        float mean = centre, m2 = sq;
        if constexpr (NW > 1) {
            if ((threadIdx.x & 63) == 0) part[turn][wave] = float2{centre, sq};
            __syncthreads();   // one a row: the other half is written next, and this one again only behind the next barrier
            const float2 of_one = part[turn][t & (NW - 1)];   // of a wave to each lane, and sums over NW lanes
            mean = quotient(sum_lanes<NW>(of_one.x * elements), (float)cols, over);
            const float d = of_one.x - mean;
            m2 = sum_lanes<NW>(fmaf(elements * d, d, of_one.y));
        }
        const float rstd = inverse_root(fmaf(m2, over, p.eps));
        if (row >= s.rows) return;
        if (t == 0 && s.mean) {
            s.mean[row] = mean;
            s.rstd[row] = rstd;
        }
        float y[V][8];   // behind the row's end gamma and beta are 0, and y is
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[v][e] = fmaf((x[v * 8 + e] - mean) * rstd, gamma[v * 8 + e], beta[v * 8 + e]);
        char* const to = static_cast<char*>(s.y) + row * s.ldy * bytes_of<YT>;
        if constexpr (bytes_of<YT> == 1) {
            Raw8<YT> q[V];
            uint32_t byte[V];
            narrow_blocks<true, YT>(y, q, byte);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * TPR + t) * 8;
                store8<YT>(to + c, q[v], cols - c, p.streams & STREAM_OUT);
                if ((t & 15) == 0 && c < cols) static_cast<uint8_t*>(s.y_scales)[row * s.lds + c / F8_BLOCK] = (uint8_t)byte[v];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * TPR + t) * 8;
                store8<YT>(to + c * bytes_of<YT>, narrow<YT>(y[v]), cols - c, p.streams & STREAM_OUT);
            }
        }
    };
    for (int64_t first = (int64_t)blockIdx.x * G; first < s.rows;) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (first >= s.rows) break;
            work(next[a]);
            first += step;
            row += step;
            turn ^= 1;
        }
    }
}

// One partial sum of the weights' gradients for every workgroup, in the order of its rows; where a shard has one workgroup, that is the result.
// GROUPS rows of TPR threads side by side in a workgroup: their sums meet in LDS at the end, so that fewer partial sums go to memory.
template <int XT, int YT, int WT, int TPR, int V>
__global__ __launch_bounds__(GRAD_NT, TPR == 512 ? 2 : 4) void norm_grad_kernel(NormGradPlan p) {
    constexpr int G = GRAD_NT / TPR, NW = TPR / 64, CAP = TPR * V * 8;
    const NormGradShard& s = p.s[blockIdx.y];
    if ((int)blockIdx.x >= s.blocks) return;
    const int t = threadIdx.x % TPR, group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0, wave = t >> 6, cols = p.cols;   // whole waves
    __shared__ float2 part[2][G][NW];
    float gamma[V * 8], dgamma[V * 8], dbeta[V * 8];
    load_weight<WT, V, TPR>(s.gamma, t, cols, 1.0f, gamma);
#pragma unroll
    for (int i = 0; i < V * 8; ++i) dgamma[i] = dbeta[i] = 0.0f;
    const float over = 1.0f / (float)cols;

    const int step = s.blocks * G;
    Raw8<XT> next_x[V];
    Raw8<YT> next_dy[V];
    uint32_t next_byte[V];
    float next_mean = 0.0f, next_rstd = 0.0f;
    const bool whole = cols == TPR * V * 8;   // no lane is without elements
    auto fetch = [&](int64_t row) {
        const bool there = row < s.rows;
        const char* const from_x = static_cast<const char*>(s.x) + row * s.ldx * bytes_of<XT>;
        const char* const from_dy = static_cast<const char*>(s.dy) + row * s.lddy * bytes_of<YT>;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + t) * 8;
            next_x[v] = load8<XT>(from_x, c, there ? cols : 0);
            next_dy[v] = load8<YT>(from_dy, c, there ? cols : 0);
            next_byte[v] = 127;
            if constexpr (bytes_of<XT> == 1)
                if (there && c < cols) next_byte[v] = static_cast<const uint8_t*>(s.x_scales)[row * s.lds + c / F8_BLOCK];
        }
        next_mean = there ? s.mean[row] : 0.0f;
        next_rstd = there ? s.rstd[row] : 0.0f;
    };
    int64_t row = (int64_t)blockIdx.x * G + group;
    fetch(row);
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * G; first < s.rows; first += step, row += step, turn ^= 1) {
        float xhat[V * 8], dy[V * 8];
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float u[8], w[8];
            const int c = (v * TPR + t) * 8, there = row < s.rows ? cols : 0;
            widen<XT>(whole ? next_x[v] : settle8<XT>(next_x[v], c, there), scale_of(next_byte[v]), u);
            widen<YT>(whole ? next_dy[v] : settle8<YT>(next_dy[v], c, there), 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {   // dy is 0 where there is no element, mean and rstd where there is no row
                xhat[v * 8 + e] = (u[e] - mean) * rstd;
                dy[v * 8 + e] = w[e];
            }
        }
        if (!whole) {   // where no element is, mean * rstd may be infinite, and times 0 NaN
            asm volatile("");   // or it would be chosen from always
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) xhat[v * 8 + e] = (v * TPR + t) * 8 + e < cols ? xhat[v * 8 + e] : 0.0f;
        }
        fetch(row + step);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < V * 8; ++i) {
            const float g = dy[i] * gamma[i];
            s1 += g;
            s2 = fmaf(g, xhat[i], s2);
            dgamma[i] = fmaf(dy[i], xhat[i], dgamma[i]);
            dbeta[i] += dy[i];
        }
        s1 = sum_wave(s1);
        s2 = sum_wave(s2);
        if constexpr (NW > 1) {
            if ((threadIdx.x & 63) == 0) part[turn][group][wave] = float2{s1, s2};
            __syncthreads();   // one a row, as in norm_kernel
            s1 = s2 = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                s1 += part[turn][group][w].x;
                s2 += part[turn][group][w].y;
            }
        }
        s1 *= over;
        s2 *= over;
        if (row >= s.rows) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + t) * 8;
            float d[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = v * 8 + e;
                d[e] = rstd * (fmaf(dy[i], gamma[i], -s1) - xhat[i] * s2);
            }
            store8<YT>(static_cast<char*>(s.dx) + (row * s.lddx + c) * bytes_of<YT>, narrow<YT>(d), cols - c, p.streams & STREAM_OUT);
        }
    }
    if (!s.dgamma) return;
    float* const to_gamma = s.blocks > 1 ? s.part + (int64_t)blockIdx.x * 2 * cols : s.dgamma;
    float* const to_beta = s.blocks > 1 ? to_gamma + cols : s.dbeta;
    if constexpr (G > 1) {
        __shared__ float sums[G][2][CAP];
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[group][0][(v * TPR + t) * 8 + e] = dgamma[v * 8 + e];
                sums[group][1][(v * TPR + t) * 8 + e] = dbeta[v * 8 + e];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += GRAD_NT) {
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                a += sums[g][0][c];
                b += sums[g][1][c];
            }
            to_gamma[c] = a;
            to_beta[c] = b;
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + t) * 8;
            Raw8<T_F32> a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a.a[e] = dgamma[v * 8 + e];
                a.b[e] = dgamma[v * 8 + 4 + e];
                b.a[e] = dbeta[v * 8 + e];
                b.b[e] = dbeta[v * 8 + 4 + e];
            }
            store8<T_F32>(to_gamma + c, a, cols - c);
            store8<T_F32>(to_beta + c, b, cols - c);
        }
    }
}

// The partial sums of a shard's workgroups joined in order: 32 columns a workgroup, eight runs of partial sums side by side.
__global__ __launch_bounds__(256) void norm_grad_join_kernel(NormGradPlan p) {
    const NormGradShard& s = p.s[blockIdx.y];
    if (s.blocks <= 1) return;
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, width = 2 * p.cols;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float a = 0.0f;
    if (c < width) {
        const float* part = s.part + c;
        for (int b = run; b < s.blocks; b += 64) {   // eight on their way, past the end the last one again, which does not count
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = part[(int64_t)min(b + 8 * u, s.blocks - 1) * width];
#pragma unroll
            for (int u = 0; u < 8; ++u) a += b + 8 * u < s.blocks ? v[u] : 0.0f;
        }
    }
    sums[run][lane] = a;
    __syncthreads();
    if (run == 0 && c < width) {
        a = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) a += sums[r][lane];
        (c < p.cols ? s.dgamma : s.dbeta - p.cols)[c] = a;
    }
}

template <typename F>
void with_elem(int32_t dtype, F&& f) {
    if (dtype == SBP_F32) f(std::integral_constant<int, T_F32>{});
    else if (dtype == SBP_BF16) f(std::integral_constant<int, T_BF16>{});
    else if (dtype == SBP_F8E4M3) f(std::integral_constant<int, T_E4M3>{});
    else f(std::integral_constant<int, T_E5M2>{});
}
template <typename F>
void with_wide(int32_t dtype, F&& f) {
    if (dtype == SBP_F32) f(std::integral_constant<int, T_F32>{});
    else f(std::integral_constant<int, T_BF16>{});
}

int bytes_each(int32_t dtype) { return dtype == SBP_F32 ? 4 : dtype == SBP_BF16 ? 2 : 1; }

// threads of a row in the gradient: fp32 rows want one vector a thread (16384 x 2048, us: 128 threads 94.9, 256 80.8; bf16 43.5, 46.4), longer ones two
// (8192 x 4096 in bf16: 128 threads 50.9, 256 45.7, 512 47.9)
int grad_tpr(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 4096 ? 256 : 512; }

}  // namespace

int32_t launch_norm(const NormPlan& given, hipStream_t stream) {
    NormPlan plan = given;
    int64_t rows = 0, all = 0;
    bool on_lines = true;
    for (int i = 0; i < plan.k; ++i) {
        rows = std::max<int64_t>(rows, plan.s[i].rows);
        all += plan.s[i].rows;
        if ((int64_t)plan.s[i].ldy * bytes_each(plan.y_dtype) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].y) % 128) on_lines = false;
    }
    plan.streams = streams_of(all * plan.cols * bytes_each(plan.x_dtype), all * plan.cols * bytes_each(plan.y_dtype), on_lines, plan.y_dtype);
    with_wide(plan.x_dtype, [&](auto x) {
        with_elem(plan.y_dtype, [&](auto y) {
            with_wide(plan.w_dtype, [&](auto w) {
                auto go = [&](auto tpr, auto v) {
                    constexpr int NT = tpr() < 256 ? 256 : tpr(), G = NT / tpr();
                    const int64_t bx = std::max<int64_t>(1, std::min<int64_t>((rows + G - 1) / G, NORM_BLOCKS * 256 / NT / plan.k));
                    hipLaunchKernelGGL((norm_kernel<x(), y(), w(), tpr(), v()>), dim3((uint32_t)bx, (uint32_t)plan.k), dim3(NT), 0, stream, plan);
                };
                using std::integral_constant;
                // one wave a row needs no barrier; else two vectors a thread.  us, bf16 into 8 bits: 65536 x 512 one wave with one vector 20.7, two
                // (half of them without elements) 29.2, two waves 38.3; 32768 x 1024 one wave 20.3, two 21.4; 8192 x 4096 two waves 28.2, four 20.5, eight 23.0;
                // 2048 x 16384 eight 27.2, sixteen 24.0 (21.1 since their pairs are joined over lanes, and not by every lane)
                if (plan.cols <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 1024) go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
                else if (plan.cols <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
                else if (plan.cols <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
                else go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
            });
        });
    });
    return launch_status(__func__);
}

// One workgroup a compute unit of this chip, as each one writes a partial sum that has to be read again; two where the rows are short and many.  us, one /
// two: 1767 x 1001 in bf16 10.7 / 13.0, 8192 x 4096 42.8 / 45.7, 2048 x 16384 57.0 / 71.6, 16384 x 512 16.1 / 16.5; 8192 x 2048 26.1 / 24.6,
// 16384 x 2048 54.0 / 46.4, 65536 x 512 49.0 / 43.9.
int32_t norm_grad_blocks(int64_t rows, int64_t cols, int32_t k) {
    const int64_t g = GRAD_NT / grad_tpr(cols), most = cols <= 2048 && rows * cols * k >= (int64_t)1 << 24 ? 512 : 256;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + g - 1) / g, most / k));
}

int32_t launch_norm_grad(const NormGradPlan& given, hipStream_t stream) {
    NormGradPlan plan = given;
    int blocks = 1;
    bool join = false, on_lines = true;
    int64_t all = 0;
    for (int i = 0; i < plan.k; ++i) {
        all += plan.s[i].rows;
        if ((int64_t)plan.s[i].lddx * bytes_each(plan.dy_dtype) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].dx) % 128) on_lines = false;
        blocks = std::max(blocks, plan.s[i].blocks);
        join = join || (plan.s[i].blocks > 1 && plan.s[i].dgamma);
    }
    plan.streams = streams_of(all * plan.cols * (bytes_each(plan.x_dtype) + bytes_each(plan.dy_dtype)), all * plan.cols * bytes_each(plan.dy_dtype), on_lines, plan.dy_dtype);
    with_elem(plan.x_dtype, [&](auto x) {
        with_wide(plan.dy_dtype, [&](auto y) {
            with_wide(plan.w_dtype, [&](auto w) {
                auto go = [&](auto tpr, auto v) {
                    hipLaunchKernelGGL((norm_grad_kernel<x(), y(), w(), tpr(), v()>), dim3((uint32_t)blocks, (uint32_t)plan.k), dim3(GRAD_NT), 0, stream, plan);
                };
                using std::integral_constant;
                if (plan.cols <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 1024) go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 4096) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
                else if (plan.cols <= 8192) go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
                else go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
            });
        });
    });
    int32_t st = launch_status(__func__);
    if (st != SBP_OK || !join) return st;
    hipLaunchKernelGGL(norm_grad_join_kernel, dim3((uint32_t)((2 * plan.cols + 31) / 32), (uint32_t)plan.k), dim3(256), 0, stream, plan);
    return launch_status(__func__);
}

}  // namespace sbp
