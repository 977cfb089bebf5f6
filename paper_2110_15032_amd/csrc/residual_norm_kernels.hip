// What stands between two blocks: the norm behind a block, its gate, the residual, and the norm in front of the next block.
//
//   t = norm1(x),  h = alpha r + gate t,  y = norm2(h)
//   norm(v) = (v - mean) rstd gamma + beta,  mean = sum v / n (RMS: 0),  rstd = 1 / sqrt(sum (v - mean)^2 / n + eps)
//
// Bound by HBM: a row of x and r is read once and stays in registers until h and y are written, TPR threads a row with V vectors of eight
// elements each.  y is computed from h before its rounding.  A wave's lanes hold consecutive vectors, so that loads and stores are of consecutive bytes, and a
// row never leaves its threads: one pass, two barriers a row (its two sums over waves).  8 devices, 8192 x 4096: bf16 around an fp32 residual 79 us (403 MB, 5.1
// TB/s), all bf16 53 (268 MB); 1 x 4096 3.3 on the device.  One row ahead: two and three gained nothing, and loads past the caches 3 % where HBM has
// the inputs and lost 13 % where the memory-side cache has (2048 x 4096, 13.9 / 15.7).  Rows of more than 8192 read a vector's weights when they need them: 4096 x 12288
// bf16 102 (3.9 TB/s; with all weights of a lane at a time, which spill, 146).
#include "row_device.h"

namespace sbp {
namespace {

// Workgroups of 256 threads of a launch: eight rows for every group of threads, as the weights are read once a workgroup, between so many (for few rows) and so
// many.  us, 16 rows / 8 / 4: 8 devices, bf16, 65536 x 512 58.2 / 52.7 / 48.7, 32768 x 1024 63.0 / 54.9 / 54.1, 16384 x 2048 50.1 / 47.3 / 47.7, 8192 x 4096 53.9 / 55.4 / 60.1 (fp32
// residual 87.9 / 78.5 / 77.6).
constexpr int NORM_BLOCKS = 1024, NORM_MOST_BLOCKS = 4096;

template <int XT, int RT, int YT, int TPR, int V, int S>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void residual_norm_kernel(ResNormPlan<S> p) {
    constexpr int NT = TPR < 256 ? 256 : TPR, G = NT / TPR, NW = TPR / 64, N = V * 8;
    constexpr int AHEAD = 1;   // rows on their way
    constexpr bool KEEP = V == 1;   // weights stay in registers; else they are read again for every row, from the caches
    const ResNormShard& s = p.s[S > 1 ? blockIdx.y : 0];
    const int t = threadIdx.x % TPR, group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0, cols = p.cols;   // whole waves
    const bool post = p.flags & RN_POST, pre = p.flags & RN_PRE, narrow_weights = p.flags & RN_BF16_WEIGHTS;
    __shared__ float2 part[2][2][G][NW];
    const RowPart<TPR, V> part_of_row(t, cols);
    float gate[8], gamma1[8], beta1[8], gamma2[8], beta2[8];   // of one vector
    auto column = [&](int v) __attribute__((always_inline)) {   // not KEEP: opaque, or addresses would be held in registers from row to row
        int c = (v * TPR + t) * 8;
        if constexpr (!KEEP) asm volatile("" : "+v"(c));
        return c;
    };
    auto load1 = [&](int v) __attribute__((always_inline)) {
        const int c = column(v);
        load_weight8(s.gate, narrow_weights, c, cols, 1.0f, gate);
        if (post) {
            load_weight8(s.gamma1, narrow_weights, c, cols, 1.0f, gamma1);
            load_weight8(s.beta1, narrow_weights, c, cols, 0.0f, beta1);
        }
    };
    auto load2 = [&](int v) __attribute__((always_inline)) {
        const int c = column(v);
        load_weight8(s.gamma2, narrow_weights, c, cols, 1.0f, gamma2);
        load_weight8(s.beta2, narrow_weights, c, cols, 0.0f, beta2);
    };
    if constexpr (KEEP) {
        load1(0);
        if (pre) load2(0);
    }

    const int step = gridDim.x * G;
    Raw8<XT> next_x[AHEAD][V];
    Raw8<RT> next_r[AHEAD][V];
    auto fetch = [&](int a, int64_t row) __attribute__((always_inline)) {
        const char* const from_x = static_cast<const char*>(s.x) + row * s.ldx * bytes_of<XT>;
        const char* const from_r = static_cast<const char*>(s.r) + row * s.ldr * bytes_of<RT>;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = column(v);
            next_x[a][v] = load8<XT>(from_x, c, row < s.rows ? cols : 0);
            next_r[a][v] = load8<RT>(from_r, c, row < s.rows ? cols : 0);
        }
    };
    int64_t row = (int64_t)blockIdx.x * G + group;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(a, row + a * step);
    auto work = [&](int a, int turn) __attribute__((always_inline)) {   // one row of every group, and the row AHEAD of it on its way
        float x[N], h[N];
        if (!part_of_row.even) {
            asm volatile("");   // or all of it would be worked out, and chosen from
            const int there = row < s.rows ? cols : 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = column(v);
                next_x[a][v] = settle8<XT>(next_x[a][v], c, there);
                next_r[a][v] = settle8<RT>(next_r[a][v], c, there);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float u[8], w[8];
            widen<XT>(next_x[a][v], 1.0f, u);
            widen<RT>(next_r[a][v], 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[v * 8 + e] = u[e];
                h[v * 8 + e] = p.alpha * w[e];
            }
        }
        fetch(a, row + AHEAD * step);
        float mean = 0.0f, rstd = 1.0f, m2;
        if (post) {
            part_of_row.spread(x, p.flags & RN_POST_LAYER, part[turn][0][group], mean, m2);
            rstd = inverse_root(fmaf(m2, part_of_row.over, p.eps1));
            if (t == 0 && row < s.rows) {
                if (s.mean1) s.mean1[row] = mean;
                if (s.rstd1) s.rstd1[row] = rstd;
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = column(v);
            if constexpr (!KEEP) {
                __builtin_amdgcn_sched_barrier(0);   // one vector's weights at a time, for their registers
                load1(v);
            }
            float u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = v * 8 + e;
                if (post) x[i] = fmaf((x[i] - mean) * rstd, gamma1[e], beta1[e]);
                u[e] = h[i] = fmaf(gate[e], x[i], h[i]);
            }
            if (row < s.rows) store8<RT>(static_cast<char*>(s.h) + (row * s.ldh + c) * bytes_of<RT>, narrow<RT>(u), cols - c, p.flags & RN_STREAM_H);
        }
        if (!pre) return;
        if (!part_of_row.whole) part_of_row.clear(h, cols);   // behind the row's end gate is 0, but x need not be finite there times it
        part_of_row.spread(h, p.flags & RN_PRE_LAYER, part[turn][1][group], mean, m2);
        rstd = inverse_root(fmaf(m2, part_of_row.over, p.eps2));
        if (row >= s.rows) return;
        if (t == 0) {
            if (s.mean2) s.mean2[row] = mean;
            if (s.rstd2) s.rstd2[row] = rstd;
        }
        float y[V][8];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (!KEEP) {
                __builtin_amdgcn_sched_barrier(0);
                load2(v);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) y[v][e] = fmaf((h[v * 8 + e] - mean) * rstd, gamma2[e], beta2[e]);
        }
        char* const to = static_cast<char*>(s.y) + row * s.ldy * bytes_of<YT>;
        if constexpr (bytes_of<YT> == 1) {
            if (!part_of_row.whole) {   // a block's largest magnitude is of elements alone
                asm volatile("");
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[v][e] = (v * TPR + t) * 8 + e < cols ? y[v][e] : 0.0f;
            }
            Raw8<YT> q[V];
            uint32_t byte[V];
            narrow_blocks<true, YT>(y, q, byte);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = column(v);
                store8<YT>(to + c, q[v], cols - c, p.flags & RN_STREAM_Y);
                if ((t & 15) == 0 && c < cols) static_cast<uint8_t*>(s.y_scales)[row * s.lds + c / F8_BLOCK] = (uint8_t)byte[v];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = column(v);
                store8<YT>(to + c * bytes_of<YT>, narrow<YT>(y[v]), cols - c, p.flags & RN_STREAM_Y);
            }
        }
    };
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * G; first < s.rows;) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (first >= s.rows) break;
            work(a, turn);
            first += step;
            row += step;
            turn ^= 1;
        }
    }
}

}  // namespace

template <int S>
int32_t launch_residual_norm(const ResNormPlan<S>& given, int n, int32_t x_type, int32_t r_type, int32_t y_type, hipStream_t stream) {
    ResNormPlan<S> plan = given;
    int64_t rows = 0, all = 0;
    bool h_lines = true, y_lines = true;
    for (int i = 0; i < n; ++i) {
        rows = std::max<int64_t>(rows, plan.s[i].rows);
        all += plan.s[i].rows;
        if ((int64_t)plan.s[i].ldh * bytes_of_type(r_type) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].h) % 128) h_lines = false;
        if ((int64_t)plan.s[i].ldy * bytes_of_type(y_type) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].y) % 128) y_lines = false;
    }
    const int64_t elements = all * plan.cols;
    if (streams_of(0, elements * bytes_of_type(r_type), h_lines, r_type) & STREAM_OUT) plan.flags |= RN_STREAM_H;
    if (streams_of(0, elements * bytes_of_type(y_type), y_lines, y_type) & STREAM_OUT) plan.flags |= RN_STREAM_Y;
    with_wide_type(x_type, [&](auto x) {
        with_wide_type(r_type, [&](auto r) {
            with_any_type(y_type, [&](auto y) {
                auto go = [&](auto tpr, auto v) {
                    constexpr int NT = tpr() < 256 ? 256 : tpr(), G = NT / tpr();
                    const int64_t some = NORM_BLOCKS * 256 / NT / n, most = v() == 1 ? NORM_MOST_BLOCKS * 256 / NT / n : some, turns = (rows + G - 1) / G;
                    const int64_t bx = std::max<int64_t>(1, std::min(turns, std::max(some, std::min(most, turns / 8))));
                    hipLaunchKernelGGL((residual_norm_kernel<x(), r(), y(), tpr(), v(), S>), dim3((uint32_t)bx, (uint32_t)n), dim3(NT), 0, stream, plan);
                };
                using std::integral_constant;
                if (plan.cols <= 512) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 1024) go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 2048) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 4096) go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
                else if (plan.cols <= 8192) go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
                else go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
            });
        });
    });
    return launch_status(__func__);
}
template int32_t launch_residual_norm<1>(const ResNormPlan<1>&, int, int32_t, int32_t, int32_t, hipStream_t);
template int32_t launch_residual_norm<RESNORM_SHARDS>(const ResNormPlan<RESNORM_SHARDS>&, int, int32_t, int32_t, int32_t, hipStream_t);

}  // namespace sbp
