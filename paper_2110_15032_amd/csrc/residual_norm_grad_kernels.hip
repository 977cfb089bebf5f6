// The gradient of what stands between two blocks (residual_norm_kernels.hip).  With hhat = (h - mean2) rstd2, xhat = (x - mean1) rstd1,
//
//   d = dh + rstd2 (g - sum g / n - hhat sum (g hhat) / n),  g = dy gamma2          (RMS: without sum g)
//   dr = alpha d,  e = gate gamma1 d,  dx = rstd1 (e - sum e / n - xhat sum (e xhat) / n)
//   A = sum over rows d xhat,  B = sum d,  C = sum dy hhat,  D = sum dy:
//   dgate = gamma1 A + beta1 B,  dgamma1 = gate A,  dbeta1 = gate B,  dgamma2 = C,  dbeta2 = D
//
// so that five weights' gradients need four sums a column.  Without the first norm xhat is x, gamma1 1 and beta1 0.  Bound by HBM: the four inputs
// of a row are read once.  Sums over rows stay in a workgroup's registers (rows of more than 8192: half of them in LDS), its partial sums go to the caller's workspace
// and are joined in order.  A workgroup goes down its rows with one row ahead; what holds it is a row's chain (two sums over waves, behind one another).  16384 x
// 4096 bf16, both norms layer, 8 devices 152 .. 162 us (154 + 7 for the join; 805 MB, 5.2 TB/s); 1767 x 1001 fp32, 3 devices 21 (18 + 4).  1024 threads have 128 registers each, and spill what does not
// fit: in rows of 4097 to 8192 75 to 89 of them with an fp32 stream and another fp32 operand, 40 to 45 with an fp32 stream alone or fp32 x and dy around a bf16 one, at most 6
// else; in rows of more than 8192, which keep two of the sums in LDS, 15 to 36: 4532 x 11752 210 us (3.0 TB/s), 4096 x 12288 156.
#include "row_device.h"

namespace sbp {
namespace {

// Past the caches: bf16 in rows of more than 2048.  16384 x 4096 158.5 us with it, 163 without, 1 device 1024 x 8192 32.1 / 36.2, 4096 x 8192 91.0 / 96.7, fp32 residual 8192 x 4096
// 125.5 / 129 - but in fp32, whose eight elements are two loads of half a line each, 198 / 170, and in short rows whose inputs the memory-side cache
// holds 24.6 / 22.1 (4096 x 1024).
template <int T, int TPR> constexpr bool streamed = T == T_BF16 && TPR >= 512;

template <int XT, int RT, int YT, int TPR, int V, int S>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void residual_norm_grad_kernel(ResNormGradPlan<S> p) {
    constexpr int NT = TPR < 256 ? 256 : TPR, G = NT / TPR, NW = TPR / 64, N = V * 8, CAP = TPR * V * 8;
    constexpr bool KEEP = V == 1;   // weights and two of the sums stay in registers
    const ResNormGradShard& s = p.s[S > 1 ? blockIdx.y : 0];
    if ((int)blockIdx.x >= s.blocks) return;
    const int t = threadIdx.x % TPR, group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TPR) : 0, cols = p.cols;   // whole waves
    const bool post = p.flags & RN_POST, pre = p.flags & RN_PRE, with_dh = p.flags & RN_DH, narrow_weights = p.flags & RN_BF16_WEIGHTS;
    __shared__ float2 part[2][2][G][NW];
    __shared__ float sums[KEEP ? (G > 1 ? G * 4 * CAP : 4) : 2 * CAP];   // KEEP: the groups' sums at the end; else C and D
    const RowPart<TPR, V> part_of_row(t, cols);
    float gamma2[8], through[8];   // of one vector; through: gate gamma1
    auto column = [&](int v) __attribute__((always_inline)) {   // not KEEP: opaque, or addresses would be held in registers from row to row
        int c = (v * TPR + t) * 8;
        if constexpr (!KEEP) asm volatile("" : "+v"(c));
        return c;
    };
    auto load1 = [&](int v) __attribute__((always_inline)) {
        const int c = column(v);
        load_weight8(s.gate, narrow_weights, c, cols, 1.0f, through);
        if (post) {
            float w[8];
            load_weight8(s.gamma1, narrow_weights, c, cols, 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) through[e] *= w[e];
        }
    };
    auto load2 = [&](int v) __attribute__((always_inline)) { load_weight8(s.gamma2, narrow_weights, column(v), cols, 1.0f, gamma2); };
    if constexpr (KEEP) {
        load1(0);
        if (pre) load2(0);
    }
    float sum_a[N], sum_b[N], sum_c[KEEP ? N : 1], sum_d[KEEP ? N : 1];
#pragma unroll
    for (int i = 0; i < N; ++i) sum_a[i] = sum_b[i] = 0.0f;
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum_c[i] = sum_d[i] = 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) sums[i * TPR + t] = sums[CAP + i * TPR + t] = 0.0f;   // a thread's own places
    }

    const int step = s.blocks * G;
    Raw8<XT> next_x[V];
    Raw8<RT> next_h[V], next_dh[V];
    Raw8<YT> next_dy[V];
    float next_mean1 = 0.0f, next_rstd1 = 1.0f, next_mean2 = 0.0f, next_rstd2 = 0.0f;
    auto fetch = [&](int64_t row) {
        const bool there = row < s.rows;
        const int upto = there ? cols : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = column(v);
            next_x[v] = load8<XT, streamed<XT, TPR>>(static_cast<const char*>(s.x) + row * s.ldx * bytes_of<XT>, c, upto);
            next_h[v] = load8<RT, streamed<RT, TPR>>(static_cast<const char*>(s.h) + row * s.ldh * bytes_of<RT>, c, pre ? upto : 0);
            next_dy[v] = load8<YT, streamed<YT, TPR>>(static_cast<const char*>(s.dy) + row * s.lddy * bytes_of<YT>, c, pre ? upto : 0);
            next_dh[v] = load8<RT, streamed<RT, TPR>>(static_cast<const char*>(s.dh) + row * s.lddh * bytes_of<RT>, c, with_dh ? upto : 0);
        }
        if (there && post) {
            next_mean1 = s.mean1 ? s.mean1[row] : 0.0f;
            next_rstd1 = s.rstd1[row];
        }
        if (there && pre) {
            next_mean2 = s.mean2 ? s.mean2[row] : 0.0f;
            next_rstd2 = s.rstd2[row];
        }
    };
    int64_t row = (int64_t)blockIdx.x * G + group;
    if constexpr (KEEP) fetch(row);
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * G; first < s.rows; first += step, row += step, turn ^= 1) {
        if constexpr (!KEEP) fetch(row);
        const int there = row < s.rows ? cols : 0;
        const float mean1 = next_mean1, rstd1 = next_rstd1, mean2 = next_mean2, rstd2 = next_rstd2;
        float xhat[N], d[N], hhat[N], dy[N];
        const bool cut = !part_of_row.whole || row >= s.rows;   // some lane has fewer than eight elements of a vector
        if (!part_of_row.whole) {
            asm volatile("");   // or all of it would be worked out, and chosen from
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * TPR + t) * 8;
                next_x[v] = settle8<XT>(next_x[v], c, there);
                next_dh[v] = settle8<RT>(next_dh[v], c, with_dh ? there : 0);
                next_h[v] = settle8<RT>(next_h[v], c, pre ? there : 0);
                next_dy[v] = settle8<YT>(next_dy[v], c, pre ? there : 0);
            }
        }
        auto take_pre = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float z[8], q[8];
                widen<RT>(next_h[v], 1.0f, z);
                widen<YT>(next_dy[v], 1.0f, q);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    hhat[v * 8 + e] = (z[e] - mean2) * rstd2;
                    dy[v * 8 + e] = q[e];
                }
            }
            if (cut) {   // where no element is, mean * rstd may be infinite, and times 0 NaN
                asm volatile("");
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) hhat[v * 8 + e] = (v * TPR + t) * 8 + e < there ? hhat[v * 8 + e] : 0.0f;
            }
        };
        auto take_post = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float u[8], w[8];
                widen<XT>(next_x[v], 1.0f, u);
                widen<RT>(next_dh[v], 1.0f, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xhat[v * 8 + e] = post ? (u[e] - mean1) * rstd1 : u[e];
                    d[v * 8 + e] = w[e];
                }
            }
            if (cut) {
                asm volatile("");
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) xhat[v * 8 + e] = (v * TPR + t) * 8 + e < there ? xhat[v * 8 + e] : 0.0f;
            }
        };
        take_pre();
        if constexpr (KEEP) {
            take_post();
            fetch(row + step);
        }
        float s1 = 0.0f, s2 = 0.0f;
        if (pre) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (!KEEP) {
                    __builtin_amdgcn_sched_barrier(0);   // one vector's weights at a time, for their registers
                    load2(v);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = v * 8 + e;
                    if constexpr (KEEP) {
                        sum_c[i] = fmaf(dy[i], hhat[i], sum_c[i]);
                        sum_d[i] += dy[i];
                    } else {
                        sums[i * TPR + t] = fmaf(dy[i], hhat[i], sums[i * TPR + t]);
                        sums[CAP + i * TPR + t] += dy[i];
                    }
                    dy[i] *= gamma2[e];
                    s1 += dy[i];
                    s2 = fmaf(dy[i], hhat[i], s2);
                }
            }
            part_of_row.sums(s1, s2, part[turn][0][group]);
            s1 = p.flags & RN_PRE_LAYER ? s1 * part_of_row.over : 0.0f;
            s2 *= part_of_row.over;
        }
        if constexpr (!KEEP) {
            __builtin_amdgcn_sched_barrier(0);   // not before, for its registers
            take_post();
        }
        if (pre) {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = fmaf(rstd2, fmaf(-hhat[i], s2, dy[i] - s1), d[i]);
            if (cut) {   // s1 is behind the row's end too
                asm volatile("");
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[v * 8 + e] = (v * TPR + t) * 8 + e < there ? d[v * 8 + e] : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            sum_a[i] = fmaf(d[i], xhat[i], sum_a[i]);
            sum_b[i] += d[i];
        }
        if (row < s.rows) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = column(v);
                float u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = p.alpha * d[v * 8 + e];
                store8<RT>(static_cast<char*>(s.dr) + (row * s.lddr + c) * bytes_of<RT>, narrow<RT>(u), cols - c, p.flags & RN_STREAM_H);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (!KEEP) {
                __builtin_amdgcn_sched_barrier(0);
                load1(v);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) d[v * 8 + e] *= through[e];
        }
        if (post) {
            s1 = s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s1 += d[i];
                s2 = fmaf(d[i], xhat[i], s2);
            }
            part_of_row.sums(s1, s2, part[turn][1][group]);
            s1 = p.flags & RN_POST_LAYER ? s1 * part_of_row.over : 0.0f;
            s2 *= part_of_row.over;
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = rstd1 * fmaf(-xhat[i], s2, d[i] - s1);
        }
        if (row < s.rows) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = column(v);
                float u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = d[v * 8 + e];
                store8<XT>(static_cast<char*>(s.dx) + (row * s.lddx + c) * bytes_of<XT>, narrow<XT>(u), cols - c, p.flags & RN_STREAM_Y);
            }
        }
    }
    if (!s.part) return;
    float* const to = s.part + (int64_t)blockIdx.x * 4 * cols;
    auto put = [&](int which, const float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * TPR + t) * 8;
            Raw8<T_F32> a;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a.a[e] = v[i * 8 + e];
                a.b[e] = v[i * 8 + 4 + e];
            }
            store8<T_F32>(to + (int64_t)which * cols + c, a, cols - c);
        }
    };
    if constexpr (G > 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {   // V is 1
            float* const at = sums + group * 4 * CAP + t * 8 + i;
            at[0] = sum_a[i];
            at[CAP] = sum_b[i];
            at[2 * CAP] = sum_c[i];
            at[3 * CAP] = sum_d[i];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += NT)
#pragma unroll
            for (int which = 0; which < 4; ++which) {
                float a = 0.0f;
#pragma unroll
                for (int g = 0; g < G; ++g) a += sums[(g * 4 + which) * CAP + c];
                to[(int64_t)which * cols + c] = a;
            }
    } else {
        put(0, sum_a);
        put(1, sum_b);
        if constexpr (KEEP) {
            put(2, sum_c);
            put(3, sum_d);
        } else {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float v[N];
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = sums[which * CAP + i * TPR + t];
                put(2 + which, v);
            }
        }
    }
}

// The workgroups' partial sums in order, and the weights' gradients from them: 32 columns a workgroup, 32 runs of partial sums side by side.
constexpr int RUNS = 32;
template <int S>
__global__ __launch_bounds__(32 * RUNS) void residual_norm_join_kernel(ResNormJoin<S> p) {
    const ResNormJoinShard& s = p.s[S > 1 ? blockIdx.y : 0];
    __shared__ float sums[4][RUNS][33], totals[4][32];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < p.cols) {
        for (int b = run; b < s.blocks; b += 2 * RUNS) {   // two on their way, past the end the last one again, which does not count
            float v[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int which = 0; which < 4; ++which) v[u][which] = s.part[((int64_t)min(b + RUNS * u, s.blocks - 1) * 4 + which) * p.cols + c];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int which = 0; which < 4; ++which) a[which] += b + RUNS * u < s.blocks ? v[u][which] : 0.0f;
        }
    }
#pragma unroll
    for (int which = 0; which < 4; ++which) sums[which][run][lane] = a[which];
    __syncthreads();
    if (run < 4) {
        float total = 0.0f;
#pragma unroll
        for (int r = 0; r < RUNS; ++r) total += sums[run][r][lane];
        totals[run][lane] = total;
    }
    __syncthreads();
    if (run != 0 || c >= p.cols) return;
#pragma unroll
    for (int which = 0; which < 4; ++which) a[which] = totals[which][lane];
    auto weight = [&](const void* w, float otherwise) {
        return !w ? otherwise : p.flags & RN_BF16_WEIGHTS ? bf16_to_f32(static_cast<const uint16_t*>(w)[c]) : static_cast<const float*>(w)[c];
    };
    const float gate = weight(s.gate, 1.0f);
    if (s.dgate) s.dgate[c] = p.flags & RN_POST ? fmaf(weight(s.gamma1, 1.0f), a[0], weight(s.beta1, 0.0f) * a[1]) : a[0];
    if (s.dgamma1) s.dgamma1[c] = gate * a[0];
    if (s.dbeta1) s.dbeta1[c] = gate * a[1];
    if (s.dgamma2) s.dgamma2[c] = a[2];
    if (s.dbeta2) s.dbeta2[c] = a[3];
}

// threads of a row
int threads_of(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }

}  // namespace

// One workgroup a CU, two or four where a row is short and there are enough rows: more hide more, but each reads the weights and leaves four sums a column for
// the join.  With 512 threads a row (130 to 141 registers; 128 in a launch for one device, all bf16) and with 1024 a CU holds one workgroup, so that what is more waits.  us, 256 / 512 / 1024 workgroups, bf16: 31327 x 360 79 / 54 / 47, 16384 x 768 60.5 / 41.8 / 49.7, 4096 x 768 21.3 / 17.0, 32768 x 1024 129 / 88 / 90, 8192 x
// 1537 67 / 48 / 56, but 1024 x 1024 11.3 / 13.2, 2000 x 1024 15.2 / 16.3; 8192 x 2560 58 / 62 / 72, 16384 x 4096 155 / 163 / 170, 4096 x 8192 96 / 108 / 133.
int32_t residual_norm_grad_blocks(int64_t rows, int64_t cols, int32_t k) {
    const int64_t g = std::max(1, 256 / threads_of(cols)), turns = (rows + g - 1) / g;
    const int64_t most = cols > 2048 || turns * k < 1280 ? 256 : cols > 512 || turns * k < 5120 ? 512 : 1024;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(turns, most / k));
}

template <int S>
int32_t launch_residual_norm_grad(const ResNormGradPlan<S>& given, int n, int32_t x_type, int32_t r_type, int32_t y_type, hipStream_t stream) {
    ResNormGradPlan<S> plan = given;
    int blocks = 1;
    int64_t all = 0;
    bool r_lines = true, x_lines = true;
    for (int i = 0; i < n; ++i) {
        blocks = std::max(blocks, plan.s[i].blocks);
        all += plan.s[i].rows;
        if ((int64_t)plan.s[i].lddr * bytes_of_type(r_type) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].dr) % 128) r_lines = false;
        if ((int64_t)plan.s[i].lddx * bytes_of_type(x_type) % 128 || reinterpret_cast<uintptr_t>(plan.s[i].dx) % 128) x_lines = false;
    }
    const int64_t elements = all * plan.cols;
    if (streams_of(0, elements * bytes_of_type(r_type), r_lines, r_type) & STREAM_OUT) plan.flags |= RN_STREAM_H;
    if (streams_of(0, elements * bytes_of_type(x_type), x_lines, x_type) & STREAM_OUT) plan.flags |= RN_STREAM_Y;
    with_wide_type(x_type, [&](auto x) {
        with_wide_type(r_type, [&](auto r) {
            with_wide_type(y_type, [&](auto y) {
                auto go = [&](auto tpr, auto v) {
                    hipLaunchKernelGGL((residual_norm_grad_kernel<x(), r(), y(), tpr(), v(), S>), dim3((uint32_t)blocks, (uint32_t)n), dim3(tpr() < 256 ? 256 : tpr()), 0, stream, plan);
                };
                using std::integral_constant;
                switch (threads_of(plan.cols)) {
                    case 64: go(integral_constant<int, 64>{}, integral_constant<int, 1>{}); break;
                    case 128: go(integral_constant<int, 128>{}, integral_constant<int, 1>{}); break;
                    case 256: go(integral_constant<int, 256>{}, integral_constant<int, 1>{}); break;
                    case 512: go(integral_constant<int, 512>{}, integral_constant<int, 1>{}); break;
                    default:
                        if (plan.cols <= 8192) go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
                        else go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
                }
            });
        });
    });
    return launch_status(__func__);
}

template <int S>
int32_t launch_residual_norm_join(const ResNormJoin<S>& join, int n, hipStream_t stream) {
    hipLaunchKernelGGL(residual_norm_join_kernel<S>, dim3((uint32_t)((join.cols + 31) / 32), (uint32_t)n), dim3(32 * RUNS), 0, stream, join);
    return launch_status(__func__);
}
template int32_t launch_residual_norm_grad<1>(const ResNormGradPlan<1>&, int, int32_t, int32_t, int32_t, hipStream_t);
template int32_t launch_residual_norm_grad<RESNORM_SHARDS>(const ResNormGradPlan<RESNORM_SHARDS>&, int, int32_t, int32_t, int32_t, hipStream_t);
template int32_t launch_residual_norm_join<1>(const ResNormJoin<1>&, int, hipStream_t);
template int32_t launch_residual_norm_join<RESNORM_SHARDS>(const ResNormJoin<RESNORM_SHARDS>&, int, hipStream_t);

}  // namespace sbp
