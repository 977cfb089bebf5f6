// Products of a few rows (tokens that are decoded) with a block's epilogue: the weight is the traffic, and is read once; up to four rows past the matrix cores.
//
//   y[m, n] = act(sum over kk of x[m, kk] w[kk, n] + bias[n]) + residual[m, n]
//
// Bound by HBM: what counts is that every compute unit has enough of the weight on its way.  One row, 4096 x 16384 bf16 on 8 devices (134 MB) 24 us, 5.6 TB/s.
#include "block8_device.h"

namespace sbp {
namespace {

__device__ inline void add8(const float (&x)[8], const float (&w)[8], float& acc) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc = fmaf(x[e], w[e], acc);
}

// Weights with the reduction index contiguous.  A wave takes R rows of the weight and every WK-th 512 elements of them, eight a lane; where the waves of a
// workgroup share rows (WK > 1) their sums meet in LDS, in order.
// STREAM: the weight past the caches: in bf16, where a token's weights do not stay in the memory-side cache.  us, past them / cached, four weights in turn: 4096 x 16384 (134 MB)
// 23.8 / 25.7, 4 rows 26.8 / 28.7; 101 MB 19.3 / 20.8, 84 MB 17.5 / 18.7, 67 MB 14.1 / 14.1, 50 MB 10.8 / 10.2, 4 rows 18.4 / 16.1; columns contiguous 134 MB 27.4 / 29.4, 84 MB
// 18.6 / 20.1, 67 MB 16.3 / 15.6.  Not in fp32, whose eight elements are two loads of half a line each: 134 MB 32.8 / 29.8, 101 MB 22.7 / 18.7, 403 MB 84.9 / 78.5.
template <int T, int M, int R, int WK, bool STREAM>
__global__ __launch_bounds__(256) void gemv_rows_kernel(GemmBlockPlan p) {
    constexpr int GROUPS = 4 / WK, AHEAD = R == 4 && M == 1 ? 4 : 2;   // steps on their way together: 4096 x 16384, one row, two 25.0 us, four 24.3; one row of the weight a wave, 4096 x 4096, two 7.9, four 10.5
    const GemmShard& s = p.s[blockIdx.y];
    if (s.m == 0) return;   // a device without rows, whose x need not be anywhere
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK;
    const int64_t n0 = ((int64_t)blockIdx.x * GROUPS + wave / WK) * R;
    float acc[R][M];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) acc[r][m] = 0.0f;
    if (n0 < s.n) {
        const char* w[R];   // rows past the last one are the last one again, and stored nowhere
        const char* x[M];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = static_cast<const char*>(s.b) + min(n0 + r, (int64_t)s.n - 1) * s.ldb * bytes_of<T>;
#pragma unroll
        for (int m = 0; m < M; ++m) x[m] = static_cast<const char*>(s.a) + (int64_t)min(m, s.m - 1) * s.lda * bytes_of<T>;
        constexpr int STEP = 512 * WK;
        for (int64_t k0 = wk * 512; k0 < s.kk; k0 += (int64_t)STEP * AHEAD) {
            Raw8<T> rw[AHEAD][R], rx[AHEAD][M];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t from = k0 + u * STEP + lane * 8;
                const int c = from < s.kk ? (int)from : s.kk;
#pragma unroll
                for (int r = 0; r < R; ++r) rw[u][r] = load8<T, STREAM>(w[r], c, s.kk);
#pragma unroll
                for (int m = 0; m < M; ++m) rx[u][m] = load8<T>(x[m], c, s.kk);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t from = k0 + u * STEP + lane * 8;
                const int c = from < s.kk ? (int)from : s.kk;
                float vx[M][8];
#pragma unroll
                for (int m = 0; m < M; ++m) widen<T>(settle8<T>(rx[u][m], c, s.kk), 1.0f, vx[m]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float vw[8];
                    widen<T>(settle8<T>(rw[u][r], c, s.kk), 1.0f, vw);
#pragma unroll
                    for (int m = 0; m < M; ++m) add8(vx[m], vw, acc[r][m]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) acc[r][m] = sum_wave(acc[r][m]);
    }
    float mine = 0.0f;   // of lane r M + m
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) mine = lane == r * M + m ? acc[r][m] : mine;
    if constexpr (WK > 1) {
        __shared__ float part[4][R * M];
        if (lane < R * M) part[wave][lane] = mine;
        __syncthreads();
        if (wk != 0) return;
        if (lane < R * M) {
#pragma unroll
            for (int i = 1; i < WK; ++i) mine += part[wave + i][lane];
        }
    }
    if (lane < R * M) {
        float v[1] = {mine};
        Ending<EPI_BLOCK>(p, blockIdx.y).finish<1>(s, lane % M, (int)min(n0 + lane / M, (int64_t)INT32_MAX), v);
    }
}

// One row, weights with their columns contiguous.  A workgroup of 16 waves takes 64 columns, a wave eight rows of them at a time, eight columns a lane; lanes and
// waves of the same columns meet at the end, in order.
template <int T, bool STREAM>
__global__ __launch_bounds__(1024) void gemv_columns_kernel(GemmBlockPlan p) {
    constexpr int NW = 16, AHEAD = 4, STEP = NW * 8;
    const GemmShard& s = p.s[blockIdx.y];
    const int n0 = blockIdx.x * 64;
    if (n0 >= s.n || s.m == 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = n0 + (lane & 7) * 8;
    float acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
    for (int64_t k0 = wave * 8 + (lane >> 3); k0 < s.kk; k0 += STEP * AHEAD) {
        Raw8<T> rw[AHEAD];
        float x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t k = k0 + u * STEP;
            rw[u] = load8<T, STREAM>(static_cast<const char*>(s.b) + k * s.ldb * bytes_of<T>, c, k < s.kk ? s.n : 0);
            x[u] = 0.0f;
            if (k < s.kk) {
                if constexpr (T == T_F32) x[u] = static_cast<const float*>(s.a)[k];
                else x[u] = bf16_to_f32(static_cast<const uint16_t*>(s.a)[k]);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            float w[8];
            widen<T>(settle8<T>(rw[u], c, k0 + u * STEP < s.kk ? s.n : 0), 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = fmaf(x[u], w[e], acc[e]);
        }
    }
    __shared__ float part[NW][64];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float v = acc[e];
        v += __shfl_xor(v, 8, 64);
        v += __shfl_xor(v, 16, 64);
        v += __shfl_xor(v, 32, 64);
        if (lane < 8) part[wave][lane * 8 + e] = v;
    }
    __syncthreads();
    if (wave != 0) return;
    float v[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NW; ++i) v[0] += part[i][lane];
    Ending<EPI_BLOCK>(p, blockIdx.y).finish<1>(s, 0, n0 + lane, v);
}

// Up to 32 rows in bf16, weights with the reduction index contiguous, few columns: a workgroup of 16 waves takes 16 of them, a wave every 16th piece of the reduction,
// straight from memory into the operands of v_mfma_f32_16x16x32_bf16 (lane l: eight elements of row l % 16 from 8 (l / 16) on); the waves' sums meet in
// LDS, in order.  The next piece is on its way while one is multiplied.  Any alignment.  Bound by how much of the weight is on its way; x comes from L2 for
// every workgroup, as many bytes as the weight with 16 rows.
template <int MT>   // 16 rows of x each
__global__ __launch_bounds__(1024) void gemm_few_kernel(GemmBlockPlan p) {
    constexpr int NW = 16, U = MT == 1 ? 6 : 4, STEP = 32 * U;   // what 128 registers hold; MT 1, 16384 x 4096, 8 rows, four 38.7 us, six 35.0
    const GemmShard& s = p.s[blockIdx.y];
    const int n0 = blockIdx.x * 16;
    if (n0 >= s.n || s.m == 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), of = lane & 15, from = (lane >> 4) * 8;
    // rows past the last one are the last one again, and stored nowhere
    const char* const w = static_cast<const char*>(s.b) + (int64_t)min(n0 + of, s.n - 1) * s.ldb * 2;
    const char* x[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x[i] = static_cast<const char*>(s.a) + (int64_t)min(i * 16 + of, s.m - 1) * s.lda * 2;
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Raw8<T_BF16> rw[U], rx[U][MT];
    auto fetch = [&](int k0) __attribute__((always_inline)) {   // k0: uniform, not past the last piece's
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = min(k0 + u * 32 + from, s.kk);
            rw[u] = load8<T_BF16>(w, c, s.kk);
#pragma unroll
            for (int i = 0; i < MT; ++i) rx[u][i] = load8<T_BF16>(x[i], c, s.kk);
        }
    };
    if (wave * STEP < s.kk) fetch(wave * STEP);
    for (int64_t k0 = wave * STEP; k0 < s.kk; k0 += NW * STEP) {
        u32x4 b[U], a[U][MT];
        if (k0 + STEP > s.kk) {
            asm volatile("");   // or it would be done always, and chosen from
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = (int)min(k0 + u * 32 + from, (int64_t)s.kk);
                rw[u] = settle8<T_BF16>(rw[u], c, s.kk);
#pragma unroll
                for (int i = 0; i < MT; ++i) rx[u][i] = settle8<T_BF16>(rx[u][i], c, s.kk);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            b[u] = rw[u].w;
#pragma unroll
            for (int i = 0; i < MT; ++i) a[u][i] = rx[u][i].w;
        }
        if (k0 + NW * STEP < s.kk) fetch((int)(k0 + NW * STEP));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u][i]), __builtin_bit_cast(bf16x8, b[u]), acc[i], 0, 0, 0);
    }
    __shared__ float part[NW][MT * 256];   // [row][column]
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][(i * 16 + (lane >> 4) * 4 + r) * 16 + of] = acc[i][r];
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= MT * 256) return;
    float v[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NW; ++i) v[0] += part[i][t];
    Ending<EPI_BLOCK>(p, blockIdx.y).finish<1>(s, t >> 4, n0 + (t & 15), v);
}

template <typename F>
void with_rows(int m, F&& f) {
    if (m == 1) f(std::integral_constant<int, 1>{});
    else if (m == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

}  // namespace

// x with the reduction index contiguous; 1 .. GEMV_ROWS rows of it where w has too, else one
int32_t launch_gemv(const GemmBlockPlan& plan, int max_m, int max_n, hipStream_t stream) {
    const bool f32 = plan.in_dtype == SBP_F32;
    int64_t columns = 0, weight = 0;
    int deepest = 0;
    for (int g = 0; g < plan.groups; ++g) {
        columns += plan.s[g].n;
        weight += (int64_t)plan.s[g].n * plan.s[g].kk * (f32 ? 4 : 2);
        deepest = std::max(deepest, plan.s[g].kk);
    }
    const uint32_t groups = (uint32_t)plan.groups;
    auto go = [&](auto t, auto past) {
        if (!plan.b_kc) {
            if (!grid_fits(tiles_along(max_n, 64), 1024)) return (int32_t)SBP_ERR_UNSUPPORTED;
            hipLaunchKernelGGL((gemv_columns_kernel<t(), past()>), dim3((uint32_t)tiles_along(max_n, 64), groups), dim3(1024), 0, stream, plan);
            return launch_status("launch_gemv");
        }
        if (!grid_fits(tiles_along(max_n, columns >= 8192 ? 16 : 1), 256)) return (int32_t)SBP_ERR_UNSUPPORTED;
        with_rows(max_m, [&](auto m) {
            // four rows a wave where that leaves a compute unit eight waves or more, else one, and the waves share a long reduction
            if (columns >= 8192) hipLaunchKernelGGL((gemv_rows_kernel<t(), m(), 4, 1, past()>), dim3((uint32_t)tiles_along(max_n, 16), groups), dim3(256), 0, stream, plan);
            else if (deepest > 1024) hipLaunchKernelGGL((gemv_rows_kernel<t(), m(), 1, 4, past()>), dim3((uint32_t)max_n, groups), dim3(256), 0, stream, plan);
            else hipLaunchKernelGGL((gemv_rows_kernel<t(), m(), 1, 1, past()>), dim3((uint32_t)tiles_along(max_n, 4), groups), dim3(256), 0, stream, plan);
        });
        return launch_status("launch_gemv");
    };
    if (f32) return go(std::integral_constant<int, T_F32>{}, std::false_type{});
    return weight > (int64_t)64 << 20 ? go(std::integral_constant<int, T_BF16>{}, std::true_type{}) : go(std::integral_constant<int, T_BF16>{}, std::false_type{});   // see STREAM
}

// 1 .. FEW_ROWS rows, bf16, both operands with the reduction index contiguous
int32_t launch_gemm_few(const GemmBlockPlan& plan, int max_m, int max_n, hipStream_t stream) {
    const dim3 grid((uint32_t)tiles_along(max_n, 16), (uint32_t)plan.groups);
    if (max_m <= 16) hipLaunchKernelGGL(gemm_few_kernel<1>, grid, dim3(1024), 0, stream, plan);
    else hipLaunchKernelGGL(gemm_few_kernel<2>, grid, dim3(1024), 0, stream, plan);
    return launch_status(__func__);
}

}  // namespace sbp
