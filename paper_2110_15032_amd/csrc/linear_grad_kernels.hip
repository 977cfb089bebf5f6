// The gradient of a product's epilogue (bias, then GeLU): da = dy gelu'(pre), and the bias' gradient, the sum of da over the rows; without an activation
// the sum of dy alone.
//
// Bound by HBM.  32 lanes take 256 columns of a row, eight each, and eight rows side by side make a workgroup; it walks down its share of the
// rows with the sums in registers, which meet in LDS at the end.  Its partial sums go to the caller's workspace and are joined in order.  8192 x 16384 bf16 with
// GeLU, 8 devices 145 us (141 + 5 for the join; 805 MB, 5.7 TB/s; GeLU's arithmetic is 89 of vector instructions); 1767 x 1001 fp32, 3 devices 12.3 (9.2 + 1.6).  Two rows
// ahead instead of four 13.6 -> 12.3 at 2000 x 3001, but 12.4 -> 13.7 at 1767 x 1001; 1024 workgroups instead of 2048 31 -> 25 at 32768 x 300, and none at
// the other sizes.
#include "row_device.h"

namespace sbp {
namespace {

constexpr int NT = 256, COLS = 256, SIDE = NT * 8 / COLS;   // columns of a workgroup, rows side by side

template <int PT, int YT, bool GELU, bool IN, int S>
__global__ __launch_bounds__(NT) void linear_grad_kernel(LinearGradPlan<S> p) {
    const LinearGradShard& s = p.s[S > 1 ? blockIdx.z : 0];
    if ((int)blockIdx.y >= s.blocks || (int64_t)blockIdx.x * COLS >= s.cols) return;
    constexpr int AHEAD = 4;   // rows of a lane on their way together
    const int lane = threadIdx.x & 31, side = threadIdx.x >> 5, c = blockIdx.x * COLS + lane * 8;
    const int step = s.blocks * SIDE;
    const bool cut = s.cols % 8 != 0;   // some lane has fewer than eight elements
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    for (int64_t first = (int64_t)blockIdx.y * SIDE + side; first < s.rows; first += (int64_t)AHEAD * step) {
        Raw8<YT> raw[AHEAD];
        Raw8<PT> at[AHEAD];
        uint32_t byte[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t row = first + (int64_t)u * step;
            const int upto = row < s.rows ? s.cols : 0;
            raw[u] = load8<YT, IN>(static_cast<const char*>(s.dy) + row * s.lddy * bytes_of<YT>, c, upto);
            if constexpr (GELU) {
                at[u] = load8<PT, IN>(static_cast<const char*>(s.pre) + row * s.ldp * bytes_of<PT>, c, upto);
                byte[u] = 127;
                if constexpr (bytes_of<PT> == 1)
                    if (c < upto) byte[u] = static_cast<const uint8_t*>(s.scales)[row * s.lds + c / F8_BLOCK];
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t row = first + (int64_t)u * step;
            const int upto = row < s.rows ? s.cols : 0;
            float d[8];
            widen<YT>(cut ? settle8<YT>(raw[u], c, upto) : raw[u], 1.0f, d);
            if constexpr (GELU) {
                float a[8];
                widen<PT>(cut ? settle8<PT>(at[u], c, upto) : at[u], scale_of(byte[u]), a);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] *= gelu_slope<YT == T_BF16>(a[e]);
                store8<YT>(static_cast<char*>(s.da) + (row * s.ldda + c) * bytes_of<YT>, narrow<YT>(d), upto - c, p.streams & STREAM_OUT);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += d[e];
        }
    }
    __shared__ __attribute__((aligned(16))) float sums[SIDE][COLS];
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[side][lane * 8 + e] = sum[e];
    __syncthreads();
    const int64_t mine = (int64_t)blockIdx.x * COLS + threadIdx.x;
    if (mine >= s.cols) return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < SIDE; ++i) v += sums[i][threadIdx.x];
    if (s.blocks > 1) s.part[(int64_t)blockIdx.y * s.cols + mine] = v;
    else s.dbias[mine] = v;
}

// The partial sums of a shard's workgroups in order: 32 columns a workgroup, eight runs of partial sums side by side.
template <int S>
__global__ __launch_bounds__(256) void linear_grad_join_kernel(LinearGradPlan<S> p) {
    const LinearGradShard& s = p.s[S > 1 ? blockIdx.y : 0];
    if (s.blocks <= 1) return;
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float a = 0.0f;
    if (c < s.cols) {
        for (int b = run; b < s.blocks; b += 32) {   // four on their way, past the end the last one again, which does not count
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = s.part[(int64_t)min(b + 8 * u, s.blocks - 1) * s.cols + c];
#pragma unroll
            for (int u = 0; u < 4; ++u) a += b + 8 * u < s.blocks ? v[u] : 0.0f;
        }
    }
    sums[run][lane] = a;
    __syncthreads();
    if (run == 0 && c < s.cols) {
        a = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) a += sums[r][lane];
        s.dbias[c] = a;
    }
}

}  // namespace

// As many as give the chip eight workgroups a compute unit, with at least a full turn of rows each.
int32_t linear_grad_blocks(int64_t rows, int64_t cols, int32_t k) {
    const int64_t across = std::max<int64_t>(1, (cols + COLS - 1) / COLS) * k;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + SIDE * 4 - 1) / (SIDE * 4), 2048 / across));
}

template <int S>
int32_t launch_linear_grad(const LinearGradPlan<S>& given, int n, int32_t dy_type, int32_t pre_type, bool gelu, hipStream_t stream) {
    LinearGradPlan<S> plan = given;
    int blocks = 1;
    int64_t cols = 1, elements = 0;
    bool on_lines = true, join = false;
    for (int i = 0; i < n; ++i) {
        const LinearGradShard& s = plan.s[i];
        blocks = std::max(blocks, s.blocks);
        cols = std::max<int64_t>(cols, s.cols);
        elements += (int64_t)s.rows * s.cols;
        join = join || s.blocks > 1;
        if ((int64_t)s.ldda * bytes_of_type(dy_type) % 128 || reinterpret_cast<uintptr_t>(s.da) % 128) on_lines = false;
    }
    const int size = bytes_of_type(dy_type);
    plan.streams = streams_of(elements * (size + (gelu ? bytes_of_type(pre_type) : 0)), gelu ? elements * size : 0, on_lines, dy_type);
    const dim3 grid((uint32_t)((cols + COLS - 1) / COLS), (uint32_t)blocks, (uint32_t)n);
    with_wide_type(dy_type, [&](auto y) {
        auto go = [&](auto a, auto act) {
            if (plan.streams & STREAM_IN) hipLaunchKernelGGL((linear_grad_kernel<a(), y(), act(), true, S>), grid, dim3(NT), 0, stream, plan);
            else hipLaunchKernelGGL((linear_grad_kernel<a(), y(), act(), false, S>), grid, dim3(NT), 0, stream, plan);
        };
        if (gelu) with_any_type(pre_type, [&](auto a) { go(a, std::true_type{}); });
        else go(std::integral_constant<int, T_BF16>{}, std::false_type{});
    });
    const int32_t st = launch_status(__func__);
    if (st != SBP_OK || !join) return st;
    hipLaunchKernelGGL(linear_grad_join_kernel<S>, dim3((uint32_t)((cols + 31) / 32), (uint32_t)n), dim3(256), 0, stream, plan);
    return launch_status(__func__);
}
template int32_t launch_linear_grad<1>(const LinearGradPlan<1>&, int, int32_t, int32_t, bool, hipStream_t);
template int32_t launch_linear_grad<LINEAR_GRAD_SHARDS>(const LinearGradPlan<LINEAR_GRAD_SHARDS>&, int, int32_t, int32_t, bool, hipStream_t);

}  // namespace sbp
