// Activations in 8 bits: saving them, restoring them, and the gradient of GeLU from a saved pre-activation.
//
// An 8-bit tensor is e4m3 or e5m2 values and, for every 128 consecutive ones of a stored row, a power of two 2^e, e the smallest integer
// >= -127 with max|x| / 2^e within the type; value = round(x / 2^e).  A power of two, because the division and the way back are then
// exact (one rounding in all, the way back to bf16 none) and the matrix instruction takes it as it is.
#include "block8_device.h"

namespace sbp {
namespace {

constexpr int NT = 256;

// Pairs of blocks of 128 of a row-major tensor, 16 lanes to a pair with eight elements of either block each (one address for both, and whole cache
// lines a load): (row, pair) by one division, then advanced by the grid stride with adds.
constexpr int UNIT = 2 * F8_BLOCK;
struct UnitWalk {
    uint32_t per_row, dr, db, b, r;
    __device__ UnitWalk(int cols) {
        per_row = (uint32_t)((cols + UNIT - 1) / UNIT);
        const uint32_t stride = gridDim.x * (NT / 16), first = blockIdx.x * (NT / 16) + (threadIdx.x >> 4);   // a grid is at most 2^16 workgroups
        dr = stride / per_row;
        db = stride % per_row;
        r = first / per_row;
        b = first % per_row;
    }
    __device__ void next() {
        r += dr;
        b += db;
        if (b >= per_row) {
            b -= per_row;
            ++r;
        }
    }
    __device__ int64_t at(int ld) const { return (int64_t)((uint64_t)r * (uint32_t)ld); }
};

// Rounding to 8 bits makes GeLU's fit to 2.2e-5 as good as an exact one; so does rounding to bf16.
template <bool FAST>
__device__ inline float gelu_of(float x) {
    if constexpr (FAST) return gelu_fast(x);
    else return gelu_whole(x);
}

// Bound by HBM: 8192 x 16384 on eight devices from bf16 (404 MB) 64 us, 6.3 TB/s; with GeLU 85 us, by its polynomial and exponential.  IN: inputs past
// the caches.
template <int XT, int QT, bool GELU, bool IN>
__global__ __launch_bounds__(NT) void quantize_kernel(Block8Plan p) {
    const Block8Shard& s = p.s[blockIdx.y];
    if (s.rows == 0 || s.cols == 0) return;
    const int lane = threadIdx.x & 15;
    for (UnitWalk w(s.cols); w.r < (uint32_t)s.rows; w.next()) {
        const int c = (int)w.b * UNIT + lane * 8;
        const char* const from = static_cast<const char*>(s.x) + w.at(s.ldx) * bytes_of<XT>;
        char* const to = static_cast<char*>(s.out) + w.at(s.ldo) + c;
        uint8_t* const scales = static_cast<uint8_t*>(s.scales) + w.at(s.lds) + w.b * 2;
        Raw8<XT> raw[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) raw[u] = load8<XT, IN>(from, c + u * F8_BLOCK, s.cols);
        float v[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            widen<XT>(settle8<XT>(raw[u], c + u * F8_BLOCK, s.cols), 1.0f, v[u]);
            if constexpr (GELU) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = gelu_of<true>(v[u][e]);
            }
        }
        Raw8<QT> q[2];
        uint32_t byte[2];
        narrow_blocks<GELU, QT>(v, q, byte);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            store8<QT>(to + u * F8_BLOCK, q[u], s.cols - c - u * F8_BLOCK, p.streams & STREAM_OUT);
            if (lane == 0 && c + u * F8_BLOCK < s.cols) scales[u] = (uint8_t)byte[u];
        }
    }
}

// Transposed: the block runs along the rows.  A workgroup takes 128 rows by 64 columns; thread t holds rows 4 (t / 8) .. + 3 of the eight
// columns 8 (t % 8), the column maxima meet over the lanes of a wave and over the waves in LDS, the bytes turn in LDS.  8192 x 8192 from bf16 (202 MB)
// 43 .. 46 us, 4.5 TB/s: a tile's loads do not overlap its turn, other workgroups' do; with GeLU 16384 x 1024 (50 MB) 14.9 us.
constexpr int TC = 64;
// Bytes of one column in LDS.  Its 4-byte words are permuted by XOR with turn_key(column / 8), a multiple of four: the eight columns 8 co + e that a
// wave's lanes write at once (eight consecutive words each) fall on different banks.  The reads of 16 bytes on the way out take twice as long as they could: a
// pass has pieces of columns 36 words apart, two of which share banks (34 % of the LDS cycles are conflicts).
constexpr int QPITCH = F8_BLOCK + 16;
__device__ inline int turn_key(int co) { return (co >> 1 & 3) * 8; }
template <int XT, int QT, bool GELU>
__global__ __launch_bounds__(NT) void quantize_transposed_kernel(Block8Plan p, int tiles_r, int tiles_c) {
    const Block8Shard& s = p.s[blockIdx.y];
    __shared__ uint32_t most[4][TC];
    __shared__ __attribute__((aligned(16))) float scale[TC];
    __shared__ __attribute__((aligned(16))) char turn[TC * QPITCH];
    const int t = threadIdx.x, wave = t >> 6, co = t & 7, rg = t >> 3;
    for (int64_t tile = blockIdx.x; tile < (int64_t)tiles_r * tiles_c; tile += gridDim.x) {
        const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c);
        const int64_t r0 = (int64_t)tr * F8_BLOCK;
        const int64_t c0 = (int64_t)tc * TC;
        if (r0 >= s.rows || c0 >= s.cols) continue;
        const int c = (int)c0 + co * 8;
        Raw8<XT> raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + rg * 4 + i;
            raw[i] = load8<XT>(static_cast<const char*>(s.x) + r * s.ldx * bytes_of<XT>, c, r < s.rows ? s.cols : 0);
        }
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            widen<XT>(settle8<XT>(raw[i], c, r0 + rg * 4 + i < s.rows ? s.cols : 0), 1.0f, v[i]);
            if constexpr (GELU) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = gelu_of<true>(v[i][e]);
            }
        }
        uint32_t m[8];
        bool finite = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = most_of<GELU>(v[0][e], v[1][e], v[2][e], v[3][e]);
            finite = finite && m[e] < 0x7F800000u;
        }
        if (!finite) {
            asm volatile("");   // or it would be worked out always, and chosen from
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = max(max(finite_magnitude(v[0][e]), finite_magnitude(v[1][e])), max(finite_magnitude(v[2][e]), finite_magnitude(v[3][e])));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = max(m[e], dpp<0x128>(m[e]));   // eight lanes on in the row of 16
            auto h = __builtin_amdgcn_permlane16_swap(m[e], m[e], false, false);
            m[e] = max((uint32_t)h[0], (uint32_t)h[1]);
            h = __builtin_amdgcn_permlane32_swap(m[e], m[e], false, false);
            m[e] = max((uint32_t)h[0], (uint32_t)h[1]);
        }
        if ((t & 63) < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) most[wave][co * 8 + e] = m[e];
        }
        __syncthreads();
        if (t < TC) {
            const uint32_t byte = scale_byte<QT>(__uint_as_float(max(max(most[0][t], most[1][t]), max(most[2][t], most[3][t]))));
            scale[t] = scale_of(byte);
            if (c0 + t < s.cols) static_cast<uint8_t*>(s.scales)[(c0 + t) * s.lds + tr] = (uint8_t)byte;
        }
        __syncthreads();
        const f32x4 s0 = *reinterpret_cast<const f32x4*>(scale + co * 8), s1 = *reinterpret_cast<const f32x4*>(scale + co * 8 + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint32_t*>(turn + (co * 8 + e) * QPITCH + (rg ^ turn_key(co)) * 4) = narrow4<QT>(v[0][e], v[1][e], v[2][e], v[3][e], e < 4 ? s0[e] : s1[e - 4]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TC * 8 / NT; ++i) {
            const int j = (i * NT + t) >> 3, at = ((i * NT + t) & 7) * 16;
            const int64_t r = r0 + at;
            if (c0 + j >= s.cols || r >= s.rows) continue;
            const u32x4 w = *reinterpret_cast<const u32x4*>(turn + j * QPITCH + (at ^ turn_key(j >> 3) * 4));
            char* dst = static_cast<char*>(s.out) + (c0 + j) * (int64_t)s.ldo + r;
            if (r + 16 <= s.rows) {
                if (p.streams & STREAM_OUT) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_byte*>(dst));
                else *reinterpret_cast<u32x4_byte*>(dst) = w;
            } else {
#pragma unroll
                for (int e = 0; e < 15; ++e)
                    if (r + e < s.rows) dst[e] = (char)(w[e >> 2] >> (8 * (e & 3)));
            }
        }
        // the next tile's maxima are written before the barrier that follows these reads of the turned bytes, its bytes after it
    }
}

// Bound by HBM: 8192 x 8192 to bf16 (202 MB) 29.8 us, 6.8 TB/s; by GeLU with it, 7777 x 4081 on three devices (95 MB) 19.3 .. 20.2 us, 4.8 TB/s.
template <int QT, int YT, bool GELU, bool IN>
__global__ __launch_bounds__(NT) void dequantize_kernel(Block8Plan p) {
    const Block8Shard& s = p.s[blockIdx.y];
    if (s.rows == 0 || s.cols == 0) return;
    const int lane = threadIdx.x & 15;
    for (UnitWalk w(s.cols); w.r < (uint32_t)s.rows; w.next()) {
        const int c = (int)w.b * UNIT + lane * 8;
        const char* const from = static_cast<const char*>(s.x) + w.at(s.ldx);
        char* const to = static_cast<char*>(s.out) + (w.at(s.ldo) + c) * bytes_of<YT>;
        const uint8_t* const scales = static_cast<const uint8_t*>(s.scales) + w.at(s.lds) + w.b * 2;
        Raw8<QT> raw[2];
        uint32_t byte[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            raw[u] = load8<QT, IN>(from, c + u * F8_BLOCK, s.cols);
            byte[u] = scales[(int)w.b * UNIT + u * F8_BLOCK < s.cols ? u : 0];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float v[8];
            widen<QT>(settle8<QT>(raw[u], c + u * F8_BLOCK, s.cols), scale_of(byte[u]), v);
            if constexpr (GELU) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = gelu_of<YT == T_BF16>(v[e]);
            }
            store8<YT>(to + u * F8_BLOCK * bytes_of<YT>, narrow<YT>(v), s.cols - c - u * F8_BLOCK, p.streams & STREAM_OUT);
        }
    }
}

// Restoring a tensor that was saved transposed: 128 saved bytes (128 rows of the result) of 64 saved rows (its columns) turn in LDS.  8192 x 8192
// to bf16 31.6 us, 6.4 TB/s.
template <int QT, int YT, bool GELU>
__global__ __launch_bounds__(NT) void dequantize_transposed_kernel(Block8Plan p, int tiles_r, int tiles_c) {
    const Block8Shard& s = p.s[blockIdx.y];
    __shared__ __attribute__((aligned(16))) char turn[TC * QPITCH];
    __shared__ float scale[TC];
    const int t = threadIdx.x, co = t & 7, rg = t >> 3;
    for (int64_t tile = blockIdx.x; tile < (int64_t)tiles_r * tiles_c; tile += gridDim.x) {
        const int tr = (int)(tile / tiles_c), tc = (int)(tile % tiles_c);
        const int64_t r0 = (int64_t)tr * F8_BLOCK, c0 = (int64_t)tc * TC;
        if (r0 >= s.rows || c0 >= s.cols) continue;
        __syncthreads();   // the tile before has been read
#pragma unroll
        for (int i = 0; i < TC * 16 / NT; ++i) {
            const int j = (i * NT + t) >> 4, at = ((i * NT + t) & 15) * 8;
            const int r = (int)r0 + at, rows = c0 + j < s.cols ? s.rows : 0;
            const Raw8<QT> raw = load8<QT>(static_cast<const char*>(s.x) + (c0 + j) * (int64_t)s.ldx, r, rows);
            *reinterpret_cast<u32x2*>(turn + j * QPITCH + at) = settle8<QT>(raw, r, rows).w;
        }
        if (t < TC) scale[t] = c0 + t < s.cols ? scale_of(static_cast<const uint8_t*>(s.scales)[(c0 + t) * s.lds + tr]) : 0.0f;
        __syncthreads();
        const int64_t c = c0 + co * 8;
        uint32_t four[8];   // rows 4 rg .. + 3 of each column
#pragma unroll
        for (int e = 0; e < 8; ++e) four[e] = *reinterpret_cast<const uint32_t*>(turn + (co * 8 + e) * QPITCH + rg * 4);
        float v[4][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            Raw8<QT> raw{};
            raw.w[0] = four[e];
            float u[8];
            widen<QT>(raw, scale[co * 8 + e], u);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i][e] = GELU ? gelu_of<YT == T_BF16>(u[i]) : u[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + rg * 4 + i;
            if (r < s.rows) store8<YT>(static_cast<char*>(s.out) + (r * s.ldo + c) * bytes_of<YT>, narrow<YT>(v[i]), (int)(c < s.cols ? s.cols - c : 0), p.streams & STREAM_OUT);
        }
    }
}

// da = dh gelu'(a).  AT: the pre-activation's type, 8 bits or as it was.  Bound by HBM: 8192 x 16384 on eight devices from 8 bits (672 MB) 110 us, 6.1 TB/s.
template <int AT, int YT, bool IN>
__global__ __launch_bounds__(NT) void gelu_grad_kernel(Block8Plan p) {
    const Block8Shard& s = p.s[blockIdx.y];
    if (s.rows == 0 || s.cols == 0) return;
    const int lane = threadIdx.x & 15;
    for (UnitWalk w(s.cols); w.r < (uint32_t)s.rows; w.next()) {
        const int c = (int)w.b * UNIT + lane * 8;
        const char* const from_a = static_cast<const char*>(s.x) + w.at(s.ldx) * bytes_of<AT>;
        const char* const from_h = static_cast<const char*>(s.dh) + w.at(s.lddh) * bytes_of<YT>;
        char* const to = static_cast<char*>(s.out) + (w.at(s.ldo) + c) * bytes_of<YT>;
        Raw8<AT> ra[2];
        Raw8<YT> rh[2];
        uint32_t byte[2] = {127, 127};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            ra[u] = load8<AT, IN>(from_a, c + u * F8_BLOCK, s.cols);
            rh[u] = load8<YT, IN>(from_h, c + u * F8_BLOCK, s.cols);
            if constexpr (bytes_of<AT> == 1) {
                const uint8_t* const scales = static_cast<const uint8_t*>(s.scales) + w.at(s.lds) + w.b * 2;
                byte[u] = scales[(int)w.b * UNIT + u * F8_BLOCK < s.cols ? u : 0];
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float a[8], h[8];
            widen<AT>(settle8<AT>(ra[u], c + u * F8_BLOCK, s.cols), scale_of(byte[u]), a);
            widen<YT>(settle8<YT>(rh[u], c + u * F8_BLOCK, s.cols), 1.0f, h);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] *= gelu_slope<YT == T_BF16>(a[e]);
            store8<YT>(to + u * F8_BLOCK * bytes_of<YT>, narrow<YT>(h), s.cols - c - u * F8_BLOCK, p.streams & STREAM_OUT);
        }
    }
}

// grid of the kernels that walk pairs of blocks
dim3 walk_grid(const Block8Plan& plan) {
    int64_t most = 0;
    for (int i = 0; i < plan.k; ++i) most = std::max(most, plan.s[i].rows * (((int64_t)plan.s[i].cols + UNIT - 1) / UNIT));
    int64_t bx = (most + NT / 16 - 1) / (NT / 16);
    bx = std::min<int64_t>(bx, (1 << 16) / plan.k);
    return dim3((uint32_t)std::max<int64_t>(bx, 1), (uint32_t)plan.k);
}
struct TileGrid {
    dim3 grid;
    int rows, cols;
};
TileGrid tile_grid(const Block8Plan& plan) {
    TileGrid g{};
    for (int i = 0; i < plan.k; ++i) {
        g.rows = std::max(g.rows, tiles_along(plan.s[i].rows, F8_BLOCK));
        g.cols = std::max(g.cols, tiles_along(plan.s[i].cols, TC));
    }
    const int64_t bx = std::min<int64_t>((int64_t)g.rows * g.cols, (1 << 18) / plan.k);
    g.grid = dim3((uint32_t)std::max<int64_t>(bx, 1), (uint32_t)plan.k);
    return g;
}

template <typename F>
void with_f8(int32_t f8, F&& f) {
    if (f8 == SBP_F8E4M3) f(std::integral_constant<int, T_E4M3>{});
    else f(std::integral_constant<int, T_E5M2>{});
}
template <typename F>
void with_wide(int32_t dtype, F&& f) {
    if (dtype == SBP_BF16) f(std::integral_constant<int, T_BF16>{});
    else f(std::integral_constant<int, T_F32>{});
}
template <typename F>
void with_bool(bool b, F&& f) {
    if (b) f(std::true_type{});
    else f(std::false_type{});
}

int bytes_each(int32_t dtype) { return dtype == SBP_F32 ? 4 : dtype == SBP_BF16 ? 2 : 1; }
// in: bytes of an element read; out_dtype: of the results
Block8Plan with_streams(Block8Plan plan, int in, int32_t out_dtype) {
    const int out = bytes_each(out_dtype);
    int64_t elements = 0;
    bool on_lines = true;
    for (int i = 0; i < plan.k; ++i) {
        const Block8Shard& s = plan.s[i];
        elements += (int64_t)s.rows * s.cols;
        if ((int64_t)s.ldo * out % 128 || reinterpret_cast<uintptr_t>(s.out) % 128) on_lines = false;
    }
    plan.streams = streams_of(elements * in, elements * out, on_lines, out_dtype);
    return plan;
}

}  // namespace

int32_t launch_quantize(const Block8Plan& given, hipStream_t stream) {
    const Block8Plan plan = with_streams(given, bytes_each(given.dtype), given.f8);
    with_f8(plan.f8, [&](auto q) {
        with_wide(plan.dtype, [&](auto x) {
            with_bool(plan.gelu != 0, [&](auto gelu) {
                if (plan.trans) {
                    const TileGrid g = tile_grid(plan);
                    hipLaunchKernelGGL((quantize_transposed_kernel<x(), q(), gelu()>), g.grid, dim3(NT), 0, stream, plan, g.rows, g.cols);
                } else {
                    with_bool(plan.streams & STREAM_IN, [&](auto in) { hipLaunchKernelGGL((quantize_kernel<x(), q(), gelu(), in()>), walk_grid(plan), dim3(NT), 0, stream, plan); });
                }
            });
        });
    });
    return launch_status(__func__);
}

int32_t launch_dequantize(const Block8Plan& given, hipStream_t stream) {
    const Block8Plan plan = with_streams(given, 1, given.dtype);
    with_f8(plan.f8, [&](auto q) {
        with_wide(plan.dtype, [&](auto y) {
            with_bool(plan.gelu != 0, [&](auto gelu) {
                if (plan.trans) {
                    const TileGrid g = tile_grid(plan);
                    hipLaunchKernelGGL((dequantize_transposed_kernel<q(), y(), gelu()>), g.grid, dim3(NT), 0, stream, plan, g.rows, g.cols);
                } else {
                    with_bool(plan.streams & STREAM_IN, [&](auto in) { hipLaunchKernelGGL((dequantize_kernel<q(), y(), gelu(), in()>), walk_grid(plan), dim3(NT), 0, stream, plan); });
                }
            });
        });
    });
    return launch_status(__func__);
}

int32_t launch_gelu_grad(const Block8Plan& given, hipStream_t stream) {
    const Block8Plan plan = with_streams(given, bytes_each(given.f8) + bytes_each(given.dtype), given.dtype);
    with_wide(plan.dtype, [&](auto y) {
        auto go = [&](auto a) {
            with_bool(plan.streams & STREAM_IN, [&](auto in) { hipLaunchKernelGGL((gelu_grad_kernel<a(), y(), in()>), walk_grid(plan), dim3(NT), 0, stream, plan); });
        };
        if (plan.f8 == SBP_F8E4M3 || plan.f8 == SBP_F8E5M2) with_f8(plan.f8, go);
        else with_wide(plan.f8, go);
    });
    return launch_status(__func__);
}

}  // namespace sbp
