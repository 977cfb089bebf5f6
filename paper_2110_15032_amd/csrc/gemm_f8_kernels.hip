// Products of 8-bit tensors: C[m, n] = sum over blocks b of 128 of 2^(ea[m, b] + eb[n, b]) sum over the block of A[m, kk] B[n, kk].
//
// Two forms of the inner sum.  bf16 results: the 8-bit matrix instruction (16x16x128, both scales in the instruction).  It aligns the
// products of a group to the largest and drops what lies about 2^-12 below it, an error of some 2^-16 of the result, well under the 2^-8
// of its rounding.  fp32 results: both operands widened to bf16 with their scales (exact) for the bf16 matrix instruction, at half the rate,
// whose sums are fp32's.
//
// The instruction's first operand is B (weights), so that a lane holds one row m and four consecutive columns n of the result.
#include "block8_device.h"

namespace sbp {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef u32x4 __attribute__((aligned(1))) u32x4_byte;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef u32x2 __attribute__((aligned(2))) u32x2_half;

// 32 bytes of a row: 16 from `at` and 16 from `at` + 64, which with four lanes to a row makes the row's block of 128.  (The order of a
// block's values does not matter, as long as both operands have the same.)
struct Frag {
    u32x4 lo, hi;
};
__device__ inline u32x4 load_some(const uint8_t* at, int valid) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (valid >= 16) return *reinterpret_cast<const u32x4_byte*>(at);
#pragma unroll
    for (int e = 0; e < 15; ++e)
        if (e < valid) v[e >> 2] |= (uint32_t)at[e] << (8 * (e & 3));
    return v;
}
template <bool WHOLE>
__device__ inline Frag load_frag(const uint8_t* at, int valid) {
    if constexpr (WHOLE) return {*reinterpret_cast<const u32x4_byte*>(at), *reinterpret_cast<const u32x4_byte*>(at + 64)};
    else return {load_some(at, valid), load_some(at + 64, valid - 64)};
}

template <int T>
__device__ inline bf16x8 widen_frag(uint32_t a, uint32_t b, float scale) {
    bf16x2 v[4];
    if constexpr (T == T_E4M3) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(a, scale, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(a, scale, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(b, scale, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(b, scale, true);
    }
    return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]), __builtin_bit_cast(uint32_t, v[3])});
}

// An operand's 32 values as the matrix instructions take them.
template <int T, bool EXACT>
struct Operand;
template <int T>
struct Operand<T, false> {
    i32x8 v;
    int scale;
    __device__ Operand(const Frag& f, uint32_t byte) : scale((int)byte) {
        v = i32x8{(int)f.lo[0], (int)f.lo[1], (int)f.lo[2], (int)f.lo[3], (int)f.hi[0], (int)f.hi[1], (int)f.hi[2], (int)f.hi[3]};
    }
};
template <int T>
struct Operand<T, true> {
    bf16x8 v[4];
    __device__ Operand(const Frag& f, uint32_t byte) {
        const float s = scale_of(byte);
        v[0] = widen_frag<T>(f.lo[0], f.lo[1], s);
        v[1] = widen_frag<T>(f.lo[2], f.lo[3], s);
        v[2] = widen_frag<T>(f.hi[0], f.hi[1], s);
        v[3] = widen_frag<T>(f.hi[2], f.hi[3], s);
    }
};
template <int BT, int AT>
__device__ inline f32x4 multiply(const Operand<BT, false>& b, const Operand<AT, false>& a, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, c, BT == T_E5M2, AT == T_E5M2, 0, b.scale, 0, a.scale);
}
template <int BT, int AT>
__device__ inline f32x4 multiply(const Operand<BT, true>& b, const Operand<AT, true>& a, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
}

template <bool F32, bool GELU>
__device__ inline float finish(float v) {
    if constexpr (!GELU) return v;
    else if constexpr (F32) return gelu_erf(v);
    else return gelu_fast(v);
}

// four consecutive columns of a row, at any alignment
template <bool F32, bool GELU>
__device__ inline void store4(const GemmF8Shard& s, int64_t m, int n, f32x4 v) {
    if (m >= s.m || n >= s.n) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = finish<F32, GELU>(v[e]);
    if constexpr (F32) {
        float* dst = static_cast<float*>(s.c) + m * s.ldc + n;
        if (n + 4 <= s.n) *reinterpret_cast<f32x4_any*>(dst) = v;
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < s.n) dst[e] = v[e];
    } else {
        uint16_t* dst = static_cast<uint16_t*>(s.c) + m * s.ldc + n;
        const u32x2 w = {f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3])};
        if (n + 4 <= s.n) *reinterpret_cast<u32x2_half*>(dst) = w;
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (n + e < s.n) dst[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}

// Few rows: the weights are the traffic, and every workgroup streams 16 of their rows past MB blocks of 16 rows of A, its four waves
// taking every fourth block of the reduction.  No LDS before the sums meet; operands at any pitch.
template <int AT, int BT, bool F32, bool GELU, int MB>
__global__ __launch_bounds__(256) void gemm_f8_stream_kernel(GemmF8Plan p, int tiles_m) {
    constexpr bool EXACT = F32;
    const GemmF8Shard& s = p.s[blockIdx.y];
    const int tn = blockIdx.x / tiles_m, tm = blockIdx.x % tiles_m;
    const int64_t n0 = (int64_t)tn * 16, m0 = (int64_t)tm * (16 * MB);
    if (n0 >= s.n || m0 >= s.m) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t n = min(n0 + r, (int64_t)s.n - 1);
    const uint8_t* const b = s.b + n * s.ldb + g * 16;
    const uint8_t* const bs = s.b_scales + n * s.ldbs;
    const uint8_t* a[MB];
    const uint8_t* as[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const int64_t m = min(m0 + i * 16 + r, (int64_t)s.m - 1);
        a[i] = s.a + m * s.lda + g * 16;
        as[i] = s.a_scales + m * s.ldas;
    }
    f32x4 acc[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int whole = s.kk / F8_BLOCK, blocks = (s.kk + F8_BLOCK - 1) / F8_BLOCK;
#pragma unroll 4
    for (int kb = wave; kb < whole; kb += 4) {
        const int64_t at = (int64_t)kb * F8_BLOCK;
        const Operand<BT, EXACT> ob(load_frag<true>(b + at, 128), bs[kb]);
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i] = multiply<BT, AT>(ob, Operand<AT, EXACT>(load_frag<true>(a[i] + at, 128), as[i][kb]), acc[i]);
    }
    if (whole < blocks && wave == (whole & 3)) {
        const int64_t at = (int64_t)whole * F8_BLOCK;
        const int valid = s.kk - whole * F8_BLOCK - g * 16;
        const Operand<BT, EXACT> ob(load_frag<false>(b + at, valid), bs[whole]);
#pragma unroll
        for (int i = 0; i < MB; ++i) acc[i] = multiply<BT, AT>(ob, Operand<AT, EXACT>(load_frag<false>(a[i] + at, valid), as[i][whole]), acc[i]);
    }
    __shared__ f32x4 sums[4][MB][64];
#pragma unroll
    for (int i = 0; i < MB; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MB; i += 4) {
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += sums[w][i][lane];
        store4<F32, GELU>(s, m0 + i * 16 + r, (int)n0 + g * 4, v);
    }
}

}  // namespace

int32_t launch_gemm_f8(const GemmF8Plan& plan, hipStream_t stream) {
    int max_m = 0, max_n = 0;
    for (int g = 0; g < plan.groups; ++g) {
        max_m = std::max(max_m, plan.s[g].m);
        max_n = std::max(max_n, plan.s[g].n);
    }
    if (max_m == 0 || max_n == 0) return SBP_OK;
    auto types = [&](auto f) {
        auto second = [&](auto a) {
            if (plan.b_dtype == SBP_F8E4M3) f(a, std::integral_constant<int, T_E4M3>{});
            else f(a, std::integral_constant<int, T_E5M2>{});
        };
        if (plan.a_dtype == SBP_F8E4M3) second(std::integral_constant<int, T_E4M3>{});
        else second(std::integral_constant<int, T_E5M2>{});
    };
    auto results = [&](auto f) {
        auto second = [&](auto o) {
            if (plan.epilogue == SBP_EPI_GELU) f(o, std::true_type{});
            else f(o, std::false_type{});
        };
        if (plan.out_dtype == SBP_F32) second(std::true_type{});
        else second(std::false_type{});
    };
    int32_t st = SBP_OK;
    types([&](auto a, auto b) {
        results([&](auto f32, auto gelu) {
            auto stream_rows = [&](auto mb) {
                const int tm = tiles_along(max_m, 16 * mb()), tn = tiles_along(max_n, 16);
                if (!grid_fits((int64_t)tm * tn, 256)) {
                    st = SBP_ERR_UNSUPPORTED;
                    return;
                }
                hipLaunchKernelGGL((gemm_f8_stream_kernel<a(), b(), f32(), gelu(), mb()>), dim3((uint32_t)(tm * tn), (uint32_t)plan.groups), dim3(256), 0, stream, plan, tm);
            };
            if (max_m <= 16) stream_rows(std::integral_constant<int, 1>{});
            else stream_rows(std::integral_constant<int, 4>{});
        });
    });
    return st != SBP_OK ? st : launch_status(__func__);
}

}  // namespace sbp
