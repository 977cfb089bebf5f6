// Device-side building blocks of 8-bit tensors (values with one power of two for every 128 of a stored row) and of row kernels that
// read and write eight consecutive elements a lane at any alignment.  Everything is internal (anonymous namespace).
#pragma once
#include "gemm_device.h"

namespace sbp {
namespace {

typedef u32x2 __attribute__((aligned(1))) u32x2_any;
typedef u32x4 __attribute__((aligned(1))) u32x4_byte;
typedef short s16x2 __attribute__((ext_vector_type(2)));

// element types as template arguments
enum ElemType : int { T_F32 = SBP_F32, T_BF16 = SBP_BF16, T_E4M3 = SBP_F8E4M3, T_E5M2 = SBP_F8E5M2 };
template <int T>
constexpr int bytes_of = T == T_F32 ? 4 : T == T_BF16 ? 2 : 1;

// Eight consecutive elements as they are stored.
template <int T>
struct Raw8;
template <>
struct Raw8<T_F32> {
    f32x4 a, b;
};
template <>
struct Raw8<T_BF16> {
    u32x4 w;
};
template <>
struct Raw8<T_E4M3> {
    u32x2 w;
};
template <>
struct Raw8<T_E5M2> {
    u32x2 w;
};

// Eight elements of a row from column c on, those behind its end (`cols`) as whatever settle8 makes zero: where the row ends among them its last
// eight are read, and nothing outside the row.  The loads are all that happens here, so that a row can be on its way while another is worked on
// (only a row shorter than eight is put together at once).  STREAM: past the caches (a
// template argument, since the compiler takes the two forms of a load in two branches for one).
template <int T, bool STREAM = false>
__device__ inline Raw8<T> load8(const char* row, int c, int cols) {
    Raw8<T> r{};
    if (c >= cols) return r;
    if (cols >= 8) {
        const char* const p = row + (int64_t)min(c, cols - 8) * bytes_of<T>;
        if constexpr (STREAM) {
            if constexpr (T == T_F32) {
                r.a = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(p));
                r.b = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(p + 16));
            } else if constexpr (T == T_BF16) r.w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p));
            else r.w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any*>(p));
        } else {
            if constexpr (T == T_F32) {
                r.a = *reinterpret_cast<const f32x4_any*>(p);
                r.b = *reinterpret_cast<const f32x4_any*>(p + 16);
            } else if constexpr (T == T_BF16) r.w = *reinterpret_cast<const u32x4_any*>(p);
            else r.w = *reinterpret_cast<const u32x2_any*>(p);
        }
    } else {   // c is 0
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < cols) {
                if constexpr (T == T_F32) {
                    const float v = reinterpret_cast<const float*>(row)[e];
                    if (e < 4) r.a[e] = v;
                    else r.b[e - 4] = v;
                } else if constexpr (T == T_BF16) r.w[e >> 1] |= (uint32_t) reinterpret_cast<const uint16_t*>(row)[e] << (16 * (e & 1));
                else r.w[e >> 2] |= (uint32_t) reinterpret_cast<const uint8_t*>(row)[e] << (8 * (e & 3));
            }
    }
    return r;
}
template <int T>
__device__ inline Raw8<T> settle8(Raw8<T> r, int c, int cols) {
    const int gone = c + 8 - cols;   // 1 .. 7: that many elements in front belong to the lane before
    if (gone <= 0 || gone >= 8 || cols < 8) return r;
    if constexpr (T == T_F32) {
        float v[8] = {r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]};
#pragma unroll
        for (int by = 4; by > 0; by >>= 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = gone & by ? (e + by < 8 ? v[e + by] : 0.0f) : v[e];
        return {f32x4{v[0], v[1], v[2], v[3]}, f32x4{v[4], v[5], v[6], v[7]}};
    } else if constexpr (T == T_BF16) {
        const uint64_t lo = (uint64_t)r.w[1] << 32 | r.w[0], hi = (uint64_t)r.w[3] << 32 | r.w[2];
        const int bits = gone * 16 & 63;
        const uint64_t x = gone >= 4 ? hi >> bits : lo >> bits | hi << (64 - bits), y = gone >= 4 ? 0 : hi >> bits;
        return {u32x4{(uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32)}};
    } else {
        const uint64_t x = ((uint64_t)r.w[1] << 32 | r.w[0]) >> (gone * 8);
        return {u32x2{(uint32_t)x, (uint32_t)(x >> 32)}};
    }
}
template <int T>
__device__ inline void store8(void* at, const Raw8<T> r, int valid, bool stream = false) {
    char* p = static_cast<char*>(at);
    if (valid >= 8 && stream) {
        if constexpr (T == T_F32) {
            __builtin_nontemporal_store(r.a, reinterpret_cast<f32x4_any*>(p));
            __builtin_nontemporal_store(r.b, reinterpret_cast<f32x4_any*>(p + 16));
        } else if constexpr (T == T_BF16) __builtin_nontemporal_store(r.w, reinterpret_cast<u32x4_any*>(p));
        else __builtin_nontemporal_store(r.w, reinterpret_cast<u32x2_any*>(p));
    } else if (valid >= 8) {
        if constexpr (T == T_F32) {
            *reinterpret_cast<f32x4_any*>(p) = r.a;
            *reinterpret_cast<f32x4_any*>(p + 16) = r.b;
        } else if constexpr (T == T_BF16) *reinterpret_cast<u32x4_any*>(p) = r.w;
        else *reinterpret_cast<u32x2_any*>(p) = r.w;
    } else if (valid > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < valid) {
                if constexpr (T == T_F32) reinterpret_cast<float*>(p)[e] = e < 4 ? r.a[e] : r.b[e - 4];
                else if constexpr (T == T_BF16) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(r.w[e >> 1] >> (16 * (e & 1)));
                else reinterpret_cast<uint8_t*>(p)[e] = (uint8_t)(r.w[e >> 2] >> (8 * (e & 3)));
            }
    }
}

// Which of a pass's tensors go past the caches.  Results: as much as the L2 caches of all XCDs hold and more, in rows that start on cache lines (else neighbouring
// waves share lines, which L2 has to keep for both).  Inputs: when the pass has more than the memory-side cache holds.  us, cached / results past
// them / inputs too: 8192 x 8192 from 8 bits to bf16 38.2 / 29.3 / 34.7, 16384 x 16384 bytes of GeLU's gradient (672 MB) 120.7 / 113.0 /
// 110.0, 8192 x 16384 into 8 bits (404 MB) 69.5 / 67.2 / 63.2, normalising 8192 x 4096 in bf16 26.9 / 22.8 / 27.2, 8192 x 4097 in
// fp32 58.1 / 58.8 / 56.6.
enum Streams : int32_t { STREAM_OUT = 1, STREAM_IN = 2 };
// fp32 results stay cached, as a lane stores its eight in two pieces (8192 x 4096 of GeLU's gradient 69.6, past the caches 72.8).
inline int32_t streams_of(int64_t read, int64_t wrote, bool on_lines, int32_t out_dtype) {
    return (wrote >= (int64_t)32 << 20 && on_lines && out_dtype != SBP_F32 ? STREAM_OUT : 0) | (read + wrote > (int64_t)256 << 20 ? STREAM_IN : 0);
}

// gelu of results in fp32: gelu_erf, but 0 of minus infinity, as gelu_fast has it (as a factor it is the lowest number, next to an erfc of 0)
__device__ inline float gelu_whole(float x) { return 0.5f * __builtin_amdgcn_fmed3f(x, -3.4028235e38f, INFINITY) * erfcf(x * -0.70710678118654752f); }

// A scale byte b stands for 2^(b - 127).  The conversions below take a power of two as the exponent field of an fp32 number, 0 there
// standing for 2^-127.
__device__ inline float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Widening: exact (an 8-bit value times a power of two is an fp32 number).  `scale`: scale_of() for 8-bit types, not looked at else.
template <int T>
__device__ inline void widen(const Raw8<T> r, float scale, float (&v)[8]) {
    if constexpr (T == T_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = r.a[e];
            v[e + 4] = r.b[e];
        }
    } else if constexpr (T == T_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(r.w[e] << 16);
            v[2 * e + 1] = __uint_as_float(r.w[e] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            f32x2 lo, hi;
            if constexpr (T == T_E4M3) {
                lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(r.w[d], scale, false);
                hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(r.w[d], scale, true);
            } else {
                lo = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(r.w[d], scale, false);
                hi = __builtin_amdgcn_cvt_scalef32_pk_f32_bf8(r.w[d], scale, true);
            }
            v[4 * d] = lo[0];
            v[4 * d + 1] = lo[1];
            v[4 * d + 2] = hi[0];
            v[4 * d + 3] = hi[1];
        }
    }
}

// Rounding to the nearest, ties to even.
template <int T>
__device__ inline Raw8<T> narrow(const float (&v)[8]) {
    static_assert(T == T_F32 || T == T_BF16, "8-bit types need a scale");
    Raw8<T> r;
    if constexpr (T == T_F32) {
        r.a = f32x4{v[0], v[1], v[2], v[3]};
        r.b = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int d = 0; d < 4; ++d) r.w[d] = f32_to_bf16x2(v[2 * d], v[2 * d + 1]);
    }
    return r;
}
// four values over 2^e, rounded to nearest even; NaN stays NaN, infinity becomes NaN (e4m3 has none) or stays (e5m2)
template <int T>
__device__ inline uint32_t narrow4(float a, float b, float c, float d, float scale) {
    s16x2 r = {0, 0};
    if constexpr (T == T_E4M3) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, a, b, scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, c, d, scale, true);
    }
    return __builtin_bit_cast(uint32_t, r);
}

// The scale byte of a block whose largest finite magnitude is `most`: the smallest e >= -127 with most / 2^e within the type, whose
// largest value is 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2), so nothing saturates.  On the bits: the exponent, one more where the
// fraction passes 0.75.
template <int T>
__device__ inline uint32_t scale_byte(float most) {
    const int e = (int)((__float_as_uint(most) + 0x1FFFFFu) >> 23) - (T == T_E4M3 ? 8 : 15);
    return (uint32_t)(e > 0 ? e : 0);
}

// Sums and maxima over the lanes of a wave.  The first four steps stay inside rows of 16 lanes (DPP: neighbours, pairs, mirrored halves,
// mirrored row), which is one block of 128 values at eight a lane.  Maxima are taken of magnitudes as bits (magnitude()).
template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ inline float dpp(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
__device__ inline float sum_wave(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    auto h = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
    h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

// The largest of a lane's magnitudes as bits, on which whatever is not finite is above every number.  COMPUTED values: an instruction for three, which
// passes over a NaN next to a number.  So it does with a quiet one, which is what arithmetic gives; a signalling one, as memory may hold it,
// becomes the result, and the next maximum passes over that with all that had been found.  Other values are therefore compared as bits:
// an instruction more for each (8192 x 16384 from bf16 63.3 us either way; with GeLU it would be 88.6 instead of 85.3).
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ inline float max3_abs(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
template <bool COMPUTED>
__device__ inline uint32_t most_of(float a, float b, float c, float d) {
    if constexpr (COMPUTED) return __float_as_uint(max3_abs(max3_abs(a, b, c), d, d));
    else return max(max(magnitude(a), magnitude(b)), max(magnitude(c), magnitude(d)));
}
template <bool COMPUTED>
__device__ inline uint32_t most_of_8(const float (&v)[8]) {
    if constexpr (COMPUTED) {
        const float m = max3_abs(v[0], v[1], v[2]);
        return __float_as_uint(max3_abs(max3_abs(m, v[3], v[4]), v[5], max3_abs(v[6], v[7], v[7])));
    } else return max(most_of<false>(v[0], v[1], v[2], v[3]), most_of<false>(v[4], v[5], v[6], v[7]));
}
__device__ inline uint32_t finite_magnitude(float v) { return magnitude(v) < 0x7F800000u ? magnitude(v) : 0u; }
__device__ inline uint32_t most_finite_of_8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, finite_magnitude(v[e]));
    return m;
}

// 8-bit form of N times eight values, 16 lanes to a block of 128, and the blocks' scale bytes.  The largest finite magnitude counts: blocks with a value that
// is not finite (COMPUTED: an infinity, or of NaN alone) are gone through again; the lanes of a block go there together.  The N
// chains over lanes are written side by side, each step of one fills the wait of the others.
template <bool COMPUTED, int T, int N>
__device__ inline void narrow_blocks(const float (&v)[N][8], Raw8<T> (&q)[N], uint32_t (&byte)[N]) {
    uint32_t m[N];
    bool finite = true;
#pragma unroll
    for (int n = 0; n < N; ++n) m[n] = most_of_8<COMPUTED>(v[n]);
    auto over_rows = [&]() {
#pragma unroll
        for (int n = 0; n < N; ++n) m[n] = max(m[n], dpp<0xB1>(m[n]));
#pragma unroll
        for (int n = 0; n < N; ++n) m[n] = max(m[n], dpp<0x4E>(m[n]));
#pragma unroll
        for (int n = 0; n < N; ++n) m[n] = max(m[n], dpp<0x141>(m[n]));
#pragma unroll
        for (int n = 0; n < N; ++n) m[n] = max(m[n], dpp<0x140>(m[n]));
    };
    over_rows();
#pragma unroll
    for (int n = 0; n < N; ++n) finite = finite && m[n] < 0x7F800000u;
    if (!finite) {
        asm volatile("");   // or it would be worked out always, and chosen from
#pragma unroll
        for (int n = 0; n < N; ++n) m[n] = most_finite_of_8(v[n]);
        over_rows();
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        byte[n] = scale_byte<T>(__uint_as_float(m[n]));
        const float s = scale_of(byte[n]);
        q[n].w[0] = narrow4<T>(v[n][0], v[n][1], v[n][2], v[n][3], s);
        q[n].w[1] = narrow4<T>(v[n][4], v[n][5], v[n][6], v[n][7], s);
    }
}

}  // namespace
}  // namespace sbp
