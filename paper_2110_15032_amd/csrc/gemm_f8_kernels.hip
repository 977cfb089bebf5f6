// Products of 8-bit tensors: C[m, n] = sum over blocks b of 128 of 2^(ea[m, b] + eb[n, b]) sum over the block of A[m, kk] B[n, kk].
//
// Two forms of the inner sum.  bf16 results: the 8-bit matrix instruction (16x16x128, both scales in the instruction).  Measured here, for either
// type: it takes the products of eight consecutive values together, finds the largest sum of their operands' exponents (a subnormal number's being the
// smallest normal one's), cuts every product toward zero at 2^-13 of that power of two, and adds the sums of eights in fp32.  So an eight is off by less
// than 2^-10 of its largest |a| times its largest |b|; on random operands a result is off by 1e-5 to 6e-5 of the results' root mean square (2^-17 ..
// 2^-14), next to the 2^-9 that rounding to bf16 costs on average.  fp32 results: both operands widened to bf16 with their scales (exact) for the bf16 matrix
// instruction, at half the rate, whose sums are fp32's.
//
// The instruction's first operand is B (weights), so that a lane holds one row m and four consecutive columns n of the result.
#include "block8_device.h"
#include "gemm_f8_choice.h"
#include "gemm_f8_stage.h"

namespace sbp {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef u32x2 __attribute__((aligned(2))) u32x2_half;

// 32 bytes of a row: 16 from `at` and 16 from `at` + 64, which with four lanes to a row makes the row's block of 128.  (The order of a
// block's values does not matter, as long as both operands have the same.)
struct Frag {
    u32x4 lo, hi;
};
// 16 bytes at `at`, those from `valid` on zero; `before` bytes of the row lie in front.  Nothing outside the row is read: where it ends among the 16,
// its last 16 are read and shifted.
__device__ inline u32x4 load_some(const uint8_t* at, int valid, int before) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (valid >= 16) return *reinterpret_cast<const u32x4_byte*>(at);
    if (valid <= 0) return v;
    if (before + valid >= 16) {
        const int gone = 16 - valid;   // bytes to shift out, 1 .. 15
        const u32x4 w = *reinterpret_cast<const u32x4_byte*>(at - gone);
        const uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
        const int bits = gone * 8 & 63;
        const uint64_t a = gone >= 8 ? hi >> bits : bits ? lo >> bits | hi << (64 - bits) : lo, b = gone >= 8 ? 0 : hi >> bits;
        return u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    }
    uint64_t lo = 0, hi = 0;   // a row of fewer than 16
#pragma unroll 1
    for (int e = valid - 1; e >= 0; --e) {
        hi = hi << 8 | lo >> 56;
        lo = lo << 8 | at[e];
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ inline Frag load_frag(const uint8_t* at) { return {*reinterpret_cast<const u32x4_byte*>(at), *reinterpret_cast<const u32x4_byte*>(at + 64)}; }

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

// An operand's 32 values as the matrix instructions take them, with the scale in the low byte of `byte`.
template <int T, bool EXACT>
struct Operand;
template <int T>
struct Operand<T, false> {
    i32x8 v;
    int scale;
    Operand() = default;
    __device__ Operand(const Frag& f, uint32_t byte) : scale((int)byte) {
        v = i32x8{(int)f.lo[0], (int)f.lo[1], (int)f.lo[2], (int)f.lo[3], (int)f.hi[0], (int)f.hi[1], (int)f.hi[2], (int)f.hi[3]};
    }
};
template <int T>
struct Operand<T, true> {
    bf16x8 v[4];
    Operand() = default;
    __device__ Operand(const Frag& f, uint32_t byte) {
        const float s = scale_of(byte & 255u);
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
    else if constexpr (F32) return gelu_whole(v);
    else return gelu_fast(v);
}

// N consecutive columns of a row, at any alignment; whole: all of them exist
template <bool F32, bool GELU, int N>
__device__ inline void store_row(const GemmF8Shard& s, int64_t m, int n, bool whole, const f32x4 (&v)[N / 4]) {
    static_assert(F32 ? N == 4 : N == 4 || N == 8, "up to 16 bytes");
    if (!whole && (m >= s.m || n >= s.n)) return;
    float u[N];
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = finish<F32, GELU>(v[e >> 2][e & 3]);
    if constexpr (F32) {
        float* dst = static_cast<float*>(s.c) + m * s.ldc + n;
        if (whole || n + N <= s.n) *reinterpret_cast<f32x4_any*>(dst) = f32x4{u[0], u[1], u[2], u[3]};
        else
#pragma unroll
            for (int e = 0; e < N - 1; ++e)
                if (n + e < s.n) dst[e] = u[e];
    } else {
        uint16_t* dst = static_cast<uint16_t*>(s.c) + m * s.ldc + n;
        if (whole || n + N <= s.n) {
            if constexpr (N == 8) *reinterpret_cast<u32x4_any*>(dst) = u32x4{f32_to_bf16x2(u[0], u[1]), f32_to_bf16x2(u[2], u[3]), f32_to_bf16x2(u[4], u[5]), f32_to_bf16x2(u[6], u[7])};
            else *reinterpret_cast<u32x2_half*>(dst) = u32x2{f32_to_bf16x2(u[0], u[1]), f32_to_bf16x2(u[2], u[3])};
        } else {
#pragma unroll
            for (int e = 0; e < N - 1; ++e)
                if (n + e < s.n) dst[e] = f32_to_bf16(u[e]);
        }
    }
}

// an address that every lane has, in scalar registers
__device__ inline gbl_char* uniform(gbl_char* at) {
    const uint64_t v = (uint64_t)(uintptr_t)at;
    return (gbl_char*)(uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v));
}

// The last, cut block of a reduction, on the wave whose turn it is: straight from memory, at any pitch.
template <int AT, int BT, bool EXACT, int MB, int NB>
__device__ inline void multiply_cut_block(const uint8_t* a, const uint32_t (&a_row)[MB], const uint32_t (&as)[MB], const uint8_t* b, const uint32_t (&b_row)[NB],
                                          const uint32_t (&bs)[NB], int left, int before, f32x4 (&acc)[MB][NB]) {
    Operand<BT, EXACT> ob[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) ob[j] = Operand<BT, EXACT>({load_some(b + b_row[j], left, before), load_some(b + b_row[j] + 64, left - 64, before + 64)}, bs[j]);
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const Operand<AT, EXACT> oa({load_some(a + a_row[i], left, before), load_some(a + a_row[i] + 64, left - 64, before + 64)}, as[i]);
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = multiply<BT, AT>(ob[j], oa, acc[i][j]);
    }
}

// Tiles of MB 16 rows by NB 16 columns whose four waves take every fourth block of the reduction: for few rows, where the weights are the traffic,
// and for few tiles.  The waves' sums meet in LDS, in order.
// Bound by the weights' bytes: 1 x 4096 x 16384 on eight devices (68 MB) 11.9 us, 5.7 TB/s; for some 32 rows and more by the loads of a compute unit.
// RING: every wave brings its blocks into LDS of its own, DEPTH of them on their way: a load takes whole cache lines of eight rows, where one into
// registers takes halves of sixteen (choose_f8_tile has both measured), and what is on its way costs no registers.  Nobody else reads it, so there is no
// barrier before the sums.  Needs rows 16-byte and scales 4-byte aligned; else (any pitch) two sets of registers, U blocks each.
template <int AT, int BT, bool F32, bool GELU, int MB, int NB, bool RING>
__global__ __launch_bounds__(256) void gemm_f8_wave_kernel(GemmF8Plan p, int tm, int tn, int order) {
    constexpr bool EXACT = F32;
    constexpr int NW = 4;
    const TileCoord t = map_tile(blockIdx.x, gridDim.x, tm, tn, p.groups, order);
    if (!t.valid) return;
    const GemmF8Shard& s = p.s[t.g];
    const int64_t m0 = (int64_t)t.tile_m * (MB * 16), n0 = (int64_t)t.tile_n * (NB * 16);
    if (m0 >= s.m || n0 >= s.n) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const uint8_t *const a = s.a + m0 * s.lda, *const as = s.a_scales + m0 * s.ldas, *const b = s.b + n0 * s.ldb, *const bs = s.b_scales + n0 * s.ldbs;
    const uint32_t last_m = (uint32_t)(s.m - 1 - (int)m0), last_n = (uint32_t)(s.n - 1 - (int)n0);   // rows past an operand's end are its last one
    uint32_t a_row[MB], as_row[MB], b_row[NB], bs_row[NB];   // of this lane's rows, from the tile's first
#pragma unroll
    for (int i = 0; i < MB; ++i) {
        const uint32_t m = min((uint32_t)(i * 16 + r), last_m);
        a_row[i] = m * (uint32_t)s.lda + g * 16;
        as_row[i] = m * (uint32_t)s.ldas;
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const uint32_t n = min((uint32_t)(j * 16 + r), last_n);
        b_row[j] = n * (uint32_t)s.ldb + g * 16;
        bs_row[j] = n * (uint32_t)s.ldbs;
    }
    f32x4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int whole = s.kk / F8_BLOCK, mine = (whole - wave + NW - 1) / NW;   // this wave's whole blocks

    // ring: a stage is 2 KB for each 16 rows (A's, then B's) and a dword of scales for each row
    constexpr int BLOCKS = MB + NB, SCALE_LOADS = (BLOCKS * 16 + 63) / 64, LOADS = 2 * BLOCKS + SCALE_LOADS, STAGE = BLOCKS * 2048 + SCALE_LOADS * 256;
    constexpr int DEPTH = std::max(2, std::min(4, 72 * 1024 / (NW * STAGE)));
    constexpr int SUMS = NW * MB * NB * 1024;
    __shared__ __attribute__((aligned(16))) char lds[RING ? std::max(NW * DEPTH * STAGE, SUMS) : SUMS];
    if constexpr (RING) {
        char* const ring = lds + wave * (DEPTH * STAGE);
        const uint32_t ring_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)ring);
        // load h of a block of 16 rows: row 8 h + lane / 8, chunk lane % 8 permuted by row / 2 (see StageF8)
        uint32_t from[2 * BLOCKS], scales_from[SCALE_LOADS];
#pragma unroll
        for (int l = 0; l < 2 * BLOCKS; ++l) {
            const int row = (l & 1) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            const bool of_a = l < 2 * MB;
            from[l] = min((uint32_t)((of_a ? l : l - 2 * MB) / 2 * 16 + row), of_a ? last_m : last_n) * (uint32_t)(of_a ? s.lda : s.ldb) + chunk * 16;
        }
#pragma unroll
        for (int l = 0; l < SCALE_LOADS; ++l) {   // rows of A, then of B, one a lane
            const int row = l * 64 + lane;
            scales_from[l] = row < MB * 16 ? min((uint32_t)row, last_m) * (uint32_t)s.ldas : min((uint32_t)min(row - MB * 16, NB * 16 - 1), last_n) * (uint32_t)s.ldbs;
        }
        auto bring = [&](int i, int slot) {
            const int kb = wave + i * NW;
            gbl_char *const at_a = (gbl_char*)(a + (int64_t)kb * F8_BLOCK), *const at_b = (gbl_char*)(b + (int64_t)kb * F8_BLOCK);
            const uint32_t to = __builtin_amdgcn_readfirstlane(ring_at + (uint32_t)slot * STAGE);
            static_for<2 * BLOCKS>([&](auto l) {
                gbl_char* const src = uniform(l() < 2 * MB ? at_a : at_b);
                const uint32_t off = from[l()], into = to;
                asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(src), "s"(into), "n"(l() * 1024) : "memory", "m0", "scc");
            });
            static_for<SCALE_LOADS>([&](auto l) {
                const uint8_t* const src = (l() * 64 + lane < MB * 16 ? as : bs) + (kb & ~3) + scales_from[l()];
                const uint32_t into = to;
                asm volatile("s_add_u32 m0, %1, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(into), "n"(BLOCKS * 2048 + l() * 256) : "memory", "m0", "scc");
            });
        };
        const int at = r * F8_BLOCK + ((g ^ (r >> 1)) << 4);
        auto frag = [&](const char* stage, int block) {
            return Frag{*reinterpret_cast<const u32x4*>(stage + block * 2048 + at), *reinterpret_cast<const u32x4*>(stage + block * 2048 + (at ^ 64))};
        };
        for (int i = 0; i < DEPTH - 1; ++i)
            if (i < mine) bring(i, i);
        int slot = 0;
        for (int i = 0; i < mine; ++i) {
            const int into = slot == 0 ? DEPTH - 1 : slot - 1;   // what was multiplied last
            if (i + DEPTH - 1 < mine) {
                bring(i + DEPTH - 1, into);
                __builtin_amdgcn_s_waitcnt(vmcnt_only((DEPTH - 1) * LOADS));
            } else {
                __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
            }
            asm volatile("" ::: "memory");
            const char* const stage = ring + slot * STAGE;
            const int shift = ((wave + i * NW) & 3) * 8;
            const uint32_t* const scale = reinterpret_cast<const uint32_t*>(stage + BLOCKS * 2048) + r;
            Operand<BT, EXACT> ob[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) ob[j] = Operand<BT, EXACT>(frag(stage, MB + j), scale[(MB + j) * 16] >> shift);
#pragma unroll
            for (int m = 0; m < MB; ++m) {
                const Operand<AT, EXACT> oa(frag(stage, m), scale[m * 16] >> shift);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    acc[m][j] = multiply<BT, AT>(ob[j], oa, acc[m][j]);
                    asm volatile("" : "+v"(acc[m][j]));   // in its place, ahead of the loads into this slot
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            slot = slot == DEPTH - 1 ? 0 : slot + 1;
        }
    } else {
        struct Block {
            Frag a[MB], b[NB];
            uint32_t as[MB], bs[NB];
        };
        auto work = [&](const Block& o) {
            Operand<BT, EXACT> ob[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) ob[j] = Operand<BT, EXACT>(o.b[j], o.bs[j]);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                const Operand<AT, EXACT> oa(o.a[i], o.as[i]);
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = multiply<BT, AT>(ob[j], oa, acc[i][j]);
            }
        };
        constexpr int U = std::max(1, (150 - MB * NB * 4) / (18 * BLOCKS));   // twice U blocks' registers next to the sums
        auto load = [&](Block (&o)[U], int first) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (first + u < mine) {
                    const int kb = wave + (first + u) * NW;
                    const int64_t at = (int64_t)kb * F8_BLOCK;
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        o[u].b[j] = load_frag(b + at + b_row[j]);
                        o[u].bs[j] = (bs + kb)[bs_row[j]];
                    }
#pragma unroll
                    for (int i = 0; i < MB; ++i) {
                        o[u].a[i] = load_frag(a + at + a_row[i]);
                        o[u].as[i] = (as + kb)[as_row[i]];
                    }
                }
        };
        auto multiply_all = [&](const Block (&o)[U], int first) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (first + u < mine) work(o[u]);
        };
        Block even[U], odd[U];
        load(even, 0);
        for (int first = 0; first < mine; first += 2 * U) {
            load(odd, first + U);
            multiply_all(even, first);
            load(even, first + 2 * U);
            multiply_all(odd, first + U);
        }
    }
    if (whole * F8_BLOCK < s.kk && wave == whole % NW) {   // the block that the reduction ends in
        uint32_t sa[MB], sb[NB];
#pragma unroll
        for (int i = 0; i < MB; ++i) sa[i] = (as + whole)[as_row[i]];
#pragma unroll
        for (int j = 0; j < NB; ++j) sb[j] = (bs + whole)[bs_row[j]];
        const int64_t at = (int64_t)whole * F8_BLOCK;
        multiply_cut_block<AT, BT, EXACT>(a + at, a_row, sa, b + at, b_row, sb, s.kk - (int)at - g * 16, (int)at + g * 16, acc);
    }
    if constexpr (RING) __syncthreads();   // the rings are free
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) sums[(wave * MB * NB + i * NB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int q = wave; q < MB * NB; q += NW) {
        f32x4 v = sums[q * 64 + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += sums[(w * MB * NB + q) * 64 + lane];
        store_row<F32, GELU, 4>(s, m0 + q / NB * 16 + r, (int)n0 + q % NB * 16 + g * 4, false, {v});
    }
}

// Tiles of WM MI 16 rows by WN NJ 16 columns, one persistent workgroup a compute unit (or two of the smaller tile) that walks over its share of
// the (shard, tile) list; a wave has MI 16 rows by NJ 16 columns.  A step is a block of 128 of the reduction: one instruction deep, one cache line
// of a row.
//
// Two stages in LDS, and two barriers a step, so that parts of a stage are free for the stage after next as soon as they have been read: B and the
// first half of every wave's row blocks behind the first barrier, the other half behind the second.  Loads go straight into LDS and have a
// step and a half to arrive (with one barrier and a step the loads alone took 467 us of the 515 of 8192 x 4096 x 16384).  The row blocks before a
// barrier are multiplied behind it, underneath the reads of the next fragments.
//
// Bound by the matrix pipe: 8192 x 4096 x 16384 on eight devices, bf16 results, 456 .. 464 us, 2.4 PFLOP/s (the
// instruction alone, on random operands, 4.1), and by LDS, which is busy for as many cycles (192 KB read and 64 KB written a step at 128 bytes, against
// 64 instructions of 32 on every SIMD).  fp32 results by the widening next to the products, once for every wave that reads a fragment:
// the larger tile has four waves of 128 x 128, one a SIMD with all its 512 registers, and half the conversions of the smaller one (8192 x 4096 x 16384
// 1005 -> 848 us, 4096 cubed 140 -> 112); bf16 results are better off with eight of 128 x 64, two a SIMD (505 with four, 479 with eight, both at an
// earlier stage of the rest).
//
// DIRECT: rows at pitches of 16 bytes, and of scales at pitches of 4, go straight into LDS; else through registers, what lies at their end byte by byte.
template <int AT, int BT, bool F32, bool GELU, int WM, int WN, int MI, int NJ, bool DIRECT>
__global__ __launch_bounds__(WM * WN * 64, NJ == 8 ? 1 : 2) void gemm_f8_tile_kernel(GemmF8Plan p, int tm, int tn, int order, int tiles) {
    constexpr bool EXACT = F32;
    constexpr int NT = WM * WN * 64, BM = WM * MI * 16, BN = WN * NJ * 16;
    using StA = StageF8<BM, NT, false>;
    using StB = StageF8<BN, NT, !F32>;
    constexpr int STAGE = StA::BYTES + StB::BYTES;
    constexpr int SCALE_ROWS = (BM + BN) / NT;   // of a thread
    static_assert((BM + BN) % NT == 0, "rows of scales divide over the workgroup");
    // chunk i of a thread lies in rows NT / 8 i + 0..; C of them are half a wave's rows, so that every other C chunks of A are first halves
    constexpr int C = MI * 64 / NT;
    static_assert(C * NT == MI * 64 && StA::PER == 2 * WM * C, "an operand's chunks fall into halves of the waves' rows");
    // scales of 16 blocks of the reduction, twice: four planes of [row] dwords, four blocks each
    constexpr int SCALE_PLANE = (BM + BN) * 4, SCALE_BYTES = 4 * SCALE_PLANE;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE + 2 * SCALE_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wm = wave / WN, wn = wave % WN;

    // the tiles of this workgroup that exist, in order
    struct At {
        int id, g, m0, n0, steps;
    };
    auto settle = [&](int id) {   // the first tile of the walk from id on that lies in its shard; id >= tiles: none
        At t{id, 0, 0, 0, 0};
        for (; t.id < tiles; t.id += (int)gridDim.x) {
            const TileCoord c = map_tile(t.id, tiles, tm, tn, p.groups, order);
            if (!c.valid) continue;
            const GemmF8Shard& s = p.s[c.g];
            if ((int64_t)c.tile_m * BM >= s.m || (int64_t)c.tile_n * BN >= s.n) continue;
            t.g = c.g;
            t.m0 = c.tile_m * BM;
            t.n0 = c.tile_n * BN;
            t.steps = (s.kk + F8_BLOCK - 1) / F8_BLOCK;
            break;
        }
        return t;
    };
    At now = settle(blockIdx.x);
    if (now.id >= tiles) return;

    // ---- loads of stages: a cursor that runs two steps ahead of the multiplication, and stays at the last stage of all (whose loads are then
    // repeated into a stage that nobody reads: the waits can count on them)
    constexpr int LOADS = StA::PER + StB::PER;   // instructions of a wave and stage
    constexpr int DEPTH = MI >= 8 ? 2 : 1;       // rows of products ahead of which a fragment of A is read: one is short where the other wave waits
    At ahead = now;
    int ahead_left;   // reduction elements from the cursor's stage to the end
    uint32_t off_a[StA::PER], off_b[StB::PER];
    gbl_char *src_a, *src_b;
    // A stage that the reduction ends in: StageF8::less() (cut_* clears what lies behind the end).  A thread's chunks of an operand lie at one place in
    // their rows.
    uint32_t less_a, less_b;
    auto shorten = [&]() {
        less_a = DIRECT ? StA::less((int)threadIdx.x, ahead_left) : 0u;
        less_b = DIRECT ? StB::less((int)threadIdx.x, ahead_left) : 0u;
    };
    auto enter = [&]() {
        const GemmF8Shard& s = p.s[ahead.g];
        ahead_left = s.kk;
        src_a = (gbl_char*)(s.a + (int64_t)ahead.m0 * s.lda);
        src_b = (gbl_char*)(s.b + (int64_t)ahead.n0 * s.ldb);
#pragma unroll
        for (int i = 0; i < StA::PER; ++i) off_a[i] = StA::offset(i * NT + (int)threadIdx.x, s.m - ahead.m0, s.lda);
#pragma unroll
        for (int i = 0; i < StB::PER; ++i) off_b[i] = StB::offset(i * NT + (int)threadIdx.x, s.n - ahead.n0, s.ldb);
        shorten();
    };
    enter();
    auto advance = [&]() {
        if (ahead_left > F8_BLOCK) {
            src_a += F8_BLOCK;
            src_b += F8_BLOCK;
            ahead_left -= F8_BLOCK;
            if (ahead_left < F8_BLOCK) shorten();
        } else {
            const At t = settle(ahead.id + (int)gridDim.x);
            if (t.id < tiles) {
                ahead = t;
                enter();
            }
        }
    };
    // one chunk of a thread into the stage whose bytes for this wave start at `at` (uniform)
    auto bring = [&](gbl_char* src, uint32_t off, uint32_t at, auto behind) {
        asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(uniform(src)), "s"(at), "n"(behind()) : "memory", "m0", "scc");
    };
    auto bring_a = [&](uint32_t at, auto i) { bring(src_a, off_a[i()] - less_a, at, std::integral_constant<int, i() * NT * 16>{}); };
    auto bring_b = [&](uint32_t at, auto i) { bring(src_b, off_b[i()] - less_b, at, std::integral_constant<int, StA::BYTES + i() * NT * 16>{}); };
    const uint32_t lds_wave = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds + (uint32_t)wave * 1024u);
    u32x4 held[DIRECT ? 1 : LOADS];   // not DIRECT: a stage on its way
    auto hold = [&]() {
        if constexpr (!DIRECT) {
            const int ahead_done = p.s[ahead.g].kk - ahead_left;
            int at = StA::chunk_of((int)threadIdx.x) * 16;
#pragma unroll
            for (int i = 0; i < StA::PER; ++i) held[i] = load_some((const uint8_t*)src_a + off_a[i], ahead_left - at, ahead_done + at);
            at = StB::chunk_of((int)threadIdx.x) * 16;
#pragma unroll
            for (int i = 0; i < StB::PER; ++i) held[StA::PER + i] = load_some((const uint8_t*)src_b + off_b[i], ahead_left - at, ahead_done + at);
        }
    };
    // B and the first halves of A, then the second halves
    constexpr int FIRST = StB::PER + WM * C, SECOND = WM * C;
    auto bring_first = [&](uint32_t at, auto n) {
        if constexpr (n() < StB::PER) bring_b(at, n);
        else bring_a(at, std::integral_constant<int, (n() - StB::PER) / C * 2 * C + (n() - StB::PER) % C>{});
    };
    auto bring_second = [&](uint32_t at, auto n) { bring_a(at, std::integral_constant<int, n() / C * 2 * C + C + n() % C>{}); };
    auto put_held = [&](char* stage) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < StA::PER; ++i) *reinterpret_cast<u32x4*>(stage + (i * NT + threadIdx.x) * 16) = held[i];
#pragma unroll
            for (int i = 0; i < StB::PER; ++i) *reinterpret_cast<u32x4*>(stage + StA::BYTES + (i * NT + threadIdx.x) * 16) = held[StA::PER + i];
        }
    };
    // what this thread brought of a stage that the reduction ends in, `left` elements from its start: the bytes behind are cleared in LDS
    auto cut = [&](char* at, int valid) {
        u32x4 v = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const int n = valid - d * 4;
            v[d] &= n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
        }
        *reinterpret_cast<u32x4*>(at) = v;
    };
    auto cut_first = [&](char* stage, int left) {
        if (!DIRECT || left >= F8_BLOCK) return;
#pragma unroll
        for (int i = 0; i < StB::PER; ++i) cut(stage + StA::BYTES + (i * NT + threadIdx.x) * 16, left - StB::chunk_of(i * NT + (int)threadIdx.x) * 16);
#pragma unroll
        for (int i = 0; i < StA::PER; ++i)
            if (i / C % 2 == 0) cut(stage + (i * NT + threadIdx.x) * 16, left - StA::chunk_of(i * NT + (int)threadIdx.x) * 16);
    };
    auto cut_second = [&](char* stage, int left) {
        if (!DIRECT || left >= F8_BLOCK) return;
#pragma unroll
        for (int i = 0; i < StA::PER; ++i)
            if (i / C % 2 == 1) cut(stage + (i * NT + threadIdx.x) * 16, left - StA::chunk_of(i * NT + (int)threadIdx.x) * 16);
    };

    // ---- scales, 16 blocks of a row at a time
    constexpr int LOADS_SCALES = 4 * SCALE_ROWS;
    auto load_scales = [&](const At t, int step, char* to) {
        const GemmF8Shard& s = p.s[t.g];
#pragma unroll
        for (int i = 0; i < SCALE_ROWS; ++i) {
            const int row = i * NT + (int)threadIdx.x;
            const bool of_a = i * NT + wave * 64 < BM;   // whole waves: BM is a multiple of 64
            const int first = of_a ? t.m0 : t.n0 - BM, last = (of_a ? s.m : s.n) - 1, pitch = of_a ? s.ldas : s.ldbs;
            const uint8_t* const from = (of_a ? s.a_scales : s.b_scales) + (int64_t)min(first + row, last) * pitch;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                char* const plane = to + d * SCALE_PLANE + (i * NT + wave * 64) * 4;
                if constexpr (DIRECT) {
                    // four blocks from the row's last four on are those again (a row ends with them, its pitch being whole dwords)
                    const int b = min(step + 4 * d, (t.steps - 1) & ~3);
                    const uint32_t lds_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)plane);
                    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(from + b), "s"(lds_at) : "memory", "m0");
                } else {
                    uint32_t v = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (step + 4 * d + e < t.steps) v |= (uint32_t)from[step + 4 * d + e] << (8 * e);
                    *reinterpret_cast<uint32_t*>(plane + lane * 4) = v;
                }
            }
        }
    };
    char* const scale_lds = lds + 2 * STAGE;

    // ---- fragments
    const int a_row = wm * MI * 16 + r, b_row = wn * NJ * 16 + StB::fragment_row(r);
    const int a_lo = a_row * F8_BLOCK + ((g ^ StA::key(a_row)) << 4), b_lo = StA::BYTES + b_row * F8_BLOCK + ((g ^ StB::key(b_row)) << 4);
    auto frag_a = [&](const char* stage, int i) {
        return Frag{*reinterpret_cast<const u32x4*>(stage + a_lo + i * 16 * F8_BLOCK), *reinterpret_cast<const u32x4*>(stage + (a_lo ^ 64) + i * 16 * F8_BLOCK)};
    };
    auto frag_b = [&](const char* stage, int j) {
        return Frag{*reinterpret_cast<const u32x4*>(stage + b_lo + StB::fragment(j)), *reinterpret_cast<const u32x4*>(stage + (b_lo ^ 64) + StB::fragment(j))};
    };

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Loads are dealt out over a step's rows of products, one or two in the middle of each: all at once behind a barrier they hold every wave of
    // the workgroup up, and the matrix pipe with them (8192 x 4096 x 16384: 591 us).  The second halves of the stage ahead go with the
    // rows before the first barrier, the first loads of the one after with the others.
    constexpr int ROWS_SECOND = MI / 2 - DEPTH, ROWS_FIRST = MI - ROWS_SECOND;
    // Waits.  Loads and stores share one in-order counter; the number is how many of the youngest may be on their way.  At the first barrier: all that
    // was brought since the second halves of this stage; at the second: since the first part of the next one.  `stores`: waits that a whole
    // tile's stores may be younger than what is waited for.
    constexpr int BEFORE_SECOND_BARRIER = (ROWS_FIRST - 2) * FIRST / ROWS_FIRST;   // first loads that go with rows before it
    constexpr int NSTORE = MI * (F32 ? NJ : NJ / 2);
    int stores = 0;
    auto wait = [&](auto youngest, bool scales_too, bool scales_now) {
        if constexpr (!DIRECT) return;   // registers wait for themselves
        if (scales_now) __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
        else if (stores > 0) __builtin_amdgcn_s_waitcnt(vmcnt_only(std::min(63, youngest() + NSTORE)));
        else if (scales_too) __builtin_amdgcn_s_waitcnt(vmcnt_only(youngest() + LOADS_SCALES));
        else __builtin_amdgcn_s_waitcnt(vmcnt_only(youngest()));
        if (stores > 0) --stores;
        asm volatile("" ::: "memory");   // nothing that loads wrote into LDS is read ahead of this
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // what this wave read and wrote in LDS
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    load_scales(now, 0, scale_lds);
    const int left0 = ahead_left;
    if constexpr (DIRECT) {
        static_for<FIRST>([&](auto n) { bring_first(lds_wave, n); });
        static_for<SECOND>([&](auto n) { bring_second(lds_wave, n); });
        advance();
        static_for<FIRST>([&](auto n) { bring_first(lds_wave + STAGE, n); });
    } else {
        hold();
        put_held(lds);
        advance();
        hold();
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
    asm volatile("" ::: "memory");
    cut_first(lds, left0);
    barrier();

    int cur = 0, scale_cur = 0;
    uint32_t sa[MI], sb[NJ];
    auto read_scales = [&](int plane) {
        const char* const from = scale_lds + scale_cur * SCALE_BYTES + plane * SCALE_PLANE;
#pragma unroll
        for (int i = 0; i < MI; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(from + (a_row + i * 16) * 4);
#pragma unroll
        for (int j = 0; j < NJ; ++j) sb[j] = *reinterpret_cast<const uint32_t*>(from + (BM + b_row) * 4 + StB::fragment(j) / F8_BLOCK * 4);
    };
    read_scales(0);
    Frag fb[NJ], fa[DEPTH + 1];
#pragma unroll
    for (int j = 0; j < NJ; ++j) fb[j] = frag_b(lds, j);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) fa[i] = frag_a(lds, i);
    while (true) {
        const GemmF8Shard& s = p.s[now.g];
        const At next = settle(now.id + (int)gridDim.x);
        const int kk_next = next.id < tiles ? p.s[next.g].kk : F8_BLOCK;
        int left = s.kk;
        for (int k = 0; k < now.steps; ++k, left -= F8_BLOCK) {
            char* const stage = lds + cur * STAGE;
            char* const other = lds + (cur ^ 1) * STAGE;
            const uint32_t at = __builtin_amdgcn_readfirstlane(lds_wave + (uint32_t)cur * STAGE);
            const int in_chunk = k & 15, last_of_chunk = min(15, now.steps - 1 - (k - in_chunk));
            // the next 16 blocks' scales (or the next tile's; this one's again where there is none, which the waits count on) at the chunk's second
            // step, its first where there is one only
            const bool more = in_chunk == min(1, last_of_chunk);
            if (more) {
                const int to = k - in_chunk + 16;
                const bool here = to < now.steps || next.id >= tiles;
                load_scales(At{0, here ? now.g : next.g, here ? now.m0 : next.m0, here ? now.n0 : next.n0, here ? now.steps : next.steps}, to < now.steps ? to : 0, scale_lds + (scale_cur ^ 1) * SCALE_BYTES);
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): what was read at the end of the last step, so that the reads below are not waited for
            Operand<BT, EXACT> ob[NJ];
#pragma unroll
            for (int j = 0; j < NJ; ++j) ob[j] = Operand<BT, EXACT>(fb[j], sb[j]);
            auto product = [&](const Operand<AT, EXACT>& oa, int i, int j) {
                acc[i][j] = multiply<BT, AT>(ob[j], oa, acc[i][j]);
                // in its place: products put off to behind a barrier, or reads brought forward, keep more fragments than there are registers
                // (256 of them fill the accumulation registers)
                if constexpr (NJ == 8) asm volatile("" : "+a"(acc[i][j]));
                else asm volatile("" : "+v"(acc[i][j]));
            };
            const uint32_t at_other = __builtin_amdgcn_readfirstlane(lds_wave + (uint32_t)(cur ^ 1) * STAGE);
            auto loads = [&](auto i) {
                if constexpr (!DIRECT) return;
                else if constexpr (i() < ROWS_SECOND) {
                    static_for<SECOND>([&](auto n) { if constexpr (n() * ROWS_SECOND / SECOND == i()) bring_second(at_other, n); });
                } else {
                    static_for<FIRST>([&](auto n) { if constexpr (n() >= (i() - ROWS_SECOND) * FIRST / ROWS_FIRST && n() < (i() - ROWS_SECOND + 1) * FIRST / ROWS_FIRST) bring_first(at, n); });
                }
            };
            auto row = [&](auto i) {
                const Operand<AT, EXACT> oa(fa[i() % (DEPTH + 1)], sa[i()]);
                static_for<NJ>([&](auto j) {
                    product(oa, i(), j());
                    if constexpr (j() == 1) loads(i);
                });
                __builtin_amdgcn_sched_barrier(0);
            };
            auto read_row = [&](int i) {   // before the row ahead of it is multiplied: it has those products to arrive
                fa[i % (DEPTH + 1)] = frag_a(stage, i);
                __builtin_amdgcn_sched_barrier(0);
            };
            static_for<ROWS_SECOND>([&](auto i) {
                read_row(i() + DEPTH);
                row(i);
            });
            advance();
            // B and the first halves have been read; the second halves are there
            wait(std::integral_constant<int, LOADS>{}, more, false);
            cut_second(stage, left);
            barrier();
            static_for<ROWS_FIRST - 2>([&](auto i) {
                read_row(i() + MI / 2);
                row(std::integral_constant<int, i() + ROWS_SECOND>{});
            });
            if constexpr (DEPTH == 1) read_row(MI - 1);
            // the second halves have been read; B and the first halves of the next stage are there
            wait(std::integral_constant<int, SECOND + BEFORE_SECOND_BARRIER>{}, more, more && in_chunk == last_of_chunk);
            put_held(other);
            cut_first(other, left > F8_BLOCK ? left - F8_BLOCK : kk_next);
            barrier();
            const Frag start = frag_a(other, 0);
            const Operand<AT, EXACT> o0(fa[(MI - 2) % (DEPTH + 1)], sa[MI - 2]), o1(fa[(MI - 1) % (DEPTH + 1)], sa[MI - 1]);
            static_for<NJ>([&](auto j) {
                product(o0, MI - 2, j());
                product(o1, MI - 1, j());
                if constexpr (j() == 1) loads(std::integral_constant<int, MI - 2>{});
                if constexpr (j() == 2) loads(std::integral_constant<int, MI - 1>{});
                fb[j()] = frag_b(other, j());
                __builtin_amdgcn_sched_barrier(0);
            });
            hold();
            fa[0] = start;
#pragma unroll
            for (int i = 1; i < DEPTH; ++i) fa[i] = frag_a(other, i);
            // the next step's scales: the next bytes of these, or the next four blocks'
            const bool chunk_ends = in_chunk == last_of_chunk;
            if (chunk_ends) scale_cur ^= 1;
            if (chunk_ends || (k & 3) == 3) {
                read_scales(chunk_ends ? 0 : (in_chunk + 1) >> 2);
            } else {
#pragma unroll
                for (int i = 0; i < MI; ++i) sa[i] >>= 8;
#pragma unroll
                for (int j = 0; j < NJ; ++j) sb[j] >>= 8;
            }
            cur ^= 1;
        }

        const bool inside = now.m0 + BM <= s.m && now.n0 + BN <= s.n;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t m = (int64_t)now.m0 + wm * MI * 16 + i * 16 + r;
            const int n = now.n0 + wn * NJ * 16;
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < NJ; ++j) store_row<F32, GELU, 4>(s, m, n + j * 16 + g * 4, inside, {acc[i][j]});
            } else {
#pragma unroll
                for (int j = 0; j < NJ; j += 2) store_row<F32, GELU, 8>(s, m, n + j * 16 + g * 8, inside, {acc[i][j], acc[i][j + 1]});
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (inside) stores = 2;
        now = next;
        if (now.id >= tiles) break;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));   // nothing may come into LDS that another workgroup has by then
}

}  // namespace

int32_t launch_gemm_f8(const GemmF8Plan& plan, hipStream_t stream) {
    int max_m = 0, max_n = 0;
    for (int g = 0; g < plan.groups; ++g) {
        max_m = std::max(max_m, plan.s[g].m);
        max_n = std::max(max_n, plan.s[g].n);
    }
    if (max_m == 0 || max_n == 0) return SBP_OK;
    for (int g = 0; g < plan.groups; ++g) {
        const GemmF8Shard& s = plan.s[g];
        if (s.lda > GEMM_F8_MAX_PITCH || s.ldb > GEMM_F8_MAX_PITCH || s.ldas > GEMM_F8_MAX_PITCH || s.ldbs > GEMM_F8_MAX_PITCH) return SBP_ERR_UNSUPPORTED;
    }
    const F8Choice c = choose_f8_tile(plan, compute_units());
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
            auto by_waves = [&](auto mb, auto nb) {
                const int tm = tiles_along(max_m, 16 * mb()), tn = tiles_along(max_n, 16 * nb());
                const int64_t all = ((int64_t)tm * tn * plan.groups + 7) & ~7ll;
                if (!grid_fits(all, 256)) {
                    st = SBP_ERR_UNSUPPORTED;
                    return;
                }
                auto go = [&](auto ring) {
                    hipLaunchKernelGGL((gemm_f8_wave_kernel<a(), b(), f32(), gelu(), mb(), nb(), ring()>), dim3((uint32_t)all), dim3(256), 0, stream, plan, tm, tn, 4);
                };
                if (c.aligned) go(std::true_type{});
                else go(std::false_type{});
            };
            auto tile = [&](auto wm, auto wn, auto mi, auto nj, auto direct) {
                constexpr int BM = wm() * mi() * 16, BN = wn() * nj() * 16;
                const int tm = tiles_along(max_m, BM), tn = tiles_along(max_n, BN);
                const int64_t tiles = (int64_t)tm * tn * plan.groups;
                if (tiles > INT32_MAX - 65536) {
                    st = SBP_ERR_UNSUPPORTED;
                    return;
                }
                const int64_t at_once = (int64_t)compute_units() * (BM > 128 ? 1 : 2), all = (tiles + 7) & ~7;
                hipLaunchKernelGGL((gemm_f8_tile_kernel<a(), b(), f32(), gelu(), wm(), wn(), mi(), nj(), direct()>), dim3((uint32_t)std::min(all, at_once)),
                                   dim3(wm() * wn() * 64), 0, stream, plan, tm, tn, tn > 8 ? 6 : 2, (int)all);
            };
            using std::integral_constant;
            const auto i2 = integral_constant<int, 2>{};
            const auto i4 = integral_constant<int, 4>{};
            const auto i8 = integral_constant<int, 8>{};
            const auto yes = std::true_type{};
            const auto no = std::false_type{};
            const auto i1 = integral_constant<int, 1>{};
            auto columns = [&](auto mb) {
                if (c.nb == 1) by_waves(mb, i1);
                else if (c.nb == 2) by_waves(mb, i2);
                else by_waves(mb, i4);
            };
            if (c.mb == 1) columns(i1);
            else if (c.mb == 2) columns(i2);
            else if (c.mb == 4) columns(i4);
            else if (!c.aligned) tile(i2, i2, i4, i4, no);
            else if (c.mb == 8) tile(i2, i2, i4, i4, yes);
            else if constexpr (f32()) tile(i2, i2, i8, i8, yes);
            else tile(i2, i4, i8, i4, yes);
        });
    });
    return st != SBP_OK ? st : launch_status(__func__);
}

}  // namespace sbp
