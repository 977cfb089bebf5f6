// Internal declarations shared by the translation units of libsbp_mi355x.so.
// Nothing here is part of the C ABI (that is include/sbp.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sbp.h"

namespace sbp {

// Balanced split (paper Sec. 3.1, "in a balanced manner"): floor(n/k) indices per shard,
// the first n mod k shards one more.  begin(k) == n.
__host__ __device__ inline int64_t split_begin(int64_t n, int32_t k, int32_t i) {
    const int64_t q = n / k, r = n % k;
    return (int64_t)i * q + (i < r ? i : r);
}
__host__ __device__ inline int64_t split_len(int64_t n, int32_t k, int32_t i) {
    return n / k + (i < n % k ? 1 : 0);
}

// Status of the launch just made; a failure is reported on stderr with HIP's own text (it means a
// launch configuration the device refused, never a data-dependent condition).
inline int32_t launch_status(const char* where) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return SBP_OK;
    fprintf(stderr, "libsbp_mi355x: kernel launch in %s failed: %s\n", where, hipGetErrorString(e));
    return SBP_ERR_LAUNCH;
}

// Tiles along an extent, which may be as large as 2^31 - 1.
inline int tiles_along(int extent, int tile) { return (int)(((int64_t)extent + tile - 1) / tile); }
// Can a grid of `blocks` workgroups of `threads` be launched?  HIP counts the work items of a grid dimension in 32 bits.
inline bool grid_fits(int64_t blocks, int threads) { return blocks <= 0xFFFFFFFFll / threads; }

// ---------------------------------------------------------------------------------------------
// Boxing: every conversion is a set of rectangle tasks.  Task t reads a rows x cols rectangle
// from n_src source shards (all at the same offset / leading dimension), combines them
// (copy when n_src == 1, sum or max in shard order otherwise) and writes the result to n_dst
// destination shards (all at the same offset / leading dimension).
// ---------------------------------------------------------------------------------------------
enum BoxOp : int32_t { BOX_COPY = 0, BOX_SUM = 1, BOX_MAX = 2 };

struct BoxPlan {
    const void* src[SBP_MAX_K];
    void* dst[SBP_MAX_K];
    int64_t rows, cols;       // global shape, in elements
    int32_t k;                // devices holding the input
    int32_t k_out;            // devices holding the output (= k on one device set; launch_boxing_cast ignores it)
    int32_t sbp_in, sbp_out;  // sbp_t values
    int32_t elem_bytes;       // 2 or 4
    // batch > 1: that many independent conversions of equal shape and signature in one launch (the groups of a
    // device grid): conversion b reads src[b * k + i] and writes dst[b * k_out + j]; batch * max(k, k_out) <=
    // SBP_MAX_K.  Only reductions (P input) take it; launch_boxing returns SBP_ERR_UNSUPPORTED, before anything is
    // enqueued, for any other conversion, and the caller then launches the conversions one by one.
    int32_t batch;
};

int32_t launch_boxing(const BoxPlan& plan, hipStream_t stream);
void set_box_reduce_variant(int32_t v);
// fp32 S(a) -> bf16 B (cast + all-gather) and bf16 P(sum) -> fp32 S(a) (cast + reduce-scatter); elem_bytes unused
int32_t launch_boxing_cast(const BoxPlan& plan, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// Grouped GEMM: shard g computes C_g[m, n] = sum_kk A_g[m, kk] * B_g[kk, n].
// a_kc: A is stored [m][kk] (kk contiguous, lda = row pitch) else [kk][m].
// b_kc: B is stored [n][kk] (kk contiguous) else [kk][n].      C is always [m][n], pitch ldc.
// ---------------------------------------------------------------------------------------------
struct GemmShard {
    const void* a;
    const void* b;
    void* c;
    float* rowmax;   // EPI_ROWMAX only: [m] fp32, max over this shard's columns of the stored results
    int32_t m, n, kk;
    int32_t lda, ldb, ldc;
};
// internal epilogue code next to the public SBP_EPI_*: store, and fold every stored row into rowmax
constexpr int32_t EPI_ROWMAX = 2;
// GeLU through erfcf (about 1e-7) where SBP_EPI_GELU is the fit of gelu_fast (2.2e-5): see launch_chosen
constexpr int32_t EPI_GELU_ERF = 3;
// Bias, activation, residual (sbp_linear): GemmBlockPlan in GemmPlan's place
constexpr int32_t EPI_BLOCK = 4;
struct GemmPlan {
    GemmShard s[SBP_MAX_K];
    int32_t groups;
    int32_t in_dtype;   // SBP_F32 | SBP_BF16
    int32_t f32_operand;  // 0: both operands have in_dtype; 1 / 2: A / B is an fp32 P(sum) partial next to a bf16 operand
    int32_t out_dtype;  // SBP_F32 | SBP_BF16
    int32_t a_kc, b_kc;
    int32_t epilogue;   // SBP_EPI_*
};

// C = act(A B + bias) + residual, pre = A B + bias.  A launch takes eight shards, as its argument block costs about a microsecond a KB.
struct GemmExtra {
    const void* bias;       // [n], null: none
    const void* residual;   // [m][n], null: none
    void* pre;              // [m][n], null: not wanted
    int32_t ldr, ldp;
};
constexpr int GEMM_BLOCK_SHARDS = 8;
enum GemmBlockFlags : int32_t { GB_BIAS_BF16 = 1, GB_RESIDUAL_BF16 = 2, GB_PRE_BF16 = 4, GB_OUT_BF16 = 8, GB_GELU = 16, GB_GELU_ERF = 32 };
struct GemmBlockPlan {
    GemmShard s[GEMM_BLOCK_SHARDS];
    GemmExtra x[GEMM_BLOCK_SHARDS];
    int32_t groups, in_dtype, a_kc, b_kc, flags;
};
int32_t launch_linear(const GemmBlockPlan& plan, hipStream_t stream);
constexpr int GEMV_ROWS = 4;
// gemv_kernels.hip: 1 .. GEMV_ROWS rows of x, stored along the reduction
int32_t launch_gemv(const GemmBlockPlan& plan, int max_m, int max_n, hipStream_t stream);
// 1 .. FEW_ROWS rows in bf16, both operands stored along the reduction
constexpr int FEW_ROWS = 32;
int32_t launch_gemm_few(const GemmBlockPlan& plan, int max_m, int max_n, hipStream_t stream);

// variant: SBP_KNOB_GEMM_VARIANT.  The launch_gemm_* functions below return SBP_ERR_UNSUPPORTED, with nothing enqueued, for a
// grid that cannot be launched (grid_fits).
int32_t launch_gemm(const GemmPlan& plan, int32_t variant, hipStream_t stream);
void set_tile_order(int32_t order);
// The ping-pong persistent kernel (gemm_pingpong_kernel.hip).  The caller has checked: bf16 operands, every
// local reduction length a multiple of 128, operand row pitches of 16 bytes.  order: tile walk (see map_tile).
int32_t launch_gemm_pingpong(const GemmPlan& plan, int max_m, int max_n, int order, hipStream_t stream);
// gemm_any_kernels.hip: bf16 operands, any reduction length, local operands below 4 GiB.  direct: rows of both operands
// 16-byte aligned, else any pitch (REG tiles always).
enum AnyTile : int32_t {
    WAVEK_32 = 0,   // 32 x 64, reduction-contiguous A only
    WAVEK_64,       // 64 x 64
    WAVEK_128,      // 128 x 64, direct only
    REG_128,        // 128 x 128
    REG_64,         // 64 x 64
    ROWS_32,        // 32 x 32, both operands reduction-contiguous, fp32 results
    ROWS_64         // 64 x 64, the same
};
int32_t launch_gemm_any(const GemmPlan& plan, int max_m, int max_n, int tile, bool direct, int order, hipStream_t stream);
int32_t launch_gemm_any(const GemmBlockPlan& plan, int max_m, int max_n, int tile, bool direct, int order, hipStream_t stream);   // not ROWS_*
// gemm_any_kernels.hip, 128 x 128 tile, any operand layout, rows 16-byte aligned, any reduction length
int32_t launch_gemm_deep(const GemmPlan& plan, int max_m, int max_n, int order, bool touch, hipStream_t stream);
int32_t launch_gemm_deep(const GemmBlockPlan& plan, int max_m, int max_n, int order, bool touch, hipStream_t stream);
// gemm_f32_kernels.hip: fp32 x fp32 (fp32 results, GeLU or no epilogue) and fp32 next to bf16 (f32_operand), any pitch and extent.
enum F32Tile : int32_t {
    F32_128 = 0,   // 128 x 128
    F32_64,        // 64 x 64
    F32_32,        // 32 x 32, waves splitting the reduction
    TERMS_128,     // 128 x 128 and 64 x 64 on the bf16 matrix instruction, fp32 operands as three bf16 terms
    TERMS_64
};
int32_t launch_gemm_f32(const GemmPlan& plan, int max_m, int max_n, int tile, int order, hipStream_t stream);
int32_t launch_gemm_f32(const GemmBlockPlan& plan, int max_m, int max_n, int tile, int order, hipStream_t stream);
// Compute units of the current device, asked of the runtime once per device and kept.
int compute_units();
// Diagnostic matrix-pipe loop (probe_kernels.hip); scratch: 1 MiB of device memory.
int32_t launch_probe_mfma(int32_t mode, int32_t iters, int32_t zero, void* scratch, hipStream_t stream);
// The same with the staging memory in a static device array of the library (modes 0-6); out: 1 MiB.
int32_t launch_probe_mfma_static(int32_t mode, int32_t iters, int32_t zero, void* out, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// Row statistics of the model-parallel softmax.
// ---------------------------------------------------------------------------------------------
struct RowStatPlan {
    const void* logits[SBP_MAX_K];
    const float* gmax[SBP_MAX_K];   // null for the max pass
    float* out[SBP_MAX_K];
    int32_t cols[SBP_MAX_K];        // local column count of every shard
    int32_t ld[SBP_MAX_K];          // row pitch of every shard, elements
    int64_t rows;
    int32_t k;
    int32_t dtype;
};
// Sparse cross entropy on S(1) logits.  Arrays sized for 32 shards keep the argument block small.
constexpr int XENT_MAX_K = 32;
struct XentPlan {
    const void* logits[XENT_MAX_K];
    const int32_t* labels[XENT_MAX_K];
    const float* gmax[XENT_MAX_K];
    const float* denom[XENT_MAX_K];
    const float* grad[XENT_MAX_K];   // backward only
    void* out[XENT_MAX_K];           // loss partials (f32) or dlogits (dtype)
    int32_t cols[XENT_MAX_K];        // local column count
    int32_t ld[XENT_MAX_K];          // row pitch of the logits, elements
    int32_t ld_out[XENT_MAX_K];      // row pitch of dlogits (backward only)
    int32_t begin[XENT_MAX_K];       // first global column of the shard
    int64_t rows;
    int32_t total_cols;
    int32_t k;
    int32_t dtype;
};
int32_t launch_xent_loss(const XentPlan& plan, hipStream_t stream);
int32_t launch_xent_grad(const XentPlan& plan, hipStream_t stream);

int32_t launch_row_stat(const RowStatPlan& plan, bool sumexp, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// 8-bit tensors: values and one power of two for every F8_BLOCK consecutive values of a stored row.
// ---------------------------------------------------------------------------------------------
constexpr int F8_BLOCK = 128;
constexpr int64_t f8_blocks(int64_t n) { return (n + F8_BLOCK - 1) / F8_BLOCK; }

// One shard of an elementwise pass over an 8-bit tensor.  rows and cols are the logical local shape; trans: the 8-bit tensor holds
// its transpose.
struct Block8Shard {
    const void* x;     // saving: the tensor to save; restoring: the 8-bit values; GeLU's gradient: the pre-activation
    void* scales;      // of the 8-bit tensor (written when saving)
    const void* dh;    // GeLU's gradient only
    void* out;
    int32_t rows, cols;
    int32_t ldx, lds, lddh, ldo;   // row pitches in elements
};
struct Block8Plan {
    Block8Shard s[SBP_MAX_K];
    int32_t k;
    int32_t f8;      // SBP_F8E4M3 | SBP_F8E5M2, or a 16- or 32-bit pre-activation's type
    int32_t dtype;   // of the other tensors
    int32_t trans;
    int32_t gelu;
    int32_t streams;   // of block8_device.h, chosen at the launch
};
int32_t launch_quantize(const Block8Plan& plan, hipStream_t stream);
int32_t launch_dequantize(const Block8Plan& plan, hipStream_t stream);
int32_t launch_gelu_grad(const Block8Plan& plan, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// Layer normalisation over rows.  Arrays sized for 32 shards keep the argument block small.
// ---------------------------------------------------------------------------------------------
constexpr int NORM_MAX_K = 32;
constexpr int NORM_MAX_COLS = 16384;   // a row stays in the registers of one workgroup
struct NormShard {
    const void* x;
    const void* gamma;   // null: ones
    const void* beta;    // null: zeros
    void* y;
    void* y_scales;
    float* mean;         // null: not wanted
    float* rstd;
    int32_t rows, ldx, ldy, lds;
};
struct NormPlan {
    NormShard s[NORM_MAX_K];
    int32_t k, cols;
    int32_t x_dtype, y_dtype, w_dtype;
    float eps;
    int32_t streams;
};
struct NormGradShard {
    const void* x;
    const void* x_scales;
    const void* gamma;
    const float* mean;
    const float* rstd;
    const void* dy;
    void* dx;
    float* dgamma;       // null: neither is wanted
    float* dbeta;
    float* part;         // [blocks][2][cols], where blocks > 1
    int32_t rows, ldx, lds, lddy, lddx, blocks;
};
struct NormGradPlan {
    NormGradShard s[NORM_MAX_K];
    int32_t k, cols;
    int32_t x_dtype, dy_dtype, w_dtype;
    int32_t streams;
};
// workgroups that launch_norm_grad gives a shard of so many rows, each of which leaves one partial sum of the weights' gradients
int32_t norm_grad_blocks(int64_t rows, int64_t cols, int32_t k);
int32_t launch_norm(const NormPlan& plan, hipStream_t stream);
int32_t launch_norm_grad(const NormGradPlan& plan, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// Grouped product of 8-bit tensors: C_g[m, n] = sum over kk of A_g[m, kk] * B_g[n, kk], both with the reduction index contiguous.
// ---------------------------------------------------------------------------------------------
constexpr int GEMM_F8_MAX_K = 32;
constexpr int GEMM_F8_MAX_PITCH = 1 << 23;   // 256 rows of a tile are counted in 32 bits
struct GemmF8Shard {
    const uint8_t* a;
    const uint8_t* a_scales;
    const uint8_t* b;
    const uint8_t* b_scales;
    void* c;
    int32_t m, n, kk;
    int32_t lda, ldas, ldb, ldbs, ldc;   // row pitches in elements
};
struct GemmF8Plan {
    GemmF8Shard s[GEMM_F8_MAX_K];
    int32_t groups;
    int32_t a_dtype, b_dtype, out_dtype;
    int32_t epilogue;   // SBP_EPI_*
};
int32_t launch_gemm_f8(const GemmF8Plan& plan, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// Lists of tensors: the sum of their squares, and all of them times a factor.
// ---------------------------------------------------------------------------------------------
// An argument block costs about a microsecond a KB, so a launch has one of about its own size: places for CAP local tensors, S devices.
constexpr int LIST_CHUNK = 1024;    // vectors of eight elements that a workgroup takes at a time, of one local tensor
constexpr int LIST_BLOCKS = 2048;   // most workgroups of a launch of the sum of squares: eight a compute unit, as many as it holds (clipping has one for every chunk)
constexpr int LIST_DENSE = 160, LIST_PITCHED = 80, LIST_SOME = 64, LIST_FEW = 16;   // CAP, at most 192
// A dense local tensor.  info: elements, from bit 48 on what of_list() says.
template <bool OUT>
struct DensePart {
    const void* in;
    uint64_t info;
};
template <>
struct DensePart<true> {
    const void* in;
    void* out;
    uint64_t info;
};
// Rows at a pitch.
template <bool OUT>
struct PitchedPart {
    const void* in;
    void* out;            // clipping only
    int32_t rows, cols, ldi, ldo, what;
};
// bit 0: in is bf16, bit 1: out is; from bit 2 on: the device, counted from the launch's first
constexpr int32_t of_list(bool in_bf16, bool out_bf16, int32_t device) { return (in_bf16 ? 1 : 0) | (out_bf16 ? 2 : 0) | device << 2; }
// Parts in the order of their devices.  Sums of squares: workgroup (x, d) takes the chunks of the launch's d-th device and leaves its sum at
// partial[(device * turns + turn) * gridDim.x + x], turn: first_turn for the launch's first device, other_turn else.
template <template <bool> class PART, int CAP>
struct SquarePlan {
    PART<false> s[CAP];
    double* partial;
    int32_t parts, first_device, turns, first_turn, other_turn;
    int32_t stream;   // past the caches
};
// The partial sums of device d, `blocks` of them a turn: those of dense[d] turns from turn d * turns on, and those of tensors with a pitch, of pitched[d] turns from `dense_turns` turns
// further on.  A device's turns: the launches that it has parts in.
template <int S>
struct SquareJoin {
    const double* partial;
    int32_t blocks, turns, dense_turns;
    int16_t dense[S], pitched[S];
    float* out[S];
};
template <template <bool> class PART, int CAP, int S>
struct ClipPlan {
    PART<true> s[CAP];
    const float* sum[S];
    float* norm[S];           // null: not wanted
    float most;
    int32_t parts, chunks, k, partial;   // partial: the sums are P(sum)
    int32_t first_device, stream;
};
template <template <bool> class PART, int CAP>
int32_t launch_square_sum(const SquarePlan<PART, CAP>& plan, int devices, int blocks, hipStream_t stream);
template <int S>
int32_t launch_square_join(const SquareJoin<S>& join, int32_t k, hipStream_t stream);
template <template <bool> class PART, int CAP, int S>
int32_t launch_clip(const ClipPlan<PART, CAP, S>& plan, hipStream_t stream);

// ---------------------------------------------------------------------------------------------
// The gradient of a block's epilogue: da = dy gelu'(pre), and the sum of da (or of dy) over the rows.
// ---------------------------------------------------------------------------------------------
constexpr int LINEAR_GRAD_SHARDS = 8;
struct LinearGradShard {
    const void* dy;
    const void* pre;      // null: no activation
    const void* scales;   // of pre, 8 bits only
    void* da;             // null: no activation
    float* dbias;
    float* part;          // [blocks][cols], where blocks > 1
    int32_t rows, cols, lddy, ldp, lds, ldda, blocks;
};
template <int S>
struct LinearGradPlan {
    LinearGradShard s[S];
    int32_t streams;      // of block8_device.h, chosen at the launch
};
template <int S>
int32_t launch_linear_grad(const LinearGradPlan<S>& plan, int n, int32_t dy, int32_t pre, bool gelu, hipStream_t stream);
// workgroups along the rows of a shard, each of which leaves a partial sum
int32_t linear_grad_blocks(int64_t rows, int64_t cols, int32_t k);

// ---------------------------------------------------------------------------------------------
// The norms behind and in front of a block, with its gate and the residual.  A launch takes S shards: the argument block costs about a
// microsecond a KB, so that a single device has a launch of its own size.
// ---------------------------------------------------------------------------------------------
constexpr int RESNORM_SHARDS = 8;
enum ResNormFlags : int32_t {
    RN_POST = 1, RN_POST_LAYER = 2, RN_PRE = 4, RN_PRE_LAYER = 8,   // which norms, and whether they take the mean off
    RN_DH = 16,                                                     // gradient: the residual stream's own
    RN_BF16_WEIGHTS = 32,
    RN_STREAM_H = 64, RN_STREAM_Y = 128                             // results past the caches (dr and dx in the gradient)
};
struct ResNormShard {
    const void* x;
    const void* r;
    void* h;
    void* y;             // pre only
    void* y_scales;
    float* mean1;        // null: not wanted
    float* rstd1;
    float* mean2;
    float* rstd2;
    const void* gate;    // null: ones
    const void* gamma1;
    const void* beta1;   // null: zeros
    const void* gamma2;
    const void* beta2;
    int32_t rows, ldx, ldr, ldh, ldy, lds;
};
template <int S>
struct ResNormPlan {
    ResNormShard s[S];
    int32_t cols, flags;
    float alpha, eps1, eps2;
};
struct ResNormGradShard {
    const void* x;
    const void* h;       // pre only
    const void* dh;      // RN_DH only
    const void* dy;      // pre only
    void* dx;
    void* dr;
    const float* mean1;
    const float* rstd1;
    const float* mean2;
    const float* rstd2;
    const void* gate;    // null: ones
    const void* gamma1;
    const void* gamma2;
    float* part;         // [blocks][4][cols], null: no weight's gradient is wanted
    int32_t rows, ldx, ldh, lddh, lddy, lddx, lddr, blocks;
};
template <int S>
struct ResNormGradPlan {
    ResNormGradShard s[S];
    int32_t cols, flags;
    float alpha;
};
struct ResNormJoinShard {
    const float* part;
    const void* gate;
    const void* gamma1;
    const void* beta1;
    float* dgate;        // null: not wanted
    float* dgamma1;
    float* dbeta1;
    float* dgamma2;
    float* dbeta2;
    int32_t blocks;
};
template <int S>
struct ResNormJoin {
    ResNormJoinShard s[S];
    int32_t cols, flags;
};
// types of x, of the residual stream and of y (its gradient); n shards, 1 .. S
template <int S>
int32_t launch_residual_norm(const ResNormPlan<S>& plan, int n, int32_t x, int32_t r, int32_t y, hipStream_t stream);
template <int S>
int32_t launch_residual_norm_grad(const ResNormGradPlan<S>& plan, int n, int32_t x, int32_t r, int32_t y, hipStream_t stream);
template <int S>
int32_t launch_residual_norm_join(const ResNormJoin<S>& join, int n, hipStream_t stream);
// workgroups that a shard of so many rows gets, each of which leaves one partial sum of the weights' gradients
int32_t residual_norm_grad_blocks(int64_t rows, int64_t cols, int32_t k);

}  // namespace sbp
