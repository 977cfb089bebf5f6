// Stages of gemm_f8_tile_kernel: ROWS rows of a block of 128 of the reduction in LDS, and where they come from.
#pragma once
#include "sbp_internal.h"

namespace sbp {
namespace {

// LDS image of an operand: rows of 128 bytes, 16-byte chunk c of a row at c ^ key(row), so that the 16 lanes of a read's pass fall on
// different banks: row / 2 where a fragment is 16 consecutive rows, as A's are, and B's for fp32 results.  For bf16 results (PAIRS) B's fragments
// are taken in pairs, rows 8 i + 0..3 of 32 and rows 8 i + 4..7, so that a lane ends with eight consecutive columns of a row, and four lanes
// store 64 consecutive bytes either way; the key is the place in the fragment over 2.
template <int ROWS, int NT, bool PAIRS>
struct StageF8 {
    static constexpr int PER = ROWS * 8 / NT;   // chunks of a thread
    static constexpr int BYTES = ROWS * F8_BLOCK;
    __host__ __device__ static int key(int row) { return PAIRS ? ((row >> 3) & 3) << 1 | ((row >> 1) & 1) : (row >> 1) & 7; }
    // row of place r in fragment j, and the byte offset of fragment j from fragment 0
    __host__ __device__ static int fragment_row(int r) { return PAIRS ? (r >> 2) * 8 + (r & 3) : r; }
    static constexpr int fragment(int j) { return (PAIRS ? (j >> 1) * 32 + (j & 1) * 4 : j * 16) * F8_BLOCK; }
    __host__ __device__ static int row_of(int p) { return p >> 3; }
    __host__ __device__ static int chunk_of(int p) { return (p & 7) ^ key(p >> 3); }
    // byte offset of chunk position p from the tile's first row; rows past the operand's end are its last one
    __host__ __device__ static uint32_t offset(int p, int rows_left, int pitch) {
        const int row = row_of(p) < rows_left ? row_of(p) : rows_left - 1;
        return (uint32_t)row * (uint32_t)pitch + (uint32_t)chunk_of(p) * 16u;
    }
    // How far in front of its place a chunk is read in a stage with `left` elements up to the reduction's end: one that starts behind the end is read
    // from the last one that does not.  That one is read whole, up to 15 bytes behind the row's last value: rows start on multiples of 16 bytes, so
    // that these share 16 aligned bytes with the value.
    __host__ __device__ static uint32_t less(int p, int left) {
        const int last = (left < F8_BLOCK ? left - 1 : F8_BLOCK - 1) >> 4;
        return chunk_of(p) > last ? (uint32_t)(chunk_of(p) - last) * 16u : 0u;
    }
};

}  // namespace
}  // namespace sbp
