"""Where gemm_split_kernel reads its fp32 operand, asked of the functions that the kernel asks: every 16-byte read of a 32-deep
stage lies inside the stored operand, for rows that end in the middle of a 32-byte chunk too.  Runs on the host."""
import os
import subprocess

import pytest

from paper_2110_15032_amd import build

PROGRAM = r"""
#include <cstdio>
#include "gemm_device.h"
using namespace sbp;
template <int R, int NT>
int check() {   // reduction-major storage: 32 rows of `limit` floats, `ld` apart, the last one not padded
    using T = Tile<R, false, NT, 32, true>;
    int bad = 0;
    for (int limit = 8; limit <= 2 * R + 12; limit += 4)
        for (int ld = limit; ld <= limit + 8; ld += 4)
            for (int first = 0; first < limit; first += R)
                for (int tid = 0; tid < NT; ++tid)
                    for (int it = 0; it < T::PER_THREAD; ++it) {
                        const uint64_t off = 2ull * T::src_offset(ld, first, limit, it * NT + tid), size = 4ull * (31ull * ld + limit);
                        const uint64_t second = off + T::second_half(first, limit, tid);
                        bad += off % 16 || off + 16 > size || second + 16 > size;
                        // the values that count: column c of the chunk comes from float c
                        const int krow = (it * NT + tid) / T::CPR, col = (int)(off / 4 - (uint64_t)krow * ld);
                        if (col + 8 <= limit && second != off + 16) ++bad;
                    }
    return bad;
}
int main() {
    const int bad = check<128, 256>() + check<128, 512>();
    printf("%d\n", bad);
    return bad != 0;
}
"""


def test_the_split_kernel_reads_inside_its_fp32_operand(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc is not installed")
    src, exe = tmp_path / "bounds.hip", str(tmp_path / "bounds")
    src.write_text(PROGRAM)
    subprocess.run([build.HIPCC, "--cuda-host-only", "-O1", "-std=c++17", "-w", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(src), "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, f"{r.stdout.strip()} reads outside the operand or of the wrong values"


STAGES = r"""
#include <cstdio>
#include "gemm_f8_stage.h"
using namespace sbp;
template <int ROWS, int NT, bool PAIRS>
int check() {   // an operand of `rows` rows of `k` values, `pitch` apart, the last one not padded
    using T = StageF8<ROWS, NT, PAIRS>;
    int bad = 0;
    for (int rows : {1, 2, 15, 16, ROWS - 1, ROWS, ROWS + 1, 2 * ROWS, 2 * ROWS + 5})
        for (int k = 1; k <= 400; ++k)
            for (int pitch = (k + 15) / 16 * 16; pitch <= (k + 15) / 16 * 16 + 16; pitch += 16)
                for (int first = 0; first < rows; first += ROWS)
                    for (int k0 = 0; k0 < k; k0 += F8_BLOCK)
                        for (int tid = 0; tid < NT; ++tid)
                            for (int i = 0; i < T::PER; ++i) {
                                const int p = i * NT + tid, row = first + T::row_of(p) < rows ? first + T::row_of(p) : rows - 1;
                                if (T::chunk_of(p) != T::chunk_of(tid)) ++bad;   // one less() for all of a thread's chunks
                                const int64_t at = (int64_t)first * pitch + k0 + T::offset(p, rows - first, pitch) - T::less(tid, k - k0);
                                const int64_t row_at = (int64_t)row * pitch, size = (int64_t)(rows - 1) * pitch + k;
                                // a multiple of 16 inside the row, which begins before the row's end: what lies behind that is in the same 16 bytes
                                bad += at % 16 != 0 || at < row_at + k0 || at >= row_at + k || at >= size || at + 16 > (size + 15) / 16 * 16;
                                // a chunk with values of the row comes from its place
                                const int64_t place = row_at + k0 + T::chunk_of(p) * 16;
                                if (place < row_at + k && at != place) ++bad;
                            }
    return bad;
}
int main() {
    const int bad = check<128, 256, false>() + check<128, 256, true>() + check<256, 256, false>() + check<256, 512, false>() + check<256, 512, true>();
    printf("%d\n", bad);
    return bad != 0;
}
"""


def test_stages_of_8_bit_operands_read_the_16_bytes_that_a_row_ends_in_and_no_more(tmp_path):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc is not installed")
    src, exe = tmp_path / "stages.hip", str(tmp_path / "stages")
    src.write_text(STAGES)
    subprocess.run([build.HIPCC, "--cuda-host-only", "-O2", "-std=c++17", "-w", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(src), "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, f"{r.stdout.strip()} reads that lie elsewhere"
