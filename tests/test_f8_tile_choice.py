"""Which kernel a product of 8-bit tensors runs on, asked of the function that the launch asks: the sizes of the GPU tests reach the tiles that they are there for,
so that a change of the choice cannot quietly move them to another.  Runs on the host."""
import os
import subprocess

import pytest

import oracle as orc
from paper_2110_15032_amd import build
from test_gpu_block8 import F8_TILES, f8_pitches

PROGRAM = r"""
#include <cstdio>
#include "gemm_f8_choice.h"
using namespace sbp;
int main() {   // lines of: groups, result type, then for each group m n k and the pitches of its values and scales
    GemmF8Plan p{};
    while (scanf("%d %d", &p.groups, &p.out_dtype) == 2) {
        for (int g = 0; g < p.groups; ++g) {
            GemmF8Shard& s = p.s[g];
            if (scanf("%d %d %d %d %d", &s.m, &s.n, &s.kk, &s.lda, &s.ldas) != 5) return 1;
            s.ldb = s.lda;
            s.ldbs = s.ldas;
        }
        const F8Choice c = choose_f8_tile(p, 256);
        printf("%d %d %d\n", c.mb, c.nb, (int)c.aligned);
    }
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc is not installed")
    at = tmp_path_factory.mktemp("choice")
    src, exe = at / "choice.hip", str(at / "choice")
    src.write_text(PROGRAM)
    subprocess.run([build.HIPCC, "--cuda-host-only", "-O1", "-std=c++17", "-w", "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), str(src), "-o", exe], check=True, capture_output=True)

    def ask(cases):
        """cases of (result, [(m, n, k, pitch, pitch of scales) of a device])"""
        text = "\n".join(f"{len(g)} {0 if yk == 'f32' else 1} " + " ".join(str(n) for s in g for n in s) for yk, g in cases)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(n) for n in line.split()) for line in out.splitlines()]
    return ask


def shards(M, K, N, k, sig, aligned):
    size = lambda n, split: [e - b for b, e in (orc.split_range(n, k, i) for i in range(k))] if split else [n] * k  # noqa: E731
    ks = size(K, sig == "P")
    return [(m, n, kk, *f8_pitches(max(ks), aligned)) for m, n, kk in zip(size(M, sig == "S0"), size(N, sig == "S1"), ks)]


def test_sizes_of_the_tests_reach_their_tiles(choose):
    got = choose([(yk, shards(M, K, N, k, sig, aligned)) for M, K, N, k, sig, yk, aligned, _ in F8_TILES])
    assert got == [(tile, tile, int(aligned)) for *_, aligned, tile in F8_TILES]


def test_a_device_without_a_reduction_goes_to_the_tiles_of_waves(choose):
    big = (4096, 4096, 512, 512, 4)
    assert choose([("f32", [big])])[0][0] >= 8
    assert choose([("f32", [big, (4096, 4096, 0, 512, 4)])])[0][0] <= 4


def test_one_row_off_its_alignment_is_not_aligned(choose):
    row = (64, 64, 512, 512, 4)
    assert [c[2] for c in choose([("bf16", [row]), ("bf16", [row, (64, 64, 512, 520, 4)]), ("bf16", [row, (64, 64, 512, 512, 6)])])] == [1, 0, 0]
