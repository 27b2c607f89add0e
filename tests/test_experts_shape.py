"""The launch arithmetic of the experts' products for a few tokens, compiled from its header, without a GPU."""
import os
import subprocess

import pytest

from paper_2607_08973_b200 import binding as sf
from tests.test_experts import Moe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Two CTAs per SM exactly where what both take, with what the system keeps of each, is no more than an SM has.
CODE = r"""
#include <cstdio>
#include "sifar_experts_shape.cuh"
using namespace sifar;
template <int G> int check()
{
    int bad = 0;
    for (size_t rows = 0; rows <= kFewMostShared; rows += 64) {
        const size_t declared = 2 * 8 * 16 * 8 * G * sizeof(float) + SIFAR_ROUTE_MAX_EXPERTS * (4 + 4 + 2) + 8 * sizeof(int);
        const size_t cta = (declared + 127) / 128 * 128 + (rows + 127) / 128 * 128 + 1024;
        const unsigned fit = 228 * 1024 / cta, want = G > 2 || fit < 2 ? 1 : 2;
        bad += few_ctas<G>((rows + 127) / 128 * 128) != want || kFewStatic<G> + rows > 227 * 1024;
    }
    return bad;
}
int main()
{
    /* up to 8 tokens always two; of 16 not where their rows take most of what there is */
    printf("%d %u %u %u\n", check<1>() + check<2>() + check<4>(), few_ctas<1>(kFewShared), few_ctas<2>(16 * (1408 * 4 + 64)), few_ctas<2>(16 * (1280 * 4 + 64)));
}
"""


def test_as_many_ctas_as_an_sm_has_room_for(tmp_path):
    src, exe = tmp_path / "shape.cpp", tmp_path / "shape"
    src.write_text(CODE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2607_08973_b200", "csrc"),
                    "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split() == ["0", "2", "1", "2"]


@pytest.mark.gpu
@pytest.mark.parametrize("T,H", [(16, 1280), (16, 1376), (16, 1408), (13, 1440), (8, 2912)])
def test_results_on_both_sides(T, H):  # noqa: N803
    Moe(T, H, 40, 6, 2, dtype=sf.F32, seed=T + H).check()
