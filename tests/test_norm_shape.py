"""The launch arithmetic of the norms' backward pass over all row lengths, compiled from its header, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Every row length, 1 .. 11 arrays, one and three sums, 16 and 32 bytes per thread and array in bf16 (whole vectors; the two around
# shifted ones, which are copied ahead in clusters alone), 32 in fp32, from one row to many.
CODE = r"""
#include <cstdio>
#include "sifar_norm_shape.cuh"
using namespace sifar;
int main()
{
    const size_t many[] = {1, 100, 149, 1000, 5000, 100000, (size_t)1 << 30};
    size_t bad = 0, three = 0;
    for (int dtype = 0; dtype < 2; ++dtype)
        for (size_t cols = 1; cols <= (size_t)SIFAR_NORM_MAX_COLS; ++cols)
            for (size_t rows : many) {
                const GradShape s = grad_shape(dtype, rows, cols);
                const unsigned threads = s.row.tx * s.ry, items = 8;
                const size_t ctas = (s.blocks + s.ry - 1) / s.ry * s.row.parts;
                bool ok = threads <= (unsigned)kMaxRowThreads && threads * s.per_sm <= (unsigned)kMaxRowThreads && s.blocks >= 1 && s.blocks <= rows;
                ok = ok && (size_t)s.row.tx * s.row.parts * items >= cols && s.row.parts <= kMaxNormCluster && ctas <= (size_t)kSms * s.per_sm;
                ok = ok && (s.row.parts == 1 || s.per_sm == 1) && (s.ry == 1 || s.row.tx == 32);
                for (unsigned arrays = 1; arrays <= 11; ++arrays)
                    for (int sums = 1; sums <= 3; sums += 2)
                        for (size_t bytes = dtype == SIFAR_BF16 ? 16 : 32; bytes <= (s.row.parts > 1 || dtype == SIFAR_F32 ? 32u : 16u); bytes += 16) {
                            const size_t row = threads * arrays * bytes, stages = grad_stages(s, rows, row, sums), smem = row * stages;
                            const size_t cta = (smem + row_sum_bytes(sums) + kCtaReserved + 127) / 128 * 128;
                            /* all CTAs of an SM at once; a block may ask for 227 KB */
                            ok = ok && stages >= 1 && stages <= kMaxStages && cta * s.per_sm <= (size_t)228 * 1024;
                            ok = ok && smem <= ring_room(1, sums) && ring_room(1, sums) + row_sum_bytes(sums) <= (size_t)227 * 1024;
                            three += stages == 3;
                        }
                if (!ok && ++bad <= 5)
                    printf("dtype %d rows %zu cols %zu: %u threads x %u, %u CTAs per SM, %u blocks\n", dtype, rows, cols, s.row.tx, s.ry, s.per_sm, s.blocks);
            }
    printf("%zu bad, %zu of three stages\n", bad, three);
    return bad != 0;
}
"""


def test_every_cta_that_the_rows_are_cut_for_has_room(tmp_path):
    src, exe = tmp_path / "shape.cpp", tmp_path / "shape"
    src.write_text(CODE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2607_08973_b200", "csrc"), "-o", str(exe), str(src)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert got.returncode == 0, got.stdout
