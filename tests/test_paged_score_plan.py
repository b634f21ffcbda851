"""CPU check of how the score kernel for many rows fills its LDS, on the code itself."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_08450_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "paged_score_plan.h"
int main() {
    for (int dim = 64; dim <= 128; dim += 64)
        for (int heads = 1; heads <= 128; ++heads) {
            const int window = paged::rows_of_window(dim, heads);
            int most = 0;
            for (int rows = 1; rows <= window; ++rows)
                if (paged::products_of(rows, heads) > most) most = paged::products_of(rows, heads);
            printf("%d %d %d %d %d %d\n", dim, heads, window, most, paged::window_of(dim), paged::product_heads(heads));
        }
}
"""


def test_a_window_of_rows_fits_the_lds(tmp_path):
    """Every head count that a call takes: the product rows that a window stages, the
    rows' places and lengths, and the products' longest rows stay inside their arrays."""
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    lines = [[int(x) for x in ln.split()] for ln in subprocess.run([exe], capture_output=True, text=True,
                                                                   check=True).stdout.splitlines()]
    assert len(lines) == 256
    bad = [(dim, heads, window, 32 * products, held) for dim, heads, window, products, held, hp in lines
           if window < 1 or 32 * products > held or window > held // hp]
    assert not bad, bad
