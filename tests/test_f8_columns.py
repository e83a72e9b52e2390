"""Where the gradient's kernel loads pieces of a row of dY from, without a GPU: the arithmetic that the kernel runs (csrc/pieces.h) in a
host program, for widths from one column on and every tile.  Every load lies in its row, and every column that is stored was taken from its own
place."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1609_07228_amd", "csrc")

PROGRAM = r"""
#include "pieces.h"
#include <cstdint>
#include <cstdio>
#include <initializer_list>
template <class Y> static int check(int n, int across, int (*from)(int, int))
{
    typedef Y Eight __attribute__((ext_vector_type(8)));
    const bool pieces_whole = n % 8 == 0;
    for (int j0 = 0; j0 < n; j0 += across)
        for (int at = j0; at < j0 + across; at += 8) {
            const bool inside = pieces_whole || j0 + across <= n;      // whole pieces, without a look at where rows end
            Eight x;
            for (int k = 0; k < 8; ++k) {
                const int64_t column = inside || n >= 8 ? (int64_t)(uint32_t)from(at, n) + k : piece_column(k, n);
                if (column < 0 || column >= n) return 1;               // read outside the row
                x[k] = (Y)column;
            }
            if (!inside) x = moved_down<Y>(x, piece_moved(at, n));
            for (int k = 0; k < 8 && at + k < n; ++k)
                if ((int64_t)x[k] != at + k) return 2;                 // another column's value
        }
    return 0;
}
// a mistake: in the tile that the row ends in, columns counted from the tile's first one
static int from_the_tile(int at, int n) { return at / 128 * 128 + 128 <= n ? at : n - 8 - at / 128 * 128; }
int main()
{
    for (int across : {64, 128, 256}) {
        for (int n = 1; n <= 1200; ++n)
            if (int bad = check<uint16_t>(n, across, piece_from) | check<uint32_t>(n, across, piece_from)) return printf("%d columns, tiles of %d: %d\n", n, across, bad), 1;
        for (int n = 65536 - 300; n <= 65536; ++n)
            if (int bad = check<uint32_t>(n, across, piece_from)) return printf("%d columns, tiles of %d: %d\n", n, across, bad), 1;
    }
    if (check<uint16_t>(130, 128, from_the_tile) != 1) return printf("the mistake is not seen\n"), 1;
    printf("all in their rows\n");
    return 0;
}
"""


def test_every_piece_lies_in_its_row_and_in_its_place(tmp_path):
    compiler = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    source, program = tmp_path / "columns.cpp", tmp_path / "columns"
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-x", "c++", "-std=c++17", "-O1", "-w", "-I", CSRC, "-o", str(program), str(source)], check=True)
    done = subprocess.run([str(program)], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0 and "all in their rows" in done.stdout, done.stdout


def test_the_tiles_are_the_kernels():
    """Columns of dY that the kernel's tiles take: 32 times two of the launches' numbers."""
    text = open(os.path.join(CSRC, "f8.hip")).read()
    tiles = {32 * int(fy) * int(wy) for fy, _, wy, _ in re.findall(r"launch_gradient<Y, F, (\d), (\d), (\d), (\d),", text)}
    assert tiles == {64, 128, 256}


@pytest.mark.parametrize("name", ["piece_from(", "piece_moved(", "piece_column(", "moved_down<Y>("])
def test_the_kernel_runs_this_arithmetic(name):
    assert name in open(os.path.join(CSRC, "f8.hip")).read()
