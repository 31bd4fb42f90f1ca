"""Index arithmetic of the sub-layer kernels, run on the host: small programs compiled from the kernels' own headers (no GPU
needed)."""
import os
import subprocess

import pytest

from paper_2103_15940_b200 import build as qbuild


def run(tmp_path, body):
    """Compiles `body` against the kernels' headers and returns the lines that it prints."""
    src, exe = tmp_path / "host.cu", tmp_path / "host"
    src.write_text("#include <cstdio>\n#include <cstdint>\n" + body)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.check_call([nvcc, "-O1", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static", "-I", os.path.join(qbuild.ROOT, "include"),
                           "-I", qbuild.CSRC, "-o", str(exe), str(src)])
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()


@pytest.fixture(scope="module")
def joined(tmp_path_factory):
    """The first and last places of [dweight, dbias] of several widths, as the kernel that joins the parts maps them."""
    out = run(tmp_path_factory.mktemp("joined"), r"""
#include "norm.cuh"
int main() {
    const int64_t widths[] = {1, 8, 1000, 16385, (1ll << 30) - 8, 1ll << 30, (1ll << 30) + 1, (1ll << 30) + 8, (1ll << 31) - 8, (1ll << 31) - 7, (1ll << 31) - 1};
    for (int64_t cols : widths) {
        const int64_t padded = (cols + 7) / 8 * 8;
        for (int64_t i : {(int64_t)0, cols - 1, padded - 1, padded, padded + cols - 1, 2 * padded - 1}) {
            const qfmt::JoinedColumn at = qfmt::joined_column(i, padded);
            std::printf("%lld %lld %d %lld\n", (long long)cols, (long long)i, (int)at.second, (long long)at.c);
        }
    }
}
""")
    return [[int(v) for v in line.split()] for line in out]


def test_joined_columns(joined):
    assert len(joined) == 66
    for cols, i, second, c in joined:
        padded = -(-cols // 8) * 8
        assert (second, c) == divmod(i, padded), (cols, i)


def test_pieces_of_ragged_rows_stay_inside_the_matrix(tmp_path):
    """Every aligned 16-byte piece that a granule is loaded in, for small matrices of every alignment and spacing of rows; inner
    rows of eight columns and more are always loaded in pieces."""
    out = run(tmp_path, r"""
#include "elements.cuh"
int main() {
    long pieces = 0, outside = 0, by_element = 0;
    for (int per : {4, 8})  // elements of a piece: containers, codes
        for (int off = 0; off < per; ++off)
            for (int rows = 1; rows <= 9; ++rows)
                for (int cols = 1; cols <= 41; ++cols)
                    for (int ld = cols; ld <= cols + 9; ++ld)
                        for (int row = 0; row < rows; ++row)
                            for (int g = 0; g * 8 < cols; ++g) {
                                const int n = cols - 8 * g < 8 ? cols - 8 * g : 8, at = off + row * ld + 8 * g, first = at % per;
                                if (!qfmt::pieces_inside(qfmt::at_edge(cols, g), row, qfmt::inner_rows(cols, rows))) {
                                    by_element += cols >= 8 && row != 0 && row + 1 != rows;
                                    continue;
                                }
                                for (int i = 0; first + n > i * per; ++i) {
                                    const int begin = at - first + i * per;
                                    ++pieces;
                                    outside += begin < off || begin + per > off + (rows - 1) * ld + cols;
                                }
                            }
    std::printf("%ld %ld %ld\n", pieces, outside, by_element);
}
""")
    pieces, outside, by_element = (int(v) for v in out[0].split())
    assert pieces > 100000 and outside == 0 and by_element == 0
