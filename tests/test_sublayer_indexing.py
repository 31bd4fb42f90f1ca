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
