"""The library and the C module of the sub-layer calls are built and loaded separately (no GPU needed)."""
import os
import subprocess
import sys

import pytest

from paper_2103_15940_b200 import build as qbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    qbuild.build()


@pytest.fixture
def module_elsewhere(tmp_path, monkeypatch):
    """The module's file is missing, at a path of the test's own."""
    path = tmp_path / "_calls.abi3.so"
    monkeypatch.setattr(qbuild, "CALLS", str(path))
    return path


def test_a_missing_module_is_built_without_the_library(module_elsewhere, monkeypatch):
    monkeypatch.setenv("NVCC", "/nonexistent/nvcc")
    before = os.path.getmtime(qbuild.LIB)
    assert qbuild.build() == qbuild.LIB and module_elsewhere.exists()
    assert os.path.getmtime(qbuild.LIB) == before and not qbuild.needs_build()


def test_the_library_is_built_where_the_module_cannot_be(module_elsewhere, tmp_path, monkeypatch):
    """A compiler without the interpreter's headers: the library is there when the error is raised."""
    nvcc = tmp_path / "nvcc"
    nvcc.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\necho built > "$2"\n')
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.setenv("CC", "false")
    monkeypatch.setattr(qbuild, "LIB", str(tmp_path / "libqfmt.so"))
    with pytest.raises(subprocess.CalledProcessError):
        qbuild.build()
    assert (tmp_path / "libqfmt.so").read_text() == "built\n" and not module_elsewhere.exists()
    assert qbuild.needs_build()


def test_other_calls_work_without_the_module():
    """A process that cannot load the module makes every call but the sub-layer ones, which name what is missing and why."""
    code = """
import sys
sys.modules["paper_2103_15940_b200._calls"] = None
import paper_2103_15940_b200 as qf
assert qf.qfmt_version() >= 100
try:
    qf.qfmt_quantize_stats(None, None, 4, qf.make_format(6, 9), stream=0)
except qf.QfmtError as e:
    assert e.status == qf.QFMT_ERR_BAD_ARG
else:
    raise AssertionError
for call in (lambda: qf.qfmt_dropout(None, 0, None, 0, None, 0, 0, 0, 0, qf.make_dropout(0.1, 1), stream=0),
             lambda: qf.qfmt_layer_norm(qf.make_norm(0, 0, 0), None, None, None, None, stream=0)):
    try:
        call()
    except ImportError as e:
        assert "_calls.abi3.so" in str(e) and isinstance(e.__cause__, ImportError)
    else:
        raise AssertionError
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=qbuild.ROOT)
