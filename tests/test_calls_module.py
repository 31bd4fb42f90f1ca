"""The C module of the Python side may be an older one than the library (no GPU needed)."""
import subprocess
import sys

import pytest

from paper_2103_15940_b200 import build as qbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    qbuild.build()


@pytest.mark.parametrize("module", ["bind=lambda *a: None", "bind=lambda *a: None, bind_step=lambda a, b: None", "nothing=0"])
def test_other_calls_work_with_an_older_module(module):
    """Its functions are fewer, or take other arguments: the calls that go through it say so, and all others work."""
    code = f"""
import sys, types
import paper_2103_15940_b200 as qf
sys.modules["paper_2103_15940_b200._calls"] = qf._calls = types.SimpleNamespace({module})
assert qf.qfmt_version() >= 100
try:
    qf.qfmt_quantize_stats(None, None, 4, qf.make_format(6, 9), stream=0)
except qf.QfmtError as e:
    assert e.status == qf.QFMT_ERR_BAD_ARG
else:
    raise AssertionError
for call in (lambda: qf.qfmt_dropout(None, 0, None, 0, None, 0, 0, 0, 0, qf.make_dropout(0.1, 1), stream=0),
             lambda: qf.qfmt_grad_clip(None, 0, 0, None, stream=0)):
    try:
        call()
    except ImportError as e:
        assert "_calls.abi3.so" in str(e) and "other sources" in str(e)
    else:
        raise AssertionError
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=qbuild.ROOT)
