"""Where the binding takes the current stream from (no GPU needed: torch's functions are replaced in a process of their own)."""
import subprocess
import sys

from paper_2103_15940_b200 import build as qbuild

FAKES = """
import os, types
import torch
import paper_2103_15940_b200 as qf
asked = []
def current_stream():
    asked.append(1)
    if os.getpid() != parent:
        raise RuntimeError("not in a forked process")
    return types.SimpleNamespace(cuda_stream=70)
parent = os.getpid()
torch.cuda.current_stream = current_stream
"""
RAW = """
torch._C._cuda_getDevice = lambda: 3
torch._C._cuda_getCurrentRawStream = lambda device: 100 + device
"""


def run(code):
    subprocess.run([sys.executable, "-c", code], check=True, cwd=qbuild.ROOT, timeout=300)


def test_torch_is_initialised_by_the_first_call():
    run(FAKES + RAW + """
assert [qf._stream_handle(None) for _ in range(3)] == [70, 103, 103] and len(asked) == 1
assert qf._stream_handle(5) == 5 and qf._stream_handle(types.SimpleNamespace(cuda_stream=6)) == 6
""")


def test_a_forked_process_asks_torch_again():
    run(FAKES + RAW + """
qf._stream_handle(None)
child = os.fork()
if child == 0:
    try:
        qf._stream_handle(None)
    except RuntimeError as e:
        os._exit(7 if "forked" in str(e) else 1)
    os._exit(2)
assert os.waitstatus_to_exitcode(os.waitpid(child, 0)[1]) == 7
assert qf._stream_handle(None) == 103
""")


def test_without_the_raw_handle_torch_is_asked_every_time():
    run(FAKES + """
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
assert [qf._stream_handle(None) for _ in range(3)] == [70, 70, 70] and len(asked) == 3
""")
