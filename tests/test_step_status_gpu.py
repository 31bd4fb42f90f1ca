"""A workspace that several calls share keeps what its status area reports until a call that reports there itself."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import workspace

pytestmark = pytest.mark.gpu


def timed_out(ws):
    """A wait that runs out, as a product would report it at the head of its workspace."""
    trace = torch.zeros(4, dtype=torch.int32, device="cuda")
    qf.qfmt_selftest_bounded_wait(ws, 20000, trace)
    assert qf.qfmt_device_status(ws) == qf.QFMT_ERR_TIMEOUT


@pytest.mark.parametrize("n", [100, 1 << 20])
def test_norm_and_clipping(n):
    g = torch.ones(n, device="cuda")
    host = qf.make_tensors([g], [g])
    chunks = qf.qfmt_plan_tensors(host, 1)
    records, record = torch.frombuffer(host, dtype=torch.uint8).cuda(), torch.zeros(2, dtype=torch.int64, device="cuda")
    ws = workspace(qf.qfmt_grad_norm_workspace_bytes(1, chunks))
    timed_out(ws)
    qf.qfmt_grad_norm(records, 1, chunks, 1.0, None, record, None, ws, ws.numel())
    qf.qfmt_grad_clip(records, 1, chunks, record)
    assert qf.qfmt_device_status(ws) == qf.QFMT_ERR_TIMEOUT
    assert float(record.view(torch.float32)[0]) == pytest.approx(n ** 0.5, rel=2.0 ** -21)


@pytest.mark.parametrize("shape", [(3, 8), (4099, 520)])
def test_pass_over_a_gradient(shape):
    rows, cols = shape
    dy, db = torch.ones(rows, cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = workspace(qf.qfmt_act_backward_workspace_bytes(rows, cols))
    timed_out(ws)
    qf.qfmt_act_backward(dy, cols, None, 0, None, 0, db, rows, cols, torch.float32, qf.QFMT_ACT_NONE, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_ERR_TIMEOUT
    assert bool((db == float(rows)).all())


@pytest.mark.parametrize("shape", [(3, 8), (4099, 520), (700, 20000)])
def test_layer_norm_backward(shape):
    rows, cols = shape
    x, dy = torch.randn(rows, cols, device="cuda"), torch.ones(rows, cols, device="cuda")
    mean, rstd, y = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dx, dw, db = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    norm = qf.make_norm(rows, cols, qf.QFMT_F32)
    qf.qfmt_layer_norm(norm, x, None, None, y, mean, rstd)
    ws = workspace(qf.qfmt_layer_norm_workspace_bytes(norm))
    timed_out(ws)
    qf.qfmt_layer_norm_backward(norm, dy, x, mean, rstd, None, dx, dw, db, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_ERR_TIMEOUT
    assert bool((db == float(rows)).all())


def test_a_call_that_reports_there_starts_anew():
    a, b = (torch.ones(s, device="cuda", dtype=torch.bfloat16) for s in ((8, 16), (16, 24)))
    A, B, y = qf.make_matrix(a), qf.make_matrix(b), torch.empty(8, 24, device="cuda", dtype=torch.bfloat16)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    timed_out(ws)
    qf.qfmt_linear_act(A, B, qf.make_epilogue(), y, 24, torch.bfloat16, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK and bool((y == 16.0).all())
