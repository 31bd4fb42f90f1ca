"""Offsets beyond 2^31 elements: products with an epilogue, passes over a gradient, the loss and lists of gradients."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import act64, close, half_step, slope64, sum_bound, workspace

pytestmark = pytest.mark.gpu
T = torch.bfloat16


def test_product_and_pass_over_its_gradient():
    m, n, k = 600011, 4096, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = (torch.randn(*s, generator=gen, device="cuda", dtype=T) for s in ((m, k), (n, k)))
    A, B = qf.make_matrix(x), qf.make_matrix(w, True)
    ws = workspace(max(qf.qfmt_linear_act_workspace_bytes(A, B), qf.qfmt_act_backward_workspace_bytes(m, n)))
    y, z = (torch.empty(m, n, device="cuda", dtype=T) for _ in range(2))
    qf.qfmt_linear_act(A, B, qf.make_epilogue(qf.QFMT_ACT_GELU, None, None, 0, z), y, n, T, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
    rows = torch.tensor([0, 255, 524287, 524288, 600000, m - 1], device="cuda")  # either side of 2^31 elements
    a64 = x[rows].double()
    z64, bound = a64 @ w.double().t(), sum_bound(a64, w.double().t(), k)
    close(z[rows], z64, bound + half_step(z64.abs() + bound, T))
    y64 = act64("gelu", z64)
    close(y[rows], y64, 1.13 * bound + y64.abs() * 2.0 ** -18 + half_step(y64.abs() + bound, T))
    db = torch.empty(n, device="cuda")
    dz = torch.empty_like(y)
    qf.qfmt_act_backward(y, n, z, n, dz, n, db, m, n, T, qf.QFMT_ACT_GELU, ws, ws.numel())
    g64 = y[rows].double()
    want = g64 * slope64("gelu", z[rows].double())
    close(dz[rows], want, g64.abs() * 2.0 ** -18 + half_step(want, T))
    cols = [0, 4095]
    for c in cols:
        terms = y[:, c].double() * slope64("gelu", z[:, c].double())
        # rows of a warp, warps and parts one after the other: at most m / 148 / 8 + 40 additions of one sum
        assert abs(float(db[c]) - float(terms.sum())) <= float(terms.abs().sum()) * ((m / 148 / 8 + 40) * 2.0 ** -24 + 2.0 ** -18)


def test_loss_of_more_logits():
    rows, hidden, vocab = 40000, 64, 70001
    gen = torch.Generator(device="cuda").manual_seed(2)
    h, w = (torch.randn(*s, generator=gen, device="cuda", dtype=T) for s in ((rows, hidden), (vocab, hidden)))
    w.mul_(0.25)
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    targets[::5] = -100
    H, W = qf.make_matrix(h), qf.make_matrix(w, True)
    ws = workspace(max(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, k) for k in (False, True)))
    loss, lse = torch.empty(2, rows, device="cuda").unbind(0)
    mean, dh, dw, db = torch.empty(1, device="cuda"), torch.empty_like(h), torch.empty_like(w), torch.empty(vocab, device="cuda")
    kind = qf.make_cross_entropy(T)
    qf.qfmt_linear_cross_entropy(H, W, kind, None, targets, loss, lse, mean, ws, ws.numel())
    qf.qfmt_linear_cross_entropy_backward(H, W, kind, None, targets, lse, None, None, dh, hidden, dw, hidden, db, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
    at = torch.tensor([1, 19999, 30678, 39998], device="cuda")
    assert bool((targets[at] >= 0).all())
    logits = h[at].double() @ w.double().t()
    want = torch.logsumexp(logits, dim=1)
    close(lse[at], want, want.abs() * 2.0 ** -20 + 2.0 ** -17)
    count = int((targets >= 0).sum())
    d = torch.exp(logits - want[:, None])
    d[torch.arange(len(at), device="cuda"), targets[at]] -= 1.0
    d64 = d @ w.double() / count
    # terms rounded to codes (half a step each, errors in sums of squares), the sum over the vocabulary, the result's rounding
    bound = (d.abs() @ w.double().abs()) / count * (2.0 ** -8 + (vocab / 16 + 64) * 2.0 ** -23) + half_step(d64, T)
    close(dh[at], d64, bound)
    assert not dh[::5].any() and not loss[::5].any()
    assert abs(float(db.double().sum())) <= 1e-3  # probabilities and targets both sum to one
    words = dw.double().sum(dim=0)
    assert bool(torch.isfinite(words).all())


def test_a_tensor_of_more_elements():
    n = (1 << 31) + 12345
    t = torch.ones(n, device="cuda", dtype=T)
    t[-1] = 3.0
    host = qf.make_tensors([t], [t])
    chunks = qf.qfmt_plan_tensors(host, 1)
    records, ws = torch.frombuffer(host, dtype=torch.uint8).cuda(), workspace(qf.qfmt_grad_norm_workspace_bytes(1, chunks))
    record = torch.zeros(2, dtype=torch.int64, device="cuda")
    want = (n + 8.0) ** 0.5
    qf.qfmt_grad_norm(records, 1, chunks, want / 2.0, None, record, None, ws, ws.numel())
    qf.qfmt_grad_clip(records, 1, chunks, record)
    assert abs(float(record.view(torch.float32)[0]) - want) <= want * 2.0 ** -22
    assert float(t[0]) == 0.5 == float(t[-2]) == float(t[1 << 31]) and float(t[-1]) == 1.5
