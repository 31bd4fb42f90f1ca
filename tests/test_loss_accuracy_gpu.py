"""Accuracy of softmax cross entropy and its gradients where the sizes of its parts differ most, on both paths of the forward pass: a pass
over W (few rows, W stored by word) and tiles.  Against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import TYPES, close, half_step, workspace
from test_cross_entropy_gpu import IGNORED, Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("times,more,scale", [(5, 19, None), (7, 11, None), (5, 19, 3.0), (7, 11, 1000.0)])
def test_a_factor_of_all_rows_is_not_rounded_to_codes(words, dtype, times, more, scale):
    """What all rows share (1 / rows that count, the loss scale) reaches the gradients in 32 bits.  W = 0, so every probability is 1/64; every
    word is the target of `times` tokens, whose H is that word's unit vector, and `more` tokens with H = 0 make the count odd: the weight
    gradient is times g (1/64 - onehot), and only that is rounded."""
    n, t = 64, TYPES[dtype]
    p = Problem(times * n + more, n, n, dtype, words, bias=False, scale=0.0)
    p.h.zero_()
    p.h[:times * n] = torch.eye(n, device="cuda").repeat(times, 1)
    p.targets[:] = torch.arange(times * n + more, device="cuda") % n
    lse = p.forward()[1]
    dh, dw, db = p.backward(lse, None, scale)
    g = times * (1.0 if scale is None else scale) / p.rows
    want = torch.full((n, n), g / 64.0, device="cuda", dtype=torch.float64) - g * torch.eye(n, device="cuda", dtype=torch.float64)
    tol = want.abs() * 2.0 ** -21  # the factor's own roundings to 32 bits
    close(dw if words else dw.t(), want, tol + half_step(want.abs() + tol, t))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1e-37, 1e-20, 1.0, 1e30, 1e38])
def test_gradients_of_losses_of_any_size(size, dtype):
    """The largest |dloss| is scaled to 2^13 on the way, whatever it is; the loss scale brings results back into the type's range."""
    p = Problem(200, 64, 500, dtype)
    scale = min(max(2.0 ** -10 / size, 2.0 ** -100), 2.0 ** 100)
    dloss = torch.full((200,), size, device="cuda") * torch.linspace(0.25, 1.0, 200, device="cuda")
    p.check_backward(dloss, scale)


@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("rows", [5, 300])
def test_repeated(rows, words):
    """The same bits every time, whatever the workspace holds."""
    p = Problem(rows, 136, 3001, "f16", words, ignored=0.2)
    H, W = p.matrices()
    kind = qf.make_cross_entropy(p.t, IGNORED)
    first = None
    for fill in (0, 0xFF, 0x7C, 0x7F, 0):
        loss, lse = torch.empty(2, rows, device="cuda").unbind(0)
        mean, dh, dw, db = torch.empty(1, device="cuda"), torch.empty_like(p.h), torch.empty_like(p.w), torch.empty(p.vocab, device="cuda")
        ws = workspace(max(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, k) for k in (False, True))).fill_(fill)
        qf.qfmt_linear_cross_entropy(H, W, kind, p.bias, p.targets, loss, lse, mean, ws, ws.numel())
        ws.fill_(fill)
        qf.qfmt_linear_cross_entropy_backward(H, W, kind, p.bias, p.targets, lse, None, None, dh, dh.stride(0), dw, dw.stride(0), db, ws, ws.numel())
        now = (loss, lse, mean, dh, dw, db)
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))
