"""Accuracy of softmax cross entropy and its gradients where the sizes of its parts differ most, on both paths of the forward pass: a pass
over W (few rows, W stored by word) and tiles.  Against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import TYPES, close, half_step, operand, workspace
from test_cross_entropy_gpu import IGNORED, Problem

pytestmark = pytest.mark.gpu


def definition(p):
    """lse and loss of all rows in 64 bits; a row's largest logit taken out of both before they are subtracted."""
    logits = p.h.double() @ (p.w.t() if p.words else p.w).double() + p.bias.double()
    most = logits.amax(dim=1, keepdim=True)
    log = torch.log(torch.exp(logits - most).sum(dim=1))
    return most[:, 0] + log, (most[:, 0] - logits.gather(1, p.targets[:, None])[:, 0]) + log


@pytest.mark.parametrize("rows", [3, 8, 40, 130])
@pytest.mark.parametrize("level", [50.0, 1000.0, -3.0e4])
def test_a_loss_is_not_rounded_to_the_logits_steps(rows, level):
    """Logits far from zero whose differences are small: the loss is formed from differences.  With H = 0 the logits are the bias, exactly."""
    p = Problem(rows, 64, 300, "bf16", scale=0.0)
    p.bias.mul_(0.25).add_(level)
    p.targets[:] = torch.arange(rows, device="cuda") * 2
    p.bias[0] = level + 10.0  # of the first row's target: its loss is small
    loss, lse, mean = p.forward()
    lse64, loss64 = definition(p)
    assert float(loss64[0]) < 0.05 and float(loss64[1]) > 1.0
    # exponentials and their sum 2^-19 of the sum, whose logarithm has as large an absolute error; the logarithm's and the result's rounding
    close(loss, loss64, loss64 * 2.0 ** -22 + 2.0 ** -19)
    close(lse, lse64, 2.0 ** -19 + lse64.abs() * 2.0 ** -23)
    close(mean, loss64.mean().view(1), loss64.mean().view(1) * 2.0 ** -22 + 2.0 ** -19)


@pytest.mark.parametrize("rows", [3, 40])
def test_the_least_loss(rows):
    """A word with all but 10^-4 of the probability, logits around 50.  The sum of exponentials is near 1 and takes at most 16 additions on its
    way, half a step of 2^-23 each; a step of the logits' is 2^-18."""
    p = Problem(rows, 64, 295, "f16", scale=0.0)
    p.bias[:] = 35.0
    p.bias[7] = 50.0 + 2.0 ** -10
    p.targets[:] = 7
    loss = p.forward()[0]
    _, loss64 = definition(p)
    close(loss, loss64, loss64 * 2.0 ** -19 + 2.0 ** -20)


@pytest.mark.parametrize("rows", [2, 8, 9, 32, 100])
@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("hidden", [32768, 50000])
def test_logits_of_one_sign_over_a_long_contraction(rows, words, hidden):
    """Sums over D are closed after 8192 elements, wherever the product goes."""
    p = Problem(rows, 64, 40, "f16", words, scale=1.0)
    gen, t = p.gen, p.t
    p.hidden = hidden
    one = lambda *s: 0.5 + torch.rand(*s, generator=gen, device="cuda")
    p.h = operand(one(rows, hidden), t)
    w = one(40, hidden) * 2.0 ** -12
    p.w = operand(w if words else w.t(), t)
    loss, lse, _ = p.forward()
    logits = p.h.double() @ (p.w.t() if words else p.w).double() + p.bias.double()
    size = logits.abs().amax(dim=1)
    want = torch.logsumexp(logits, dim=1)
    tol = size * ((8192 / 16 + hidden / 16384 + 24) * 2.0 ** -23) + 2.0 ** -19 + want.abs() * 2.0 ** -22
    close(lse, want, tol)
    close(loss, want - logits.gather(1, p.targets[:, None])[:, 0], 2.0 * tol)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("words", [True, False])
def test_weight_gradients_of_one_sign_over_many_tokens(words, dtype):
    """Sums over tokens are closed after 8192: with W = 0 and 64 words every probability is 1/64, a code, so what the sums lose shows."""
    rows = 1 << 18
    p = Problem(rows, 40, 64, dtype, words, bias=False, scale=0.0)
    p.h = operand(0.5 + torch.rand(rows, 40, generator=p.gen, device="cuda"), p.t)
    p.targets[:] = 5
    lse = p.forward()[1]
    dh, dw, db = p.backward(lse, mean=False)
    d = torch.full((64,), 1.0 / 64.0, device="cuda", dtype=torch.float64)
    d[5] -= 1.0
    want = d[:, None] * p.h.double().sum(dim=0)[None]
    tol = want.abs() * ((8192 / 16 + rows / 16384 + 24) * 2.0 ** -23)
    tol = tol + half_step(want.abs() + tol, p.t)
    close(dw if words else dw.t(), want, tol)
    # column sums: the exponential 2^-21; 32 rows, then a 32nd of the parts one after the other, half a step each
    close(db, d * rows, (d * rows).abs() * (2.0 ** -21 + (rows / 1024 + 40) * 2.0 ** -24))
    assert not dh.any()  # W is zero


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
