"""The backward passes of products and of the loss where offsets pass 2^31 elements, with values from either side."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import close, half_step, slope64, sum_bound, workspace

pytestmark = pytest.mark.gpu
T = torch.bfloat16


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=T)


def test_backward_product():
    """residual, z and dz beyond 2^31 elements, and the column sums over all rows."""
    m, n, k = 600011, 4096, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    dy, w, z, r = randn(gen, m, k), randn(gen, n, k), randn(gen, m, n), randn(gen, m, n)
    A, B = qf.make_matrix(dy), qf.make_matrix(w, True)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    dz, db = torch.empty_like(z), torch.empty(n, device="cuda")
    qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(qf.QFMT_ACT_SILU, None, r, 0, z), dz, n, db, T, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
    rows = torch.tensor([0, 255, 524287, 524288, 600000, m - 1], device="cuda")
    a64, b64 = dy[rows].double(), w.double().t()
    g64 = a64 @ b64 + r[rows].double()
    want = g64 * slope64("silu", z[rows].double())
    bound = (sum_bound(a64, b64, k) + g64.abs() * 2.0 ** -23) * 1.13 + g64.abs() * 2.0 ** -18
    close(dz[rows], want, bound + half_step(want.abs() + bound, T))
    for c in (0, 31, 2048, 4095):
        g64 = dy.double() @ w[c].double() + r[:, c].double()
        terms = g64 * slope64("silu", z[:, c].double())
        # the terms' own error, 32 rows, a 32nd of the parts one after the other
        size = (dy.double().abs() @ w[c].double().abs()) * (28 * 2.0 ** -23) + g64.abs() * 2.0 ** -18
        assert abs(float(db[c]) - float(terms.sum())) <= float(size.sum()) * 1.13 + float(terms.abs().sum()) * ((m / 1024 + 40) * 2.0 ** -24)


class Loss:
    def __init__(self, rows, hidden, vocab, seed, every=5):
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.hidden, self.vocab = rows, hidden, vocab
        self.h, self.w = randn(gen, rows, hidden), randn(gen, vocab, hidden)
        self.w.mul_(2.0 * hidden ** -0.5)
        self.targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        self.targets[::every] = -100
        H, W = qf.make_matrix(self.h), qf.make_matrix(self.w, True)
        ws = workspace(max(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, k) for k in (False, True)))
        self.loss, self.lse = torch.empty(2, rows, device="cuda").unbind(0)
        self.dh, self.dw, self.db = torch.empty_like(self.h), torch.empty_like(self.w), torch.empty(vocab, device="cuda")
        kind = qf.make_cross_entropy(T)
        qf.qfmt_linear_cross_entropy(H, W, kind, None, self.targets, self.loss, self.lse, None, ws, ws.numel())
        qf.qfmt_linear_cross_entropy_backward(H, W, kind, None, self.targets, self.lse, None, None, self.dh, hidden, self.dw, hidden, self.db, ws,
                                              ws.numel())
        assert qf.qfmt_device_status(ws) == qf.QFMT_OK
        self.at = (self.targets >= 0).nonzero()[:, 0]

    def check_rows(self, rows):
        """lse and dH of some rows."""
        assert bool((self.targets[rows] >= 0).all())
        logits = self.h[rows].double() @ self.w.double().t()
        want = torch.logsumexp(logits, dim=1)
        close(self.lse[rows], want, want.abs() * 2.0 ** -20 + 2.0 ** -17)
        d = torch.exp(logits - want[:, None])
        d[torch.arange(len(rows), device="cuda"), self.targets[rows]] -= 1.0
        d64 = d @ self.w.double() / len(self.at)
        # terms rounded to codes (half a step), the sum over the words, the logits' error; the result's rounding
        bound = (d.abs() @ self.w.double().abs()) / len(self.at) * (2.0 ** -8 + 2.0 ** -12)
        close(self.dh[rows], d64, bound + half_step(d64.abs() + bound, T))

    def check_words(self, words):
        """dW and dbias of some words, over all rows that count."""
        dw, dw_size, db, db_size = 0.0, 0.0, 0.0, 0.0
        for at in self.at.split(1 << 17):
            h = self.h[at].double()
            d = torch.exp(h @ self.w[words].double().t() - self.lse[at].double()[:, None])
            d -= (self.targets[at][:, None] == words[None]).double()
            dw, dw_size, db, db_size = dw + d.t() @ h, dw_size + d.abs().t() @ h.abs(), db + d.sum(dim=0), db_size + d.abs().sum(dim=0)
        n = len(self.at)
        bound = dw_size / n * (2.0 ** -8 + 2.0 ** -12)
        close(self.dw[words], dw / n, bound + half_step(dw.abs() / n + bound, T))
        # the logits' error (sums of |h||w| are below 2^6), the exponential's, and a 32nd of the parts one after the other
        close(self.db[words], db / n, db_size / n * ((self.hidden / 16 + 24) * 2.0 ** -17 + 2.0 ** -18 + (self.rows / 1024 + 40) * 2.0 ** -24))


def test_loss_over_many_pieces():
    """A vocabulary in many pieces, the last one short: words of the first, of inner ones and of the last."""
    p = Loss(40000, 64, 70001, seed=2)
    p.check_rows(torch.tensor([1, 19999, 30678, 39998], device="cuda"))
    p.check_words(torch.tensor([0, 1, 255, 256, 1023, 1024, 35000, 69631, 69632, 69999, 70000], device="cuda"))
    assert not p.dh[::5].any() and not p.loss[::5].any() and not p.lse[::5].any()


def test_loss_of_many_rows():
    """H, its copy of the rows that count and dH pass 2^31 elements."""
    p = Loss(2200003, 1024, 600, seed=3, every=200)
    assert len(p.at) * 1024 > 1 << 31
    p.check_rows(torch.tensor([1, 2097151, 2097153, 2108000 + 1, 2200002], device="cuda"))
    p.check_words(torch.tensor([0, 255, 256, 511, 599], device="cuda"))
    assert not p.dh[::200].any()


def test_loss_of_many_words():
    """W and dW pass 2^31 elements."""
    p = Loss(41, 1024, 2200003, seed=4)
    p.check_rows(torch.tensor([1, 39], device="cuda"))
    p.check_words(torch.tensor([0, 1, 2097151, 2097152, 2097153, 2200001, 2200002], device="cuda"))
    p.check_words(p.targets[p.at])
