"""Softmax cross entropy on top of the product that makes the logits, and its gradients, against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import TYPES, close, half_step, operand, placed, randn, untouched, workspace

pytestmark = pytest.mark.gpu
IGNORED = -100


class Problem:
    def __init__(self, rows, hidden, vocab, dtype, words=True, ignored=0.0, bias=True, scale=2.0, seed=0):
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        t = self.t = TYPES[dtype]
        self.rows, self.hidden, self.vocab = rows, hidden, vocab
        self.h = operand(randn(gen, rows, hidden), t, 8)
        w = randn(gen, vocab, hidden) * scale * hidden ** -0.5
        self.w = operand(w if words else w.t(), t)
        self.words = words
        self.bias = randn(gen, vocab) if bias else None
        self.targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        self.targets[torch.rand(rows, generator=gen, device="cuda") < ignored] = IGNORED
        self.ignore = IGNORED

    def logits(self):
        """Of the rows that count, with the bound of the 32-bit ones."""
        h, w = self.h.double()[self.counts()], (self.w.t() if self.words else self.w).double()
        bias = torch.zeros(self.vocab, device="cuda", dtype=torch.float64) if self.bias is None else self.bias.double()
        size = (h.abs() @ w.abs()).amax(dim=1, keepdim=True) if len(h) else h.new_zeros(0, 1)
        logits = h @ w + bias
        # words that a bias has taken out have no part in it
        most = torch.where(logits.abs() < 1e30, logits, 0.0).abs().amax(dim=1, keepdim=True) if len(h) else h.new_zeros(0, 1)
        return logits, size * ((self.hidden / 16 + 8) * 2.0 ** -23) + most * 2.0 ** -22

    def counts(self):
        return (self.targets != self.ignore).nonzero()[:, 0]

    def matrices(self):
        return qf.make_matrix(self.h), qf.make_matrix(self.w, self.words)

    def forward(self, mean=True):
        H, W = self.matrices()
        ws = workspace(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, False))
        out = torch.full((2, self.rows + 2), float("nan"), device="cuda")
        loss, lse = out[0, 1:], out[1, 1:]
        m = torch.full((1,), float("nan"), device="cuda")
        kind = qf.make_cross_entropy(self.t, self.ignore)
        qf.qfmt_linear_cross_entropy(H, W, kind, self.bias, self.targets, loss, lse, m if mean else None, ws, ws.numel())
        assert qf.qfmt_device_status(ws) == qf.QFMT_OK
        assert bool(torch.isnan(out[:, 0]).all()) and bool(torch.isnan(out[:, -1]).all())
        return loss[:-1], lse[:-1], m

    def check_forward(self):
        loss, lse, mean = self.forward()
        at, (logits, bound) = self.counts(), self.logits()
        want = torch.zeros(2, self.rows, device="cuda", dtype=torch.float64)
        tol = torch.full((self.rows,), 1e-300, device="cuda", dtype=torch.float64)
        want[0, at] = torch.logsumexp(logits, dim=1)
        want[1, at] = want[0, at] - logits.gather(1, self.targets[at][:, None])[:, 0]
        # exponentials and their sum: 2^-19; the logarithm and the product with ln 2: steps of lse
        tol[at] = bound[:, 0] + 2.0 ** -19 + want[0, at].abs() * 2.0 ** -22
        close(lse, want[0], tol)
        close(loss, want[1], 2.0 * tol)
        n = max(1, len(at))
        close(mean, want[1].sum().view(1) / n, 2.0 * tol.sum().view(1) / n + 1e-30 + want[1].sum().abs() / n * 2.0 ** -23)
        return lse

    def backward(self, lse, dloss=None, scale=None, mean=True, want=(True, True, True), pads=(0, 0), shifts=(0, 0)):
        H, W = self.matrices()
        ws = workspace(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, True))
        dh, hbuf = placed(self.h.shape, self.t, pads[0], shifts[0])
        dw, wbuf = placed(self.w.shape, self.t, pads[1], shifts[1])
        db = torch.full((self.vocab,), float("nan"), device="cuda")
        dls = None
        if scale is not None:
            dls = torch.zeros(14, device="cuda")
            dls[0] = scale
        kind = qf.make_cross_entropy(self.t, self.ignore, mean)
        qf.qfmt_linear_cross_entropy_backward(H, W, kind, self.bias, self.targets, lse, dloss, dls, dh if want[0] else None, dh.stride(0),
                                              dw if want[1] else None, dw.stride(0), db if want[2] else None, ws, ws.numel())
        assert qf.qfmt_device_status(ws) == qf.QFMT_OK
        assert untouched(dh, hbuf) and untouched(dw, wbuf)
        return dh, dw, db

    def gradients(self, lse, dloss=None, scale=None, mean=True):
        """The formulas, with bounds for what the kernels give."""
        at, (logits, bound) = self.counts(), self.logits()
        g = torch.ones(len(at), device="cuda", dtype=torch.float64)
        if dloss is not None:
            g = g * dloss[at].double()
        if mean:
            g = g / max(1, len(at))
        if scale is not None:
            g = g * scale
        g = g[:, None]
        l = lse[at].double()[:, None]
        p = torch.exp(logits - l)
        d = p.clone()
        d[torch.arange(len(at), device="cuda"), self.targets[at]] -= 1.0
        d *= g
        # p: the logit's and the exponent's errors; d: rounded to codes once (binary16 relative to the largest |g|)
        info = torch.finfo(self.t)
        de = g.abs() * p * (bound + l.abs() * 2.0 ** -22 + 2.0 ** -20) + d.abs() * 2.0 ** -21
        most = float(g.abs().max()) if len(at) else 0.0
        dc = de + (d.abs() + de) * (info.eps / 2) + (most * 2.0 ** -37 if self.t == torch.float16 else 1e-40)
        h, w = self.h.double()[at], (self.w.t() if self.words else self.w).double()
        dh, dh_tol = torch.zeros(2, self.rows, self.hidden, device="cuda", dtype=torch.float64).unbind(0)
        dh[at] = d @ w.t()
        tol = dc @ w.abs().t() + (d.abs() @ w.abs().t()) * ((self.vocab / 16 + 64) * 2.0 ** -23)
        dh_tol[at] = tol + half_step(dh[at].abs() + tol, self.t)
        dh_tol += 1e-300
        dw = h.t() @ d
        tol = h.abs().t() @ dc + (h.abs().t() @ d.abs()) * ((len(at) / 16 + 8) * 2.0 ** -23)
        dw_tol = tol + half_step(dw.abs() + tol, self.t)
        db = d.sum(dim=0)
        db_tol = de.sum(dim=0) + d.abs().sum(dim=0) * ((len(at) / 256 + 40) * 2.0 ** -23) + 1e-37
        return (dh, dw.t() if self.words else dw, db), (dh_tol, dw_tol.t() if self.words else dw_tol, db_tol)

    def check_backward(self, dloss=None, scale=None, mean=True, **kw):
        lse = self.forward(mean=False)[1]
        got = self.backward(lse, dloss, scale, mean, **kw)
        for name, a, b, tol in zip(("dh", "dw", "dbias"), got, *self.gradients(lse, dloss, scale, mean)):
            close(a, b, tol)
        return got


SHAPES = [(1, 1, 1), (1, 64, 300), (2, 8, 3), (5, 33, 129), (31, 72, 1000), (64, 128, 256), (257, 200, 515), (300, 64, 5003), (1000, 520, 2049),
          (2500, 96, 777)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, words, dtype):
    Problem(*shape, dtype, words, seed=shape[2]).check_forward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, words, dtype):
    Problem(*shape, dtype, words, seed=shape[2]).check_backward(scale=2.0 ** 10)


@pytest.mark.parametrize("ignored", [0.1, 0.85, 0.999, 1.0])
@pytest.mark.parametrize("shape", [(40, 64, 300), (900, 100, 1111), (3000, 136, 260)])
def test_rows_that_do_not_count(shape, ignored):
    """They get zeros, and whatever H holds there has no effect."""
    p = Problem(*shape, "bf16", True, ignored, bias=False)
    out = [t.clone() for t in (*p.forward(), *p.check_backward())]
    p.check_forward()
    p.h[p.targets == IGNORED] = float("nan")
    for a, b in zip(out, (*p.forward(), *p.backward(out[1]))):
        assert torch.equal(a, b)
    assert not out[0][p.targets == IGNORED].any() and not out[3][p.targets == IGNORED].any()


def test_no_row_counts():
    p = Problem(70, 64, 300, "f16")
    p.targets[:] = IGNORED
    loss, lse, mean = p.forward()
    assert not loss.any() and not lse.any() and not mean.any()
    for g in p.backward(lse):
        assert not g.any()


def test_no_rows():
    p = Problem(3, 64, 300, "bf16")
    H, W = qf.qfmt_matrix_t(None, 0, 64, 64, 0), qf.make_matrix(p.w, True)
    ws = workspace(qf.qfmt_linear_cross_entropy_workspace_bytes(H, W, True))
    mean, db = torch.full((1,), float("nan"), device="cuda"), torch.full((300,), float("nan"), device="cuda")
    dw = torch.full((300, 64), float("nan"), device="cuda", dtype=p.t)
    kind = qf.make_cross_entropy(p.t)
    qf.qfmt_linear_cross_entropy(H, W, kind, None, None, None, None, mean, ws, ws.numel())
    qf.qfmt_linear_cross_entropy_backward(H, W, kind, None, None, None, None, None, None, 0, dw, 64, db, ws, ws.numel())
    assert not mean.any() and not db.any() and not dw.any()


def test_another_word_that_does_not_count():
    """A target inside the vocabulary (padding) as the one that does not count."""
    p = Problem(200, 72, 500, "bf16")
    p.targets[::3], p.ignore = 0, 0
    p.check_forward()
    p.check_backward()


def test_targets_that_are_no_words():
    p = Problem(100, 64, 300, "bf16")
    good = p.forward()
    p.targets[5], p.targets[50], p.targets[51] = 300, -1, 1 << 40
    loss, lse, mean = p.forward()
    bad = torch.zeros(100, dtype=torch.bool, device="cuda")
    bad[5] = bad[50] = bad[51] = True
    assert bool(torch.isnan(loss[bad]).all()) and bool(torch.isnan(lse[bad]).all()) and bool(torch.isnan(mean).all())
    assert torch.equal(loss[~bad], good[0][~bad])
    dh = p.backward(lse)[0]
    assert bool(torch.isnan(dh[bad]).all()) and bool(torch.isfinite(dh[~bad]).all())


def test_words_taken_out():
    """A bias of -infinity takes a word out: its probability is 0 and so is its row of the weight's gradient; a bias of the type's
    lowest value comes to the same."""
    for low in (float("-inf"), -3.4e38):
        p = Problem(90, 64, 1000, "bf16")
        out = torch.arange(1000, device="cuda") % 3 == 0
        out[600:900] = True
        p.bias[out] = low
        p.targets = torch.where(out[p.targets], torch.full_like(p.targets, 1), p.targets)
        p.check_forward()
        dh, dw, db = p.check_backward()
        assert not dw[out].any() and not db[out].any()


def test_all_words_at_the_lowest_value():
    """A row of equal logits, however low: every word has the same probability."""
    p = Problem(70, 64, 300, "bf16", scale=0.0)
    p.bias[:] = -3.4e38
    loss, lse, _ = p.forward()
    assert bool((lse == p.bias[0]).all()) and not loss.any()  # log(300) is far below a step of such an lse
    dh, dw, db = p.backward(lse, mean=False)
    # with lse rounded to -3.4e38 the formula gives every word probability exp(0) = 1
    want = 70.0 - torch.bincount(p.targets, minlength=300)
    assert torch.equal(db, want.float())


def test_all_words_taken_out():
    p = Problem(3, 64, 300, "bf16")
    p.bias[:] = float("-inf")
    loss, lse, mean = p.forward()
    assert bool((lse == float("-inf")).all()) and bool(torch.isnan(loss).all())


def test_infinite_and_nan_logits():
    p = Problem(40, 64, 300, "f16")
    p.bias[7] = float("inf")
    assert bool(torch.isnan(p.forward()[0]).all())  # infinity minus infinity, as the formula says
    p.bias[7] = float("nan")
    assert bool(torch.isnan(p.forward()[0]).all())
    p.bias[7] = 0.0
    p.h[3] = float("nan")
    loss = p.forward()[0]
    assert bool(torch.isnan(loss[3])) and int(torch.isnan(loss).sum()) == 1


@pytest.mark.parametrize("scale", [0.0, 30.0, 200.0])
def test_logits_of_any_size(scale):
    """All equal, and so far apart that one word has all the probability."""
    p = Problem(130, 128, 700, "bf16", scale=scale, bias=False)
    p.check_forward()
    p.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("mean", [True, False])
def test_gradients_of_rows_of_their_own(dtype, mean):
    p = Problem(500, 72, 1500, dtype, ignored=0.2)
    dloss = randn(p.gen, 500) * torch.exp2(4.0 * randn(p.gen, 500))
    dloss[::7] = 0.0
    dloss[p.targets == IGNORED] = float("nan")
    p.check_backward(dloss, 2.0 ** 12, mean)


@pytest.mark.parametrize("factor", [2.0 ** -60, 2.0 ** 40])
def test_gradients_of_any_size(factor):
    """bfloat16 codes hold them; binary16 ones on the way are scaled, so that only the results are limited by the type."""
    p = Problem(300, 64, 900, "bf16")
    p.check_backward(torch.full((300,), factor, device="cuda"))
    p = Problem(300, 64, 900, "f16")
    p.check_backward(torch.full((300,), 2.0 ** -6, device="cuda"))


@pytest.mark.parametrize("want", [(True, False, False), (False, True, False), (False, False, True), (False, True, True)])
def test_what_is_left_out(want):
    p = Problem(270, 100, 1300, "bf16", ignored=0.1)
    lse = p.forward()[1]
    for w, a, b in zip(want, p.backward(lse), p.backward(lse, want=want)):
        assert torch.equal(a, b) if w else bool(torch.isnan(b).all())


@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("pads,shifts", [((8, 8), (0, 0)), ((0, 0), (1, 1)), ((3, 5), (2, 7))])
def test_strides_and_alignments(words, pads, shifts):
    for hidden in (136, 131):
        p = Problem(140, hidden, 1100, "f16", words, ignored=0.3)
        lse = p.forward()[1]
        for a, b in zip(p.backward(lse), p.backward(lse, pads=pads, shifts=shifts)):
            assert torch.equal(a, b)


def test_pieces_of_the_vocabulary():
    """Many rows: the vocabulary is walked in several pieces, the last one short."""
    p = Problem(9000, 64, 7700, "bf16", ignored=0.5)
    p.check_forward()
    p.check_backward(scale=2.0 ** 14)


def test_gradients_by_differences():
    p = Problem(60, 64, 400, "f16", ignored=0.2)
    loss, lse, _ = p.forward()
    dh, dw, db = p.backward(lse, mean=True, scale=2.0 ** 8)
    at = p.counts()

    def mean(h, w, b):
        logits = h[at] @ w.t() + b
        return float((torch.logsumexp(logits, dim=1) - logits.gather(1, p.targets[at][:, None])[:, 0]).mean())

    args, eps = [p.h.double(), p.w.double(), p.bias.double()], 2.0 ** -10
    for i, g in enumerate((dh, dw, db)):
        for _ in range(3):
            v = torch.randn(g.shape, generator=p.gen, device="cuda", dtype=torch.float64)
            lo, hi = list(args), list(args)
            lo[i], hi[i] = args[i] - eps * v, args[i] + eps * v
            slope = (mean(*hi) - mean(*lo)) / (2.0 * eps)
            # each element is off by about two half steps of its own and of its terms; their errors add up in squares
            g64 = g.double() / 2.0 ** 8
            size = float((g64 * v).square().sum().sqrt())
            assert abs(slope - float((g64 * v).sum())) < 64 * 2.0 ** -11 * size + 2.0 ** -18


def test_captured_graphs_share_a_workspace():
    """Two captured graphs and eager calls between them, all on one workspace, one stream."""
    a, b = Problem(300, 64, 900, "bf16", ignored=0.5, seed=1), Problem(500, 72, 700, "bf16", seed=2)
    calls = []
    ws = workspace(max(qf.qfmt_linear_cross_entropy_workspace_bytes(*p.matrices(), k) for p in (a, b) for k in (False, True)))
    for p in (a, b):
        H, W = p.matrices()
        kind = qf.make_cross_entropy(p.t)
        out = [torch.empty(p.rows, device="cuda"), torch.empty(p.rows, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(p.h),
               torch.empty_like(p.w), torch.empty(p.vocab, device="cuda")]

        def call(p=p, H=H, W=W, kind=kind, out=out):
            qf.qfmt_linear_cross_entropy(H, W, kind, p.bias, p.targets, *out[:3], ws, ws.numel())
            qf.qfmt_linear_cross_entropy_backward(H, W, kind, p.bias, p.targets, out[1], None, None, out[3], out[3].stride(0), out[4],
                                                  out[4].stride(0), out[5], ws, ws.numel())
        calls.append((call, out))
    graphs = []
    for call, _ in calls:
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for step in range(3):
        for p in (a, b):
            p.targets.copy_(torch.randint(0, p.vocab, (p.rows,), generator=p.gen, device="cuda"))
            p.targets[torch.rand(p.rows, generator=p.gen, device="cuda") < 0.3 * step] = IGNORED
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for call, out in calls:
            got = [t.clone() for t in out]
            call()
            torch.cuda.synchronize()
            for x, y in zip(got, out):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("rows", [1, 3, 8, 9, 16, 17, 32, 33])
def test_few_rows(rows, words, dtype):
    for hidden, vocab in ((64, 1), (8, 65), (1024, 3001), (100, 40000)):
        Problem(rows, hidden, vocab, dtype, words, 0.2 if rows > 4 else 0.0, seed=rows).check_forward()


def test_few_rows_with_words_taken_out_and_targets_that_are_none():
    p = Problem(20, 72, 900, "bf16")
    p.bias[100:800] = float("-inf")
    p.targets[:] = torch.arange(20, device="cuda")
    p.check_forward()
    p.targets[3], p.targets[4], p.targets[5] = 900, -1, IGNORED
    p.h[5] = float("nan")
    loss, lse, mean = p.forward()
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[3] = bad[4] = True
    assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(lse), bad) and bool(torch.isnan(mean))
    assert float(loss[5]) == 0.0 == float(lse[5])
    p.bias[:] = float("-inf")
    assert bool((p.forward()[1][:3] == float("-inf")).all())
    p.bias[:] = -3.4e38
    p.h[:] = 0.0
    assert bool((p.forward()[1][:3] == p.bias[0]).all())


@pytest.mark.parametrize("words", [True, False])
@pytest.mark.parametrize("shape", [(33, 64, 1000), (64, 40, 30000), (100, 200, 777), (500, 33, 100), (1000, 64, 515), (1024, 100, 1000)])
def test_little_work(shape, words):
    """Passes over W for blocks of 32 rows, the mean over all of them."""
    for ignored in (0.0, 0.4):
        p = Problem(*shape, "bf16", words, ignored, seed=shape[0])
        p.check_forward()
    p.targets[shape[0] // 2] = -7
    loss, lse, mean = p.forward()
    assert int(torch.isnan(loss).sum()) == 1 and bool(torch.isnan(mean))
    p.targets[:] = IGNORED
    loss, lse, mean = p.forward()
    assert not loss.any() and not lse.any() and not mean.any()
