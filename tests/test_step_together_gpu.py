"""One training step through the calls as a program makes them: a feed-forward layer with GELU and a residual, the loss over a
vocabulary, all gradients, the loss scale's controller and clipping; eagerly and captured."""
import math

import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import act64, operand, randn, workspace

pytestmark = pytest.mark.gpu
IGNORED = -100


class Step:
    """y = gelu(x W1 + b1) W2 + b2 + x, loss = cross entropy of y E^T + c; weights in codes, gradients of weights in fp32 or codes."""

    def __init__(self, rows, hidden, inner, vocab, dtype, most, seed):
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        t = self.t = dtype
        self.rows, self.hidden, self.inner, self.vocab, self.most = rows, hidden, inner, vocab, most
        self.x = operand(randn(gen, rows, hidden), t)
        self.w1, self.w2 = operand(randn(gen, hidden, inner) * hidden ** -0.5, t), operand(randn(gen, inner, hidden) * inner ** -0.5, t)
        self.e = operand(randn(gen, vocab, hidden) * hidden ** -0.5, t)
        self.b1, self.b2, self.c = 0.1 * randn(gen, inner), 0.1 * randn(gen, hidden), 0.1 * randn(gen, vocab)
        self.targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        self.targets[torch.rand(rows, generator=gen, device="cuda") < 0.3] = IGNORED
        like = lambda v: torch.empty_strided(v.shape, v.stride(), device="cuda", dtype=t)
        self.z = operand(torch.empty(rows, inner, device="cuda"), t)
        self.a, self.dz, self.y, self.dy, self.dx = like(self.z), like(self.z), like(self.x), like(self.x), like(self.x)
        self.loss, self.lse = torch.empty(2, rows, device="cuda").unbind(0)
        self.mean = torch.empty(1, device="cuda")
        self.de = torch.empty(vocab, hidden, device="cuda", dtype=t)
        self.dw1, self.dw2 = torch.empty(hidden, inner, device="cuda"), torch.empty(inner, hidden, device="cuda")
        self.db1, self.db2, self.dc = torch.empty(inner, device="cuda"), torch.empty(hidden, device="cuda"), torch.empty(vocab, device="cuda")
        self.grads = [self.dw1, self.dw2, self.db1, self.db2, self.dc, self.de]
        rec = qf.qfmt_dls_t(2.0 ** 8, 2.0, 0.5, 1.0, 2.0 ** 16, 1000, 0, 0, 0, 0, 0)
        self.dls = torch.frombuffer(bytearray(bytes(rec)), dtype=torch.uint8).cuda()
        self.stats = torch.zeros(qf.STATS_WORDS, dtype=torch.int64, device="cuda")
        self.norm = torch.zeros(2, dtype=torch.int64, device="cuda")
        host = qf.make_tensors(self.grads, self.grads)
        self.count, self.chunks = len(host), qf.qfmt_plan_tensors(host, len(host))
        self.list = torch.frombuffer(host, dtype=torch.uint8).cuda()
        mat = qf.make_matrix
        self.m = {k: mat(getattr(self, k)) for k in ("x", "w1", "w2", "e", "a", "dz", "y", "dy")}
        self.m.update({k + "t": mat(getattr(self, k), True) for k in ("x", "w1", "w2", "e", "a")})
        m, g, act = self.m, qf.QFMT_ACT_GELU, qf.qfmt_linear_act_workspace_bytes
        self.kind = qf.make_cross_entropy(t, IGNORED)
        self.fmt = qf.make_format(5, 10) if t is torch.float16 else qf.make_format(8, 7)
        pack = qf.qfmt_gemm_packed16_workspace_bytes
        self.ws = workspace(max(act(m["x"], m["w1"]), act(m["a"], m["w2"]), act(m["dy"], m["w2t"]), act(m["dz"], m["w1t"]),
                                pack(m["at"], m["dy"]), pack(m["xt"], m["dz"]), qf.qfmt_act_backward_workspace_bytes(rows, hidden),
                                qf.qfmt_grad_norm_workspace_bytes(self.count, self.chunks),
                                *(qf.qfmt_linear_cross_entropy_workspace_bytes(m["y"], m["et"], k) for k in (False, True))))
        ld = self.z.stride(0)
        self.up = qf.make_epilogue(g, self.b1, None, 0, self.z, ld)
        self.down = qf.make_epilogue(qf.QFMT_ACT_NONE, self.b2, self.x, self.x.stride(0))
        self.through = qf.make_epilogue(g, None, None, 0, self.z, ld)
        self.back = qf.make_epilogue(qf.QFMT_ACT_NONE, None, self.dy, self.dy.stride(0))

    def run(self):
        m, ws, n = self.m, self.ws, self.ws.numel()
        h, f, t = self.hidden, self.inner, self.t
        ldh, ldf = self.x.stride(0), self.z.stride(0)
        qf.qfmt_linear_act(m["x"], m["w1"], self.up, self.a, ldf, t, ws, n)
        qf.qfmt_linear_act(m["a"], m["w2"], self.down, self.y, ldh, t, ws, n)
        qf.qfmt_linear_cross_entropy(m["y"], m["et"], self.kind, self.c, self.targets, self.loss, self.lse, self.mean, ws, n)
        qf.qfmt_linear_cross_entropy_backward(m["y"], m["et"], self.kind, self.c, self.targets, self.lse, None, self.dls, self.dy, ldh, self.de, h,
                                              self.dc, ws, n)
        qf.qfmt_act_backward(self.dy, ldh, None, 0, None, 0, self.db2, self.rows, h, t, qf.QFMT_ACT_NONE, ws, n)
        qf.qfmt_linear_act_backward(m["dy"], m["w2t"], self.through, self.dz, ldf, self.db1, t, ws, n)
        qf.qfmt_gemm_packed16(m["at"], m["dy"], self.dw2, h, self.fmt, ws, n)
        qf.qfmt_gemm_packed16(m["xt"], m["dz"], self.dw1, f, self.fmt, ws, n)
        qf.qfmt_linear_act_backward(m["dz"], m["w1t"], self.back, self.dx, ldh, None, t, ws, n)
        qf.qfmt_grad_norm(self.list, self.count, self.chunks, self.most, self.dls, self.norm, self.stats, ws, n)
        qf.qfmt_grad_clip(self.list, self.count, self.chunks, self.norm)
        qf.qfmt_dls_update(self.dls, self.stats, 1)

    def results(self):
        return [v.clone() for v in (self.mean, self.y, self.dx, *self.grads, self.norm, self.dls)]

    def formulas(self):
        """Loss and gradients by differentiating in 64 bits."""
        p = [v.double().requires_grad_() for v in (self.x, self.w1, self.w2, self.b1, self.b2, self.c, self.e)]
        x, w1, w2, b1, b2, c, e = p
        y = act64("gelu", x @ w1 + b1) @ w2 + b2 + x
        at = (self.targets != IGNORED).nonzero()[:, 0]
        loss = torch.nn.functional.cross_entropy((y @ e.t() + c)[at], self.targets[at])
        dx, *grads = torch.autograd.grad(loss, p)
        return loss.detach(), y.detach(), dx, grads


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [(300, 64, 136, 1000), (40, 33, 70, 517), (1200, 256, 520, 5003), (6, 64, 128, 900)])
def test_gradients_of_a_step(sizes, dtype):
    s = Step(*sizes, dtype, 1e6, seed=sizes[0])
    s.run()
    loss, y, dx, (dw1, dw2, db1, db2, dc, de) = s.formulas()
    scale = 2.0 ** 8
    # What is rounded to codes on the way (z, a, y, d, dy, dz) is off by half a step of its value each: at most four of them meet in any
    # result, and each result is a sum of many such terms, whose errors add up in squares; eps stands for all of them with room for the
    # inner product's growth of relative errors by cancellation, which the norm over the whole tensor averages.
    eps = torch.finfo(dtype).eps
    assert abs(float(s.mean) - float(loss)) <= 8 * eps * float(loss)
    for got, want, k in ((s.y, y, 1.0), (s.dx, dx, scale), (s.dw1, dw1, 1.0), (s.dw2, dw2, 1.0), (s.db1, db1, 1.0), (s.db2, db2, 1.0),
                         (s.dc, dc, 1.0), (s.de, de, 1.0)):  # gradients of parameters have the loss scale taken out
        err = float((got.double() / k - want).norm() / want.norm())
        assert err <= 4 * eps, err
    norm = float(s.norm.view(torch.float32)[0])
    want = math.sqrt(sum(float(g.square().sum()) for g in (dw1, dw2, db1, db2, dc, de)))
    assert abs(norm - want) <= 4 * eps * want


def test_clipped_and_captured():
    s = Step(200, 72, 136, 700, torch.bfloat16, 0.25, seed=3)
    s.run()
    clipped = math.sqrt(sum(float(g.double().square().sum()) for g in s.grads))
    assert abs(clipped - 0.25) <= 0.25 * 2.0 ** -7
    want = s.results()[:-1]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(s.results()[:-1], want):  # all but the controller's record, which counts steps
            assert torch.equal(a, b)
    after = qf.qfmt_dls_t.from_buffer_copy(s.dls.cpu().numpy().tobytes())
    assert after.n_steps == 4 and after.n_skipped == 0 and after.clean_steps == 4


def test_two_steps_at_once():
    """Two steps with workspaces of their own on two streams."""
    steps = [Step(150, 64, 136, 900, torch.bfloat16, 1.0, seed=k) for k in (1, 2)]
    for s in steps:
        s.run()
    torch.cuda.synchronize()
    want = [s.results()[:-1] for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(4):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.results()[:-1], w):
            assert torch.equal(a, b)
        assert qf.qfmt_device_status(s.ws) == qf.QFMT_OK


def test_an_overflow_skips_the_step():
    """binary16 with a loss scale that the gradients do not stand: the controller halves it and nothing is clipped."""
    s = Step(64, 64, 128, 300, torch.float16, 1.0, seed=5)
    s.dls.view(torch.float32)[0] = 2.0 ** 40
    s.run()
    after = qf.qfmt_dls_t.from_buffer_copy(s.dls.cpu().numpy().tobytes())
    assert after.skip == 1 and after.scale == 2.0 ** 39 and int(s.norm[1]) > 0 and float(s.norm.view(torch.float32)[1]) == 1.0
