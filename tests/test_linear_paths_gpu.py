"""Products with an epilogue on every path they may take, each named by its test: a pass over the weights, tiles on single CTAs, tiles on
CTA pairs, and tiles whose K is shared with the epilogue in a pass of its own.  Against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import ACTS, close, half_step, randn, workspace
from test_linear_act_gpu import backward, code, forward, product

pytestmark = pytest.mark.gpu


def ceil(a, b):
    return -(-a // b)


def path_of(m, n, k, ta=False, tb=False):
    """Where a product goes by its sizes and layouts."""
    if not ta and k <= 1 << 16 and ((tb and m <= 32) or (m <= 1024 and m * n * k <= 1 << 27)):
        return "weights"
    singles, pairs, stages = ceil(m, 128) * ceil(n, 256), ceil(m, 256) * ceil(n, 256), ceil(k, 64)
    pair = singles > 148 and 4 * ceil(singles, 148) > 3 * ceil(pairs, 74)
    if min((74 // pairs if pair else 148 // singles), stages // 4, 16) > 1:
        return "shared"
    return "pairs" if pair else "tiles"


# aligned and ragged columns
PATHS = [("weights", (300, 328, 200)), ("weights", (300, 325, 200)), ("tiles", (1100, 328, 200)), ("tiles", (1100, 325, 200)),
         ("pairs", (5000, 1000, 72)), ("pairs", (5003, 1001, 70)), ("shared", (1100, 328, 1000)), ("shared", (1100, 325, 1001))]
EACH = pytest.mark.parametrize("path,shape", PATHS, ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ACTS)
@EACH
def test_activations(path, shape, act, dtype):
    assert path_of(*shape) == path and path_of(*shape, tb=True) == path
    forward(*shape, dtype, act)
    backward(*shape, dtype, act)


@pytest.mark.parametrize("ta,tb", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("path,shape", [("tiles", (136, 200, 72)), ("tiles", (130, 70, 50)), ("pairs", (5000, 1000, 72)), ("pairs", (5003, 1001, 70)),
                                        ("shared", (136, 200, 1000)), ("shared", (131, 203, 1003))])
def test_layouts(path, shape, ta, tb):
    assert not ta or path_of(*shape, ta, tb) == path
    forward(*shape, "bf16", "silu", ta, tb)
    backward(*shape, "f16", "gelu_tanh", ta, tb)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@EACH
def test_what_is_left_out(path, shape, residual, keep, bias):
    act = "gelu" if bias else "relu"
    forward(*shape, "bf16", act, residual=residual, keep=keep, bias=bias)
    backward(*shape, "f16", act if keep else "none", residual=residual, dbias=bias)


@pytest.mark.parametrize("pads,shifts", [((8, 16, 8), (0, 0, 0)), ((0, 0, 0), (1, 0, 0)), ((3, 0, 0), (0, 0, 0)), ((0, 5, 0), (0, 3, 0)),
                                         ((0, 0, 1), (0, 0, 7)), ((1, 2, 3), (4, 5, 6))])
@EACH
def test_strides_and_alignments(path, shape, pads, shifts):
    """Any of them gives the bits of the dense, aligned tensors."""
    assert torch.equal(forward(*shape, "bf16", "gelu", pads=pads, shifts=shifts), forward(*shape, "bf16", "gelu"))
    for act in ("gelu", "none"):
        (dz, db), (dz0, db0) = (backward(*shape, "f16", act, pads=p, shifts=s) for p, s in ((pads, shifts), ((0, 0, 0), (0, 0, 0))))
        assert torch.equal(dz, dz0) and torch.equal(db[1:-1], db0[1:-1])


@EACH
def test_in_place(path, shape):
    gen = torch.Generator(device="cuda").manual_seed(3)
    (m, n, k), t = shape, torch.bfloat16
    A, B, a64, b64, held = product(gen, m, n, k, t, False, False)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    r, z, y = randn(gen, m, n).to(t), randn(gen, m, n).to(t), torch.empty(m, n, device="cuda", dtype=t)
    same = r.clone()
    qf.qfmt_linear_act(A, B, qf.make_epilogue(code("gelu"), None, r), y, n, t, ws, ws.numel())
    qf.qfmt_linear_act(A, B, qf.make_epilogue(code("gelu"), None, same), same, n, t, ws, ws.numel())
    assert torch.equal(y, same)
    for act in ("gelu", "none"):
        qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code(act), None, r, 0, z), y, n, None, t, ws, ws.numel())
        for alias in ("r", "z"):
            rr, zz = r.clone(), z.clone()
            out = rr if alias == "r" else zz
            qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code(act), None, rr, 0, zz), out, n, None, t, ws, ws.numel())
            assert torch.equal(y, out)


@EACH
def test_infinities_and_nan(path, shape):
    (m, n, k), t = shape, torch.float16
    x, w = torch.zeros(m, ceil(k, 8) * 8, device="cuda", dtype=t)[:, :k], torch.zeros(k, ceil(n, 8) * 8, device="cuda", dtype=t)[:, :n]
    x[:, 0], w[0] = 1.0, 1.0
    x[7, 0], x[8, 0], x[9, 0], x[10, 0] = float("inf"), float("-inf"), float("nan"), 6e4
    w[0, 3] = 2.0
    A, B = qf.make_matrix(x), qf.make_matrix(w)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    y = torch.empty(m, n, device="cuda", dtype=t)
    for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        qf.qfmt_linear_act(A, B, qf.make_epilogue(code(act)), y, n, t, ws, ws.numel())
        assert bool((y[7] == float("inf")).all()) and bool(torch.isnan(y[9]).all())
        assert float(y[10, 0]) == 6e4 and float(y[10, 3]) == float("inf") and bool(torch.isfinite(y[11:]).all())
        if act == "none":
            assert bool((y[8] == float("-inf")).all())
        if act == "relu":
            assert not y[8].any()
    z = torch.ones(m, n, device="cuda", dtype=t)
    db = torch.empty(n, device="cuda")
    for act in ("none", "relu", "gelu", "silu"):
        x[8, 0], x[9, 0] = 1.0, 1.0
        qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code(act), None, None, 0, z), y, n, db, t, ws, ws.numel())
        assert bool((y[7] == float("inf")).all()) and bool((db == float("inf")).all()) and bool(torch.isfinite(y[11:]).all())
        x[9, 0] = float("nan")
        qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code(act), None, None, 0, z), y, n, db, t, ws, ws.numel())
        assert bool(torch.isnan(y[9]).all()) and bool(torch.isnan(db).all()) and bool(torch.isfinite(y[11:]).all())


@pytest.mark.parametrize("ta", [False, True])
@EACH
def test_an_infinite_weight(path, shape, ta):
    """Column sums are those of the matrix' own rows: infinite where every dz of the column is, whatever the rows beyond a tile's."""
    (m, n, k), t = shape, torch.bfloat16
    pad = lambda v: ceil(v, 8) * 8
    x = (torch.ones(k, pad(m), device="cuda", dtype=t)[:, :m] if ta else torch.ones(m, pad(k), device="cuda", dtype=t)[:, :k])
    w = torch.ones(k, pad(n), device="cuda", dtype=t)[:, :n]
    w[0, 3], w[k - 1, n - 1] = float("inf"), float("-inf")
    A, B = qf.make_matrix(x, ta), qf.make_matrix(w)
    z, dz, db = torch.ones(m, n, device="cuda", dtype=t), torch.empty(m, n, device="cuda", dtype=t), torch.empty(n, device="cuda")
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    for act in ("none", "relu"):
        qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code(act), None, None, 0, z), dz, n, db, t, ws, ws.numel())
        want = torch.full((n,), float(m * k), device="cuda")
        want[3], want[n - 1] = float("inf"), float("-inf")
        assert torch.equal(db, want)


@EACH
def test_captured_on_a_side_stream(path, shape):
    gen = torch.Generator(device="cuda").manual_seed(9)
    (m, n, k), t = shape, torch.bfloat16
    A, B, a64, b64, (x, w) = product(gen, m, n, k, t, False, False)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    y, z, dz = (torch.empty(m, n, device="cuda", dtype=t) for _ in range(3))
    db = torch.empty(n, device="cuda")
    e = qf.make_epilogue(code("silu"), None, None, 0, z)

    def call():
        qf.qfmt_linear_act(A, B, e, y, n, t, ws, ws.numel())
        qf.qfmt_linear_act_backward(A, B, e, dz, n, db, t, ws, ws.numel())

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    torch.cuda.synchronize()
    for _ in range(3):
        x.copy_(randn(gen, m, k))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y, z, dz, db)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, z, dz, db)))
        assert qf.qfmt_device_status(ws) == qf.QFMT_OK


def test_less_workspace_shares_less():
    """As many parts as the workspace holds; the least is none, and the sums of the product stay in one piece."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    t, (m, n, k) = torch.float16, (1100, 328, 2056)
    assert path_of(m, n, k) == "shared"
    A, B, a64, b64, held = product(gen, m, n, k, t, False, True)
    full = qf.qfmt_linear_act_workspace_bytes(A, B)
    one = m * n * 4
    assert full >= 256 + 7 * one
    want, bound = a64 @ b64, (a64.abs() @ b64.abs()) * ((k / 16 + 24) * 2.0 ** -23)
    for size in (256, 256 + 2 * one, 256 + 4 * one, full):
        ws, y = workspace(size), torch.empty(m, n, device="cuda", dtype=t)
        qf.qfmt_linear_act(A, B, qf.make_epilogue(), y, n, t, ws, size)
        close(y, want, bound + half_step(want.abs() + bound, t))
        if size == 256:
            assert int((ws[16:] != 0xA5).sum()) == 0  # nothing but the status area
