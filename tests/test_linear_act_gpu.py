"""Products with bias, activation and residual in the epilogue, forward and backward, against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import ACTS, TYPES, act64, close, half_step, operand, placed, randn, slope64, sum_bound, untouched, workspace

pytestmark = pytest.mark.gpu


def code(act):
    return getattr(qf, "QFMT_ACT_" + act.upper())


def product(gen, m, n, k, dtype, ta, tb, scale=1.0):
    a, b = randn(gen, m, k) * scale, randn(gen, k, n) * k ** -0.5
    da, db = operand(a.t() if ta else a, dtype, 8), operand(b.t() if tb else b, dtype)
    a64, b64 = (da.t() if ta else da).double(), (db.t() if tb else db).double()
    return qf.make_matrix(da, ta), qf.make_matrix(db, tb), a64, b64, (da, db)


def forward(m, n, k, dtype, act, ta=False, tb=False, residual=True, keep=True, bias=True, pads=(0, 0, 0), shifts=(0, 0, 0), seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    A, B, a64, b64, held = product(gen, m, n, k, t, ta, tb)
    bv = 0.2 * randn(gen, n) if bias else None
    y, ybuf = placed((m, n), t, pads[0], shifts[0])
    z, zbuf = placed((m, n), t, pads[1], shifts[1]) if keep else (None, None)
    r = placed((m, n), t, pads[2], shifts[2], randn(gen, m, n))[0] if residual else None
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    e = qf.make_epilogue(code(act), bv, r, n + pads[2], z, n + pads[1])
    qf.qfmt_linear_act(A, B, e, y, n + pads[0], t, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
    z64 = a64 @ b64 + (bv.double() if bias else 0.0)
    bound = sum_bound(a64, b64, k) + z64.abs() * 2.0 ** -23
    y64 = act64(act, z64)
    want = y64 + (r.double() if residual else 0.0)
    close(y, want, bound * 1.13 + y64.abs() * 2.0 ** -18 + half_step(want.abs() + bound, t))
    if keep:
        close(z, z64, bound + half_step(z64.abs() + bound, t))
        assert untouched(z, zbuf)
    assert untouched(y, ybuf)
    return y


def backward(m, n, k, dtype, act, ta=False, tb=True, residual=True, dbias=True, pads=(0, 0, 0), shifts=(0, 0, 0), seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    A, B, a64, b64, held = product(gen, m, n, k, t, ta, tb, 2.0 ** -4)
    dz, dbuf = placed((m, n), t, pads[0], shifts[0])
    z = placed((m, n), t, pads[1], shifts[1], 2.0 * randn(gen, m, n))[0] if act != "none" else None
    r = placed((m, n), t, pads[2], shifts[2], randn(gen, m, n) * 2.0 ** -4)[0] if residual else None
    db = torch.full((n + 2,), float("nan"), device="cuda") if dbias else None
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    e = qf.make_epilogue(code(act), None, r, n + pads[2], z, n + pads[1])
    qf.qfmt_linear_act_backward(A, B, e, dz, n + pads[0], None if db is None else db[1:], t, ws, ws.numel())
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
    g64 = a64 @ b64 + (r.double() if residual else 0.0)
    slope = slope64(act, z.double()) if act != "none" else torch.ones_like(g64)
    want = g64 * slope
    bound = (sum_bound(a64, b64, k) + g64.abs() * 2.0 ** -23) * 1.13 + g64.abs() * 2.0 ** -18
    close(dz, want, bound + half_step(want.abs() + bound, t))
    assert untouched(dz, dbuf)
    if dbias:
        parts = (m + 255) // 256 + 40
        close(db[1:n + 1], want.sum(dim=0), bound.sum(dim=0) + want.abs().sum(dim=0) * parts * 2.0 ** -23 + 1e-37)
        assert bool(torch.isnan(db[0])) and bool(torch.isnan(db[n + 1]))
    return dz, db


SHAPES = [(1, 1, 1), (1, 8, 64), (3, 5, 7), (1, 1000, 520), (33, 257, 65), (128, 256, 192), (255, 129, 63), (256, 256, 256), (257, 511, 1025),
          (700, 1913, 1001), (2048, 4096, 512), (17, 300, 6000)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    forward(*shape, dtype, "gelu", tb=shape[0] % 2 == 0, seed=shape[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype):
    backward(*shape, dtype, "gelu", tb=shape[0] % 2 == 0, seed=shape[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    for shape in ((300, 328, 200), (5, 328, 1200)):  # in the product's epilogue, and behind shared sums
        forward(*shape, dtype, act)
        backward(*shape, dtype, act)


@pytest.mark.parametrize("ta", [False, True])
@pytest.mark.parametrize("tb", [False, True])
@pytest.mark.parametrize("shape", [(200, 320, 136), (264, 200, 72), (130, 70, 50)])
def test_operand_layouts(shape, ta, tb):
    forward(*shape, "bf16", "silu", ta, tb)
    backward(*shape, "f16", "silu", ta, tb)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_what_is_left_out(residual, keep, bias):
    for shape in ((300, 264, 128), (2, 264, 1024)):
        forward(*shape, "bf16", "relu", residual=residual, keep=keep, bias=bias)
        backward(*shape, "bf16", "relu", residual=residual, dbias=keep)


@pytest.mark.parametrize("pads,shifts", [((8, 16, 8), (0, 0, 0)), ((0, 0, 0), (1, 0, 0)), ((3, 0, 0), (0, 0, 0)), ((0, 5, 0), (0, 3, 0)),
                                         ((0, 0, 1), (0, 0, 7)), ((1, 2, 3), (4, 5, 6))])
@pytest.mark.parametrize("n", [264, 261])
def test_strides_and_alignments(n, pads, shifts):
    """Any of them gives the bits of the dense, aligned tensors."""
    for m, k in ((290, 96), (3, 1024)):
        same = torch.equal(forward(m, n, k, "bf16", "gelu", pads=pads, shifts=shifts), forward(m, n, k, "bf16", "gelu"))
        assert same
        (dz, db), (dz0, db0) = backward(m, n, k, "f16", "gelu", pads=pads, shifts=shifts), backward(m, n, k, "f16", "gelu")
        assert torch.equal(dz, dz0)
        if k == 96 or n % 8:  # behind shared sums an aligned pass adds a row's columns in another order
            assert torch.equal(db[1:-1], db0[1:-1])


def test_no_contraction():
    """K = 0 leaves z = bias; M = 0 and N = 0 nothing, but the column sums of no rows are zero."""
    t, n = torch.bfloat16, 72
    x, w = torch.empty(5, 0, device="cuda", dtype=t), torch.empty(0, n, device="cuda", dtype=t)
    A, B = qf.qfmt_matrix_t(None, 5, 0, 0, 0), qf.qfmt_matrix_t(None, 0, n, n, 0)
    bias, y = randn(torch.Generator(device="cuda").manual_seed(1), n), torch.full((5, n), float("nan"), device="cuda", dtype=t)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    qf.qfmt_linear_act(A, B, qf.make_epilogue(code("gelu"), bias), y, n, t, ws, ws.numel())
    want = act64("gelu", bias.double()).expand(5, n)
    close(y, want, want.abs() * 2.0 ** -18 + half_step(want, t))
    db = torch.full((n,), float("nan"), device="cuda")
    A = qf.qfmt_matrix_t(None, 0, 8, 8, 0)
    B = qf.qfmt_matrix_t(w.data_ptr() or None, 8, n, n, 0)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(), None, n, db, t, ws, ws.numel())
    assert not db.any()


def test_in_place():
    gen = torch.Generator(device="cuda").manual_seed(3)
    for m, k in ((300, 128), (4, 2048)):
        n, t = 520, torch.bfloat16
        A, B, a64, b64, held = product(gen, m, n, k, t, False, False)
        ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
        r, z = randn(gen, m, n).to(t), randn(gen, m, n).to(t)
        y = torch.empty(m, n, device="cuda", dtype=t)
        qf.qfmt_linear_act(A, B, qf.make_epilogue(code("gelu"), None, r), y, n, t, ws, ws.numel())
        same = r.clone()
        qf.qfmt_linear_act(A, B, qf.make_epilogue(code("gelu"), None, same), same, n, t, ws, ws.numel())
        assert torch.equal(y, same)
        for alias in ("r", "z"):
            rr, zz = r.clone(), z.clone()
            qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code("gelu"), None, r, 0, z), y, n, None, t, ws, ws.numel())
            out = rr if alias == "r" else zz
            qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(code("gelu"), None, rr, 0, zz), out, n, None, t, ws, ws.numel())
            assert torch.equal(y, out)


def test_infinities_and_nan():
    """They travel as the formulas say: relu and the linear output keep them, what is too large for the codes becomes infinite."""
    t = torch.float16
    x = torch.zeros(300, 64, device="cuda", dtype=t)
    w = torch.zeros(64, 72, device="cuda", dtype=t)
    x[:, 0], w[0] = 1.0, 1.0
    x[7, 0], x[8, 0], x[9, 0], x[10, 0] = float("inf"), float("-inf"), float("nan"), 6e4
    w[0, 3] = 2.0
    A, B = qf.make_matrix(x), qf.make_matrix(w)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    for act in ("none", "relu", "gelu", "silu"):
        y = torch.empty(300, 72, device="cuda", dtype=t)
        qf.qfmt_linear_act(A, B, qf.make_epilogue(code(act)), y, 72, t, ws, ws.numel())
        assert bool(torch.isinf(y[7]).all()) and bool((y[7] > 0).all()) and bool(torch.isnan(y[9]).all())
        assert float(y[10, 0]) == 6e4 or act in ("gelu", "silu")
        assert bool(torch.isinf(y[10, 3])) and bool(torch.isfinite(y[11:]).all())
        if act == "relu":
            assert not y[8].any()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_activations_over_the_whole_range(act, dtype):
    """Slopes at every code (or many containers): dz of dy = 1."""
    t = TYPES[dtype]
    if dtype == "f32":
        z = torch.cat([torch.linspace(-30.0, 30.0, 1 << 16, device="cuda"), torch.logspace(-30, 30, 1 << 12, device="cuda"),
                       -torch.logspace(-30, 30, 1 << 12, device="cuda")])
    else:
        z = torch.arange(-(1 << 15), 1 << 15, device="cuda", dtype=torch.int32).to(torch.int16).view(t)
        z = z[torch.isfinite(z)]
    z = z[:z.numel() // 64 * 64].view(-1, 64)
    dy, dz = torch.ones_like(z), torch.empty_like(z)
    qf.qfmt_act_backward(dy, 64, z, 64, dz, 64, None, z.shape[0], 64, t, code(act))
    # differentiating tanh's form overflows where the slope has long been 0 or 1
    want = slope64(act, z.double().clamp(-100.0, 100.0))
    if act == "relu":
        want = (z > 0).double()
    # 64-bit: |slope| error 2^-18 (codes); containers: a few steps of the terms, which are at most 1.2 |z| exp(-z^2/2) in size, plus
    # the argument's own rounding, z^2 2^-24 of the term
    abs_err = 2.0 ** -18 if dtype != "f32" else 2.0 ** -20
    close(dz, want, abs_err + half_step(want, t))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu", "relu"])
@pytest.mark.parametrize("shape,pad,shift", [((1, 1), 0, 0), ((5, 7), 1, 1), ((64, 256), 0, 0), ((777, 1913), 3, 0), ((1000, 520), 8, 0),
                                             ((33, 264), 0, 3), ((4099, 72), 0, 0), ((3, 5000), 0, 0)])
def test_act_backward(shape, pad, shift, act, dtype):
    gen = torch.Generator(device="cuda").manual_seed(shape[1])
    t, (rows, cols) = TYPES[dtype], shape
    dy = placed(shape, t, pad, shift, randn(gen, *shape))[0]
    z = placed(shape, t, pad, shift, 2.0 * randn(gen, *shape))[0]
    dz, buf = placed(shape, t, pad, shift)
    db = torch.full((cols,), float("nan"), device="cuda")
    ws = workspace(qf.qfmt_act_backward_workspace_bytes(rows, cols))
    ld = cols + pad
    qf.qfmt_act_backward(dy, ld, None if act == "none" else z, ld, dz, ld, db, rows, cols, t, code(act), ws, ws.numel())
    slope = slope64(act, z.double()) if act != "none" else torch.ones(shape, device="cuda", dtype=torch.float64)
    want = dy.double() * slope
    bound = dy.double().abs() * (0.0 if act in ("none", "relu") else 2.0 ** -18 if dtype != "f32" else 2.0 ** -20)
    close(dz, want, bound + half_step(want, t))
    assert untouched(dz, buf)
    sums = bound.sum(dim=0) + want.abs().sum(dim=0) * (rows / 8 + 40) * 2.0 ** -24 + 1e-37
    close(db, want.sum(dim=0), sums)
    alone = torch.full((cols,), float("nan"), device="cuda")  # the sums without dz
    qf.qfmt_act_backward(dy, ld, None if act == "none" else z, ld, None, ld, alone, rows, cols, t, code(act), ws, ws.numel())
    assert torch.equal(alone, db)
    same = dy.clone()
    qf.qfmt_act_backward(same, cols, None if act == "none" else z, ld, same, cols, None, rows, cols, t, code(act))
    assert torch.equal(same, dz)


def test_act_backward_of_no_rows():
    db = torch.full((9,), float("nan"), device="cuda")
    qf.qfmt_act_backward(None, 9, None, 9, None, 9, db, 0, 9, torch.float32, qf.QFMT_ACT_NONE)
    assert not db.any()


def test_gradients_by_differences():
    """d loss / d x of two layers, y = act(x W1 + b) W2 + x, through the calls, against central differences of the plain form."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    m, d, f, t = 40, 64, 136, torch.float16
    x, w1, w2 = (v.to(t) for v in (randn(gen, m, d), randn(gen, d, f) * d ** -0.5, randn(gen, f, d) * f ** -0.5))
    b, dy = 0.1 * randn(gen, f), randn(gen, m, d).to(t)
    h, z, dz, dx = (torch.empty(m, n, device="cuda", dtype=t) for n in (f, f, f, d))
    y, db = torch.empty(m, d, device="cuda", dtype=t), torch.empty(f, device="cuda")
    mat = qf.make_matrix
    ws = workspace(max(qf.qfmt_linear_act_workspace_bytes(mat(x), mat(w1)), qf.qfmt_linear_act_workspace_bytes(mat(h), mat(w2)),
                       qf.qfmt_linear_act_workspace_bytes(mat(dy), mat(w2, True))))
    qf.qfmt_linear_act(mat(x), mat(w1), qf.make_epilogue(code("gelu"), b, None, 0, z), h, f, t, ws, ws.numel())
    qf.qfmt_linear_act(mat(h), mat(w2), qf.make_epilogue(code("none"), None, x), y, d, t, ws, ws.numel())
    qf.qfmt_linear_act_backward(mat(dy), mat(w2, True), qf.make_epilogue(code("gelu"), None, None, 0, z), dz, f, db, t, ws, ws.numel())
    qf.qfmt_linear_act_backward(mat(dz), mat(w1, True), qf.make_epilogue(code("none"), None, dy), dx, d, None, t, ws, ws.numel())

    def loss(x64, b64):
        return float(((act64("gelu", x64 @ w1.double() + b64) @ w2.double() + x64) * dy.double()).sum())

    x64, b64, eps = x.double(), b.double(), 2.0 ** -12
    for _ in range(4):
        # the codes on the way (h, z, dz) are off by half a step each: 2^-11 of terms whose sizes add up in squares
        v = torch.randn(m, d, generator=gen, device="cuda", dtype=torch.float64)
        slope = (loss(x64 + eps * v, b64) - loss(x64 - eps * v, b64)) / (2.0 * eps)
        size = float((dx.double() * v).square().sum().sqrt())
        assert abs(slope - float((dx.double() * v).sum())) < 16 * 2.0 ** -11 * size + 2.0 ** -10
        u = torch.randn(f, generator=gen, device="cuda", dtype=torch.float64)
        slope = (loss(x64, b64 + eps * u) - loss(x64, b64 - eps * u)) / (2.0 * eps)
        size = float((dz.double() * u).square().sum().sqrt())
        assert abs(slope - float((db.double() * u).sum())) < 16 * 2.0 ** -11 * size + 2.0 ** -10


def test_captured_and_replayed_on_a_side_stream():
    gen = torch.Generator(device="cuda").manual_seed(9)
    t, n = torch.bfloat16, 264
    A, B, a64, b64, (x, w) = product(gen, 5, n, 2048, t, False, False)
    ws = workspace(qf.qfmt_linear_act_workspace_bytes(A, B))
    y, z = torch.empty(5, n, device="cuda", dtype=t), torch.empty(5, n, device="cuda", dtype=t)
    e = qf.make_epilogue(code("silu"), None, None, 0, z)
    call = lambda: qf.qfmt_linear_act(A, B, e, y, n, t, ws, ws.numel())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    torch.cuda.synchronize()
    for _ in range(3):
        x.copy_(randn(gen, 5, 2048))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, y)
        assert qf.qfmt_device_status(ws) == qf.QFMT_OK


def test_less_workspace_gives_fewer_splits():
    gen = torch.Generator(device="cuda").manual_seed(2)
    t, m, n, k = torch.bfloat16, 9, 520, 4096
    A, B, a64, b64, held = product(gen, m, n, k, t, False, True)
    full = qf.qfmt_linear_act_workspace_bytes(A, B)
    want = a64 @ b64
    for size in (256, full // 2, full):
        ws, y = workspace(size), torch.empty(m, n, device="cuda", dtype=t)
        qf.qfmt_linear_act(A, B, qf.make_epilogue(), y, n, t, ws, size)
        close(y, want, sum_bound(a64, b64, k) + half_step(want.abs() * (1 + 2.0 ** -10), t))


@pytest.mark.parametrize("ta", [False, True])
@pytest.mark.parametrize("tb", [False, True])
@pytest.mark.parametrize("m", [1, 7, 8, 9, 16, 17, 31, 32, 33, 40, 100])
def test_few_rows(m, ta, tb):
    """Up to 32 rows the weights are walked in one launch, beyond that tiles share a long K."""
    for n, k in ((1000, 2056), (64, 16), (4099, 64), (15, 4100), (80, 9000)):
        if not (ta and m % 8):  # a transposed operand's rows are m long
            forward(m, n, k, "bf16" if m % 2 else "f16", "gelu", ta, tb, seed=m)
        backward(m, n, k, "f16" if m % 2 else "bf16", "silu", ta, tb, seed=m)


@pytest.mark.parametrize("act", ACTS)
def test_activations_behind_shared_sums(act):
    for n in (328, 325):
        forward(40, n, 2000, "bf16", act)
        backward(40, n, 2000, "f16", act)


def test_less_workspace_shares_less():
    gen = torch.Generator(device="cuda").manual_seed(2)
    t, m, n, k = torch.float16, 70, 520, 4096
    A, B, a64, b64, held = product(gen, m, n, k, t, False, True)
    full = qf.qfmt_linear_act_workspace_bytes(A, B)
    want = a64 @ b64
    for size in (256, full // 2, full):
        ws, y = workspace(size), torch.empty(m, n, device="cuda", dtype=t)
        qf.qfmt_linear_act(A, B, qf.make_epilogue(), y, n, t, ws, size)
        close(y, want, sum_bound(a64, b64, k) + half_step(want.abs() * (1 + 2.0 ** -10), t))
