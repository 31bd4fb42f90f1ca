"""GPU tests of dropout, layer normalisation and the fused sub-layer output against plain 64-bit forms.

Masks and what dropout writes are exact (integers, one or two single-precision roundings, one rounding to the storage
type); normalised values and gradients stay within bounds on single-precision evaluation that sublayer_reference
derives from the lengths of the sums."""
import numpy as np
import pytest
import torch

import oracle
import paper_2103_15940_b200 as qf
import sublayer_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
SENTINEL = 77.0


class Buffer:
    """A rows x cols matrix inside a larger buffer: `off` elements before it, `pad` after every row, all of them marked."""

    def __init__(self, rows, cols, kind, off=0, pad=0, data=None):
        self.rows, self.cols, self.ld = rows, cols, cols + pad
        self.all = torch.full((off + rows * self.ld + 64,), SENTINEL, dtype=ref.KINDS[kind], device=DEV)
        self.off = off
        self.ptr = self.all.data_ptr() + off * self.all.element_size()
        self.view = self.all[off:off + rows * self.ld].view(rows, self.ld)[:, :cols]
        if data is not None:
            self.view.copy_(data)

    def get(self):
        rest = self.all.clone()
        rest[self.off:self.off + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = SENTINEL
        assert torch.all(rest == SENTINEL)  # nothing outside the matrix was written
        return self.view.cpu()


def values(gen, rows, cols, kind):
    t = torch.randn(rows, cols, generator=gen) * torch.exp2(torch.randn(rows, 1, generator=gen)) + torch.randn(rows, 1, generator=gen)
    return t.to(ref.KINDS[kind])


def vectors(gen, cols):
    return 1.0 + 0.25 * torch.randn(cols, generator=gen), 0.25 * torch.randn(cols, generator=gen)


def dtype_of(kind):
    return {"f32": qf.QFMT_F32, "f16": qf.QFMT_F16, "bf16": qf.QFMT_BF16}[kind]


SHAPES = [(1, 1), (5, 1), (3, 2), (7, 7), (4, 8), (9, 9), (33, 31), (17, 64), (130, 100), (2, 255), (40, 256), (19, 257),
          (300, 768), (77, 1000), (150, 1024), (5, 1913), (64, 2048), (700, 513), (31, 4096), (3, 5003), (20, 8192), (6, 8200),
          (4, 10007), (3, 16384), (2, 20001), (2, 65536), (2, 70001)]
LAYOUTS = [(0, 0), (0, 8), (8, 16), (1, 0), (3, 5), (4, 4)]


# ---- dropout ----------------------------------------------------------------------------------------------------------


def run_dropout(x, r, p, seed, offset, kind, off=0, pad=0, in_place=None, d_offset=None):
    rows, cols = x.shape
    bx = Buffer(rows, cols, kind, off, pad, x)
    br = Buffer(rows, cols, kind, off, 0 if pad else 3, r) if r is not None else None
    bo = {None: None, "x": bx, "r": br}[in_place] or Buffer(rows, cols, kind, off, pad)
    qf.qfmt_dropout(bx.ptr, bx.ld, br and br.ptr, br.ld if br else 0, bo.ptr, bo.ld, rows, cols, ref.KINDS[kind],
                    qf.make_dropout(p, seed, offset, d_offset))
    torch.cuda.synchronize()
    return bo.get()


def expect_dropout(x, r, p, seed, offset, kind):
    y = ref.drop32(x, ref.keep_mask(*x.shape, p, seed, offset), p)
    return (y if r is None else r.float() + y).to(ref.KINDS[kind])


def same_bits(got, want):
    w = torch.int32 if got.dtype == torch.float32 else torch.int16
    assert torch.equal(got.view(w), want.view(w))


def test_generator_gives_the_published_answers():
    """Philox4x32-10's known answers for an all-zero and an all-ones counter and key."""
    z, f = np.uint64(0), np.uint64(0xFFFFFFFF)
    assert [int(v) for v in ref.philox((z,) * 4, (0, 0))] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert [int(v) for v in ref.philox((f,) * 4, (0xFFFFFFFF,) * 2)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dropout_is_exact(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 131 + cols)
    x, r = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    seed, offset = 0x1234567890ABCDEF ^ cols, (rows << 33) + 5
    for i, (off, pad) in enumerate(LAYOUTS):
        p, res = (0.1, 0.5, 0.9)[i % 3], r if i % 2 else None
        same_bits(run_dropout(x, res, p, seed, offset, kind, off, pad), expect_dropout(x, res, p, seed, offset, kind))


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.25, 0.999999, 1.0])
def test_dropout_probabilities(kind, p):
    gen = torch.Generator().manual_seed(3)
    x, r = values(gen, 37, 203, kind), values(gen, 37, 203, kind)
    for res in (None, r):
        got = run_dropout(x, res, p, 9, 1 << 40, kind)
        same_bits(got, expect_dropout(x, res, p, 9, 1 << 40, kind))
        if p == 1.0:
            assert torch.equal(got, torch.zeros_like(x) if res is None else res)


@pytest.mark.parametrize("kind", ref.KINDS)
def test_dropped_infinities_and_nan_are_zero(kind):
    x = torch.full((64, 72), float("nan"), dtype=ref.KINDS[kind])
    x[:, ::2] = float("inf")
    keep = ref.keep_mask(64, 72, 0.5, 4, 2)
    got = run_dropout(x, None, 0.5, 4, 2, kind)
    assert torch.all(got[~keep] == 0) and torch.equal(torch.isnan(got), keep & torch.isnan(x))
    assert torch.equal(torch.isinf(got), keep & torch.isinf(x))


def test_mask_statistics_and_streams_of_the_generator():
    """The share of kept elements over 4 Mi draws, and no likeness between masks of neighbouring offsets, seeds, rows."""
    ones = torch.ones(2048, 2048)
    p, n = 0.1, 2048 * 2048
    a, b, c = (run_dropout(ones, None, p, s, o, "f32") != 0 for s, o in ((1, 1), (1, 2), (2, 1)))
    q = 1 - ref.threshold(p) / 65536
    five_sigma = 5 * (q * (1 - q) / n) ** 0.5
    for m in (a, b, c):
        assert abs(m.double().mean().item() - q) < five_sigma
    for u, v in ((a, b), (a, c), (a[:-1], a[1:]), (a[:, :-8], a[:, 8:]), (a[:, :-1], a[:, 1:])):
        both = (u & v).double().mean().item()
        assert abs(both - q * q) < 5 * (q * q / u.numel()) ** 0.5
    assert abs((ones * a).double().mean().item() / q - 1) < 2 * five_sigma


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("in_place", ["x", "r"])
def test_dropout_in_place(kind, in_place):
    gen = torch.Generator().manual_seed(5)
    x, r = values(gen, 50, 333, kind), values(gen, 50, 333, kind)
    same_bits(run_dropout(x, r, 0.3, 7, 8, kind, in_place=in_place), expect_dropout(x, r, 0.3, 7, 8, kind))


def test_dropout_is_its_own_backward_pass_and_linear():
    """<D(x), g> = <x, D(g)> element by element, and D(x + d) - D(x) = D(d) on values where nothing rounds."""
    gen = torch.Generator().manual_seed(6)
    x, d = (torch.randint(-64, 64, (40, 96), generator=gen).float() for _ in range(2))
    p = 0.5  # scale 2: exact
    D = lambda t: run_dropout(t, None, p, 11, 12, "f32")
    assert torch.equal(D(x + d) - D(x), D(d))
    assert torch.equal(D(x) * d, x * D(d))


def test_offset_kept_on_the_device_and_replayed_graphs():
    """d_offset is added when the kernel runs: a captured call draws another mask at every replay."""
    x = torch.ones(64, 512, device=DEV)
    out = torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = qf.make_dropout(0.5, 21, 100, step)
    call = lambda: qf.qfmt_dropout(x, 512, None, 0, out, 512, 64, 512, qf.QFMT_F32, drop)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        step.add_(1)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu() != 0, ref.keep_mask(64, 512, 0.5, 21, 100 + k))


# ---- layer normalisation ----------------------------------------------------------------------------------------------


def run_norm(x, w, b, kind, off=0, pad=0, eps=EPS, in_place=False, fmt=None, stats=None, accumulate=0, want=True):
    rows, cols = x.shape
    bx = Buffer(rows, cols, kind, off, pad, x)
    by = bx if in_place else Buffer(rows, cols, kind, off, pad)
    dw, db = (None if v is None else v.to(DEV) for v in (w, b))
    mean, rstd = (torch.full((rows + 1,), SENTINEL, device=DEV) for _ in range(2))
    qf.qfmt_layer_norm(qf.make_norm(rows, cols, ref.KINDS[kind], eps, ld_x=bx.ld, ld_y=by.ld), bx.ptr, dw, db, by.ptr,
                       mean if want else None, rstd if want else None, fmt, stats, accumulate)
    torch.cuda.synchronize()
    assert mean[-1] == SENTINEL and rstd[-1] == SENTINEL
    return by.get(), mean[:-1].cpu(), rstd[:-1].cpu()


def check_norm(got, h, w, b, kind, eps=EPS):
    w = torch.ones(h.shape[1]) if w is None else w
    b = torch.zeros(h.shape[1]) if b is None else b
    y, mean, rstd, tol, tol_m, tol_r = ref.forward(h.double(), w.double(), b.double(), eps)
    ref.close(got[0], y, tol, kind)
    ref.close(got[1], mean, tol_m)
    ref.close(got[2], rstd, tol_r)


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_forward(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 17 + cols)
    x = values(gen, rows, cols, kind)
    w, b = vectors(gen, cols)
    first = None
    for off, pad in LAYOUTS:
        got = run_norm(x, w, b, kind, off, pad)
        check_norm(got, x, w, b, kind)
        first = first or got
        for u, v in zip(first, got):  # the layout changes how rows are read, not what is computed
            assert torch.equal(u, v)


@pytest.mark.parametrize("kind", ref.KINDS)
def test_norm_without_weight_bias_or_statistics_and_in_place(kind):
    gen = torch.Generator().manual_seed(2)
    x = values(gen, 45, 333, kind)
    w, b = vectors(gen, 333)
    for ww, bb in ((None, None), (w, None), (None, b)):
        check_norm(run_norm(x, ww, bb, kind), x, ww, bb, kind)
    plain = run_norm(x, w, b, kind)
    assert torch.equal(run_norm(x, w, b, kind, want=False)[0], plain[0])
    assert torch.equal(run_norm(x, w, b, kind, in_place=True)[0], plain[0])
    assert torch.equal(run_norm(x, w, b, kind, in_place=True, off=3, pad=2)[0], plain[0])


@pytest.mark.parametrize("cols", [31, 253, 257, 389, 511, 515])
def test_places_of_one_warp_are_read_before_the_next_row_arrives(cols):
    """Ragged containers go through a place in shared memory that the next row takes over; teams of a warp or less (up to 512
    columns) have no block-wide barrier.  Many rows a team, against the aligned layout bit by bit."""
    gen = torch.Generator().manual_seed(cols)
    rows = 40000
    x, r = torch.randn(rows, cols, generator=gen), torch.randn(rows, cols, generator=gen)
    w, b = vectors(gen, cols)
    pad = -cols % 8
    aligned, fused = run_norm(x, w, b, "f32", 0, pad), run_fused(x, r, w, b, 0.1, 2, 3, "f32", 0, pad)
    for off, more in ((1, 0), (2, 1), (3, 2)):
        for got, want in ((run_norm(x, w, b, "f32", off, more), aligned), (run_fused(x, r, w, b, 0.1, 2, 3, "f32", off, more), fused)):
            for u, v in zip(got, want):
                assert torch.equal(u, v)


@pytest.mark.parametrize("cols", [64, 1000, 1024, 8200, 70001])
def test_large_centre_loses_nothing(cols):
    """Rows whose mean is 2^12 times their spread, and rows that begin with an outlier: the variance is taken about the mean."""
    gen = torch.Generator().manual_seed(cols)
    x = torch.randn(12, cols, generator=gen) * 0.25 + 1024.0
    x[6:] = torch.randn(6, cols, generator=gen)
    x[6:, 0] = 3.0e4
    w, b = vectors(gen, cols)
    check_norm(run_norm(x, w, b, "f32"), x, w, b, "f32")


def test_sums_of_very_long_rows():
    """Rows of 4 Mi equal columns, or equal gradients: whatever a thread adds up one after the other must not be lost in a growing
    sum.  At most 16 roundings on any path: three in a granule, nine in the tree over the block, the division, the rest for the
    conversion from a thread's own sum."""
    cols = (1 << 22) + 3
    gen = torch.Generator().manual_seed(1)
    x = torch.full((3, cols), 1.1)
    x[1] = -0.3
    x[2] = torch.randn(cols, generator=gen)
    w, b = torch.ones(cols), torch.zeros(cols)
    y, mean, rstd = run_norm(x, w, b, "f32")
    want = x.double().mean(dim=1)
    d_mean = 16 * ref.U * x.double().abs().mean(dim=1)
    assert torch.all((mean.double() - want).abs() <= d_mean)
    assert torch.all(y[:2].double().abs() <= (d_mean * EPS ** -0.5 * 1.01)[:2, None])
    dy = torch.full((3, cols), 0.3)
    dy[2] = x[2] * 0.7 + 0.1
    h = torch.stack((x[2], x[2].flip(0), x[2]))
    mean, rstd = saved(h)
    dx = run_norm_backward(h, dy, mean, rstd, w, "f32")[0].double()
    xhat = (h.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy.double()
    c1, c2 = g.mean(dim=1, keepdim=True), (g * xhat).mean(dim=1, keepdim=True)
    d_c1, d_c2 = 16 * ref.U * g.abs().mean(dim=1, keepdim=True), 20 * ref.U * (g * xhat).abs().mean(dim=1, keepdim=True)
    tol = rstd.double()[:, None] * (d_c1 + xhat.abs() * d_c2 + 6 * ref.U * (g.abs() + c1.abs() + (xhat * c2).abs()))
    assert torch.all((dx - rstd.double()[:, None] * (g - c1 - xhat * c2)).abs() <= 1.01 * tol)


def test_rows_that_do_not_vary_and_special_rows():
    x = torch.randn(6, 520, generator=torch.Generator().manual_seed(1))
    x[0], x[1] = 0.0, 3.0
    x[2, 5], x[3, 7], x[4, 511] = float("nan"), float("inf"), -float("inf")
    w, b = vectors(torch.Generator().manual_seed(1), 520)
    y, mean, rstd = run_norm(x, w, b, "f32")
    assert torch.equal(y[0], b) and torch.equal(y[1], b) and rstd[0] == pytest.approx(EPS ** -0.5, rel=1e-6)
    assert torch.all(torch.isnan(y[2:5])) and torch.isnan(mean[2]) and mean[3] == float("inf") and mean[4] == -float("inf")
    check_norm((y[5:], mean[5:], rstd[5:]), x[5:], w, b, "f32")
    y, _, rstd = run_norm(x[:1], w, b, "f32", eps=0.0)  # 0 * inf
    assert torch.all(torch.isnan(y)) and rstd[0] == float("inf")


def oracle_rounding(y32, e, m, den, kind):
    if kind == "f32":
        q, st = oracle.quantize_stats(y32.numpy(), e, m, den, 1.0)
        return torch.from_numpy(q), st
    codes, st = oracle.quantize_stats_pack16(y32.numpy(), e, m, den, 1.0)
    return torch.from_numpy(codes.view(np.int16).copy()).view(ref.KINDS[kind]).reshape(y32.shape), st


FORMATS = [("f32", 6, 9), ("f32", 5, 10), ("f32", 8, 7), ("f32", 4, 3), ("f16", 5, 10), ("bf16", 8, 7)]


@pytest.mark.parametrize("kind,e,m", FORMATS)
@pytest.mark.parametrize("den", [0, 1])
@pytest.mark.parametrize("rows,cols", [(37, 1000), (64, 1024), (5, 9), (2, 70001), (130, 64)])
def test_rounding_to_a_format_with_statistics(rows, cols, kind, e, m, den):
    """The rounded output and its counts are those of the oracle on the unrounded 32-bit result of the same rows."""
    gen = torch.Generator().manual_seed(rows + cols)
    x = values(gen, rows, cols, kind)
    w, b = vectors(gen, cols)
    w *= torch.exp2(12 * torch.randn(cols, generator=gen))   # denormals and overflows of the smaller formats
    b *= 2.0 ** -20
    b[::3] = 0.0
    w[::3] = 0.0
    y32 = run_norm(x.float(), w, b, "f32")[0]
    want, st = oracle_rounding(y32, e, m, den, kind)
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    for off, pad in ((0, 0), (3, 1)):
        got = run_norm(x, w, b, kind, off, pad, fmt=qf.make_format(e, m, den), stats=stats)[0]
        same_bits(got, want)
        assert np.array_equal(stats.cpu().numpy().view(np.uint64), st)
    run_norm(x, w, b, kind, fmt=qf.make_format(e, m, den), stats=stats, accumulate=1)
    assert np.array_equal(stats.cpu().numpy().view(np.uint64), 2 * st)
    same_bits(run_norm(x, w, b, kind, fmt=qf.make_format(e, m, den))[0], want)


def run_norm_backward(x, dy, mean, rstd, w, kind, off=0, pad=0, in_place=False, fmt=None, stats=None, want=(True, True, True),
                      ws_fill=0xFF):
    rows, cols = x.shape
    bx, bdy = Buffer(rows, cols, kind, off, pad, x), Buffer(rows, cols, kind, off, pad, dy)
    bdx = bdy if in_place else Buffer(rows, cols, kind, off, pad)
    norm = qf.make_norm(rows, cols, ref.KINDS[kind], EPS, ld_x=bx.ld, ld_dy=bdy.ld, ld_dx=bdx.ld)
    need = qf.qfmt_layer_norm_workspace_bytes(norm)
    ws = torch.full((need + 16,), ws_fill, dtype=torch.uint8, device=DEV)
    dw, db = (torch.full((cols + 1,), SENTINEL, device=DEV) for _ in range(2))
    qf.qfmt_layer_norm_backward(norm, bdy.ptr, bx.ptr, mean.to(DEV), rstd.to(DEV), None if w is None else w.to(DEV),
                                bdx.ptr if want[0] else None, dw if want[1] else None, db if want[2] else None, ws, need, fmt, stats)
    torch.cuda.synchronize()
    assert dw[-1] == SENTINEL and db[-1] == SENTINEL and torch.all(ws[need:] == ws_fill)
    return bdx.get(), dw[:-1].cpu(), db[:-1].cpu()


def saved(x):
    x = x.double()
    mean = x.mean(dim=1)
    return mean.float(), (1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(dim=1) + EPS)).float()


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", SHAPES + [(0, 100), (2500, 64), (5000, 9), (1300, 1024)])
def test_norm_backward(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    x, dy = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    mean, rstd = saved(x)
    w, _ = vectors(gen, cols)
    want = ref.backward(x.double(), dy.double(), mean.double(), rstd.double(), w.double())
    first = None
    for off, pad in LAYOUTS:
        got = run_norm_backward(x, dy, mean, rstd, w, kind, off, pad)
        ref.close(got[0], want[0], want[3], kind)
        ref.close(got[1], want[1], want[4])
        ref.close(got[2], want[2], want[5])
        first = first or got
        for u, v in zip(first, got):
            assert torch.equal(u, v)
    again = run_norm_backward(x, dy, mean, rstd, w, kind)  # nothing depends on the order of blocks
    for u, v in zip(first, again):
        assert torch.equal(u, v)


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(61, 513), (40, 1024), (3, 70001)])
def test_norm_backward_parts(rows, cols, kind):
    """Every output is optional, and none changes when another is left out; no weight; in place; rounded output."""
    gen = torch.Generator().manual_seed(8)
    x, dy = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    mean, rstd = saved(x)
    w, _ = vectors(gen, cols)
    full = run_norm_backward(x, dy, mean, rstd, w, kind)
    for want in ((True, False, False), (False, True, True), (True, True, False), (True, False, True), (False, False, True)):
        got = run_norm_backward(x, dy, mean, rstd, w, kind, want=want)
        for k in range(3):
            assert torch.equal(got[k], full[k] if want[k] else torch.full_like(full[k], SENTINEL))
    for u, v in zip(run_norm_backward(x, dy, mean, rstd, w, kind, in_place=True), full):
        assert torch.equal(u, v)
    ones = run_norm_backward(x, dy, mean, rstd, torch.ones(cols), kind)
    for u, v in zip(run_norm_backward(x, dy, mean, rstd, None, kind), ones):
        assert torch.equal(u, v)
    e, m = {"f32": (6, 9), "f16": (5, 10), "bf16": (8, 7)}[kind]
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    dx32 = run_norm_backward(x.float(), dy.float(), mean, rstd, w, "f32")[0]
    got = run_norm_backward(x, dy, mean, rstd, w, kind, fmt=qf.make_format(e, m), stats=stats)
    q, st = oracle_rounding(dx32, e, m, 1, kind)
    same_bits(got[0], q)
    assert np.array_equal(stats.cpu().numpy().view(np.uint64), st)
    assert torch.equal(got[1], full[1]) and torch.equal(got[2], full[2])


@pytest.mark.parametrize("kind,e,m", FORMATS)
@pytest.mark.parametrize("rows,cols", [(3, 8200), (5, 13001), (2, 16384)])
def test_rounded_gradients_of_wide_rows(rows, cols, kind, e, m):
    """Rows that take most of the shared memory, with the largest histograms beside them."""
    gen = torch.Generator().manual_seed(cols)
    x, dy = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    mean, rstd = saved(x)
    w, _ = vectors(gen, cols)
    want = ref.backward(x.double(), dy.double(), mean.double(), rstd.double(), w.double())
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    for off, pad in ((0, 0), (1, 3)):
        got = run_norm_backward(x, dy, mean, rstd, w, kind, off, pad, fmt=qf.make_format(e, m, 0), stats=stats)
        ref.close(got[1], want[1], want[4])
        ref.close(got[2], want[2], want[5])
        rounding = 2.0 ** -(m + 1) * want[0].abs() + 2.0 ** (2 - 2 ** (e - 1))   # half a last place, or flushed below 2^E_min
        fine = want[0].abs() < 2.0 ** (2 ** (e - 1) - 1)                        # below overflow
        err = (got[0].double() - want[0]).abs()
        assert torch.all((err <= want[3] * (1 + 2.0 ** -m) + rounding)[fine])
        st = stats.cpu()
        assert int(st[qf.ST_TOTAL]) == rows * cols == int(st[:256].sum())
    plain = run_norm_backward(x.float(), dy.float(), mean, rstd, w, "f32")[0]
    st = oracle_rounding(plain, e, m, 0, kind)[1]
    assert abs(int(st[qf.ST_DENORMAL]) - int(stats.cpu()[qf.ST_DENORMAL])) <= 2 + rows * cols // 1000


@pytest.mark.parametrize("kind,e,m", FORMATS)
@pytest.mark.parametrize("rows,cols", [(37, 1000), (5, 12289), (7, 13001), (300, 16384), (2, 20001)])
def test_gradients_do_not_depend_on_whether_statistics_are_wanted(rows, cols, kind, e, m):
    gen = torch.Generator().manual_seed(rows + cols)
    h, dy = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    mean, rstd = saved(h)
    w, _ = vectors(gen, cols)
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    fmt = qf.make_format(e, m, 0)
    plain = run_norm_backward(h, dy, mean, rstd, w, kind)
    full = run_fused_backward(h, dy, None, mean, rstd, w, 0.1, 1, 2, kind)
    for off, pad in ((0, 0), (3, 1)):
        got = [run_norm_backward(h, dy, mean, rstd, w, kind, off, pad, fmt=fmt, stats=s) for s in (None, stats)]
        for u, v, p in zip(*got, (None, *plain[1:])):
            assert torch.equal(u, v) and (p is None or torch.equal(u, p))
        got = [run_fused_backward(h, dy, None, mean, rstd, w, 0.1, 1, 2, kind, off, pad, fmt=fmt, stats=s) for s in (None, stats)]
        for u, v, p in zip(*got, (None, *full[1:])):
            assert torch.equal(u, v) and (p is None or torch.equal(u, p))
        assert int(stats[qf.ST_TOTAL]) == rows * cols


def test_norm_backward_against_differences():
    """The gradients against central differences of the 64-bit forward pass along random directions.  With step s the
    difference is off by O(s^2) = 1e-8 of the gradient's scale, single precision by less than 1e-5 of it."""
    gen = torch.Generator().manual_seed(13)
    rows, cols, s = 23, 333, 1e-4
    x, dy = torch.randn(rows, cols, generator=gen), torch.randn(rows, cols, generator=gen)
    w, b = vectors(gen, cols)
    mean, rstd = saved(x)
    dx, dw, db = (t.double() for t in run_norm_backward(x, dy, mean, rstd, w, "f32"))
    loss = lambda x, w, b: (ref.forward(x, w, b, EPS)[0] * dy.double()).sum()
    x, w, b = x.double(), w.double(), b.double()
    for k in range(8):
        d, dwdir, dbdir = (torch.randn(t.shape, generator=gen, dtype=torch.float64) for t in (x, w, b))
        for at, (u, v, z), grad in ((d, (1, 0, 0), dx), (dwdir, (0, 1, 0), dw), (dbdir, (0, 0, 1), db)):
            up = loss(x + s * u * d, w + s * v * dwdir, b + s * z * dbdir)
            dn = loss(x - s * u * d, w - s * v * dwdir, b - s * z * dbdir)
            scale = float((at.abs() * grad.abs()).sum())
            assert abs(float((up - dn) / (2 * s) - (at * grad).sum())) <= 1e-5 * scale


# ---- the fused form ---------------------------------------------------------------------------------------------------


def run_fused(x, r, w, b, p, seed, offset, kind, off=0, pad=0, h_in=None, y_in=None, fmt=None, stats=None, want_h=True, drop=True):
    rows, cols = x.shape
    bx = Buffer(rows, cols, kind, off, pad, x)
    br = Buffer(rows, cols, kind, off, pad, r) if r is not None else None
    pick = {None: None, "x": bx, "r": br}
    bh, by = pick[h_in] or Buffer(rows, cols, kind, off, pad), pick[y_in] or Buffer(rows, cols, kind, off, pad)
    mean, rstd = (torch.full((rows,), SENTINEL, device=DEV) for _ in range(2))
    norm = qf.make_norm(rows, cols, ref.KINDS[kind], EPS, ld_x=bx.ld, ld_residual=br.ld if br else 0, ld_h=bh.ld, ld_y=by.ld)
    qf.qfmt_dropout_add_layer_norm(norm, qf.make_dropout(p, seed, offset) if drop else None, bx.ptr, br and br.ptr, w.to(DEV),
                                   b.to(DEV), bh.ptr if want_h else None, by.ptr, mean, rstd, fmt, stats)
    torch.cuda.synchronize()
    return by.get(), mean.cpu(), rstd.cpu(), bh.get()


def h32(x, r, p, seed, offset):
    d = ref.drop32(x, ref.keep_mask(*x.shape, p, seed, offset), p)
    return d if r is None else r.float() + d


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_fused_forward(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 3 + cols)
    x, r = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    w, b = vectors(gen, cols)
    seed, offset = 99 + cols, (cols << 34) + rows
    h = h32(x, r, 0.1, seed, offset)
    first = None
    for off, pad in LAYOUTS:
        got = run_fused(x, r, w, b, 0.1, seed, offset, kind, off, pad)
        same_bits(got[3], h.to(ref.KINDS[kind]))
        check_norm(got[:3], h, w, b, kind)
        first = first or got
        for u, v in zip(first, got):
            assert torch.equal(u, v)


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(61, 513), (40, 1024), (3, 70001)])
def test_fused_forward_parts(rows, cols, kind):
    gen = torch.Generator().manual_seed(1)
    x, r = values(gen, rows, cols, kind), values(gen, rows, cols, kind)
    w, b = vectors(gen, cols)
    full = run_fused(x, r, w, b, 0.3, 5, 6, kind)
    assert torch.equal(run_fused(x, r, w, b, 0.3, 5, 6, kind, want_h=False)[0], full[0])
    for h_in, y_in in (("x", None), ("r", None), (None, "x"), (None, "r"), ("x", "r"), ("r", "x")):
        got = run_fused(x, r, w, b, 0.3, 5, 6, kind, h_in=h_in, y_in=y_in)
        assert torch.equal(got[0], full[0]) and torch.equal(got[3], full[3])
    for res in (r, None):   # no mask; everything dropped, which leaves rows of zeros when there is no residual
        h = x.float() if res is None else res.float() + x.float()
        for p, drop in ((0.3, False), (0.0, True)):
            got = run_fused(x, res, w, b, p, 5, 6, kind, drop=drop)
            same_bits(got[3], h.to(ref.KINDS[kind]))
            check_norm(got[:3], h, w, b, kind)
        got = run_fused(x, res, w, b, 1.0, 5, 6, kind)
        h = torch.zeros(rows, cols) if res is None else res.float()
        assert torch.equal(got[3].float(), h)
        check_norm(got[:3], h, w, b, kind)
    got = run_fused(x, None, w, b, 0.3, 5, 6, kind)
    check_norm(got[:3], h32(x, None, 0.3, 5, 6), w, b, kind)
    e, m = {"f32": (6, 9), "f16": (5, 10), "bf16": (8, 7)}[kind]
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    y32 = run_fused(x.float(), r.float(), w, b, 0.3, 5, 6, "f32")[0]
    got = run_fused(x, r, w, b, 0.3, 5, 6, kind, fmt=qf.make_format(e, m), stats=stats)
    q, st = oracle_rounding(y32, e, m, 1, kind)
    same_bits(got[0], q)
    assert torch.equal(got[3], full[3]) and np.array_equal(stats.cpu().numpy().view(np.uint64), st)


def test_special_values_in_dropped_places_do_not_reach_the_row():
    gen = torch.Generator().manual_seed(4)
    x, r = torch.randn(20, 264, generator=gen), torch.randn(20, 264, generator=gen)
    w, b = vectors(gen, 264)
    keep = ref.keep_mask(20, 264, 0.5, 1, 1)
    clean = run_fused(x, r, w, b, 0.5, 1, 1, "f32")
    x[~keep] = float("nan")
    x[:, ::3][~keep[:, ::3]] = float("inf")
    for u, v in zip(clean, run_fused(x, r, w, b, 0.5, 1, 1, "f32")):
        assert torch.equal(u, v)


def run_fused_backward(h, dy, dh, mean, rstd, w, p, seed, offset, kind, off=0, pad=0, dx_in=None, dr_in=None, fmt=None, stats=None,
                       want=(True, True, True, True), drop=True):
    rows, cols = h.shape
    bh, bdy = Buffer(rows, cols, kind, off, pad, h), Buffer(rows, cols, kind, off, pad, dy)
    bdh = Buffer(rows, cols, kind, off, pad, dh) if dh is not None else None
    pick = {None: None, "dy": bdy, "dh": bdh}
    bdx, bdr = pick[dx_in] or Buffer(rows, cols, kind, off, pad), pick[dr_in] or Buffer(rows, cols, kind, off, pad)
    norm = qf.make_norm(rows, cols, ref.KINDS[kind], EPS, ld_h=bh.ld, ld_dy=bdy.ld, ld_dh=bdh.ld if bdh else 0, ld_dx=bdx.ld,
                        ld_dresidual=bdr.ld)
    need = qf.qfmt_layer_norm_workspace_bytes(norm)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    dw, db = (torch.full((cols,), SENTINEL, device=DEV) for _ in range(2))
    qf.qfmt_dropout_add_layer_norm_backward(norm, qf.make_dropout(p, seed, offset) if drop else None, bdy.ptr, bdh and bdh.ptr, bh.ptr,
                                            mean.to(DEV), rstd.to(DEV), w.to(DEV), bdx.ptr if want[0] else None,
                                            bdr.ptr if want[1] else None, dw if want[2] else None, db if want[3] else None, ws, need,
                                            fmt, stats)
    torch.cuda.synchronize()
    return bdx.get(), bdr.get(), dw.cpu(), db.cpu()


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", SHAPES + [(0, 100), (1300, 1024)])
def test_fused_backward(rows, cols, kind):
    gen = torch.Generator().manual_seed(rows * 5 + cols)
    h, dy, dh = (values(gen, rows, cols, kind) for _ in range(3))
    mean, rstd = saved(h)
    w, _ = vectors(gen, cols)
    p, seed, offset = 0.1, 7 * cols, 1 + (rows << 35)
    g, dw, db, tol, tol_w, tol_b = ref.backward(h.double(), dy.double(), mean.double(), rstd.double(), w.double())
    keep = ref.keep_mask(rows, cols, p, seed, offset)
    scale = 65536 / (65536 - ref.threshold(p))
    first = None
    for i, (off, pad) in enumerate(LAYOUTS):
        more = dh if i % 2 else None
        total = g if more is None else g + dh.double()
        t = tol if more is None else tol + 2 * ref.U * (g.abs() + dh.double().abs())
        got = run_fused_backward(h, dy, more, mean, rstd, w, p, seed, offset, kind, off, pad)
        ref.close(got[1], total, t, kind)
        ref.close(got[0], torch.where(keep, total * scale, 0.0), (t + 2 * ref.U * total.abs()) * scale, kind)
        assert torch.all(got[0][~keep] == 0)
        ref.close(got[2], dw, tol_w)
        ref.close(got[3], db, tol_b)
        first = first or got
        if i % 2 == 0:
            assert torch.equal(first[0], got[0]) and torch.equal(first[1], got[1])
        assert torch.equal(first[2], got[2]) and torch.equal(first[3], got[3])


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(61, 513), (40, 1024), (3, 70001)])
def test_fused_backward_parts(rows, cols, kind):
    gen = torch.Generator().manual_seed(2)
    h, dy, dh = (values(gen, rows, cols, kind) for _ in range(3))
    mean, rstd = saved(h)
    w, _ = vectors(gen, cols)
    args = (mean, rstd, w, 0.3, 5, 6, kind)
    full = run_fused_backward(h, dy, dh, *args)
    for k in range(4):
        want = [True] * 4
        want[k] = False
        got = run_fused_backward(h, dy, dh, *args, want=want)
        for j in range(4):
            assert torch.equal(got[j], full[j] if j != k else torch.full_like(full[j], SENTINEL))
    for dx_in, dr_in in (("dy", None), ("dh", None), (None, "dy"), (None, "dh"), ("dy", "dh"), ("dh", "dy")):
        for u, v in zip(run_fused_backward(h, dy, dh, *args, dx_in=dx_in, dr_in=dr_in), full):
            assert torch.equal(u, v)
    plain = run_norm_backward(h, dy, mean, rstd, w, kind)
    got = run_fused_backward(h, dy, None, mean, rstd, w, 0.3, 5, 6, kind, drop=False)
    for u, v in zip(got, (plain[0], plain[0], plain[1], plain[2])):
        assert torch.equal(u, v)
    assert torch.all(run_fused_backward(h, dy, dh, mean, rstd, w, 1.0, 5, 6, kind)[0] == 0)
    e, m = {"f32": (6, 9), "f16": (5, 10), "bf16": (8, 7)}[kind]
    stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
    dx32 = run_fused_backward(h.float(), dy.float(), dh.float(), *args[:-1], "f32")[0]
    got = run_fused_backward(h, dy, dh, *args, fmt=qf.make_format(e, m), stats=stats)
    q, st = oracle_rounding(dx32, e, m, 1, kind)
    same_bits(got[0], q)
    assert torch.equal(got[1], full[1]) and np.array_equal(stats.cpu().numpy().view(np.uint64), st)


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(2367, 1283), (2368, 1281), (2500, 1533), (2400, 2048), (2368, 2560), (4735, 2056), (4736, 2049), (2375, 3071)])
def test_backward_of_several_teams_with_two_granules(rows, cols, kind):
    """Widths at which several teams of a block hold two granules a thread where there are enough rows."""
    test_norm_backward(rows, cols, kind)
    test_fused_backward(rows, cols, kind)


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(4740, 2049)])
def test_parts_of_several_teams_with_two_granules(rows, cols, kind):
    test_norm_backward_parts(rows, cols, kind)
    test_fused_backward_parts(rows, cols, kind)


@pytest.mark.parametrize("kind,e,m", FORMATS)
@pytest.mark.parametrize("rows,cols", [(2368, 1530), (4736, 2558)])
def test_rounded_gradients_of_several_teams_with_two_granules(rows, cols, kind, e, m):
    test_rounded_gradients_of_wide_rows(rows, cols, kind, e, m)


# ---- how large errors are on the whole --------------------------------------------------------------------------------


def rms(t):
    return float(t.double().square().mean().sqrt())


@pytest.mark.parametrize("rows,cols", [(4000, 64), (900, 203), (500, 768), (600, 1021), (300, 1024), (2400, 1283), (120, 4096), (70, 4093),
                                       (60, 8200), (40, 16384), (9, 70001)])
def test_errors_of_single_precision_are_those_of_a_few_roundings(rows, cols):
    """Root mean squares over whole tensors of ordinary rows, which the worst-case bounds above leave six bits for.

    One rounding is at most U of its result, U / sqrt(3) in the mean square, and they add up in squares.  y: three at full size (the
    difference, the two products) are U together, the inverse root's error is at most 2^-22.9 = 2.2 U, sums over a row that
    end near zero or are halved add less than U: below 4 U of |xhat w| + |b|.  dx: g, two products, the factor rstd: below 4 U of its three terms.
    Column sums: a chain of k roundings of a growing sum is U sqrt(k) / 2.4 of its final size; at most 8 rows a granule's owner ahead of
    5 parts of a warp's and 32 warps' (k < 64, 3.3 U), and the products: below 8 U of the terms' root sum of squares."""
    gen = torch.Generator().manual_seed(rows + 3 * cols)
    x, r, dy = (torch.randn(rows, cols, generator=gen) for _ in range(3))
    w, b = vectors(gen, cols)
    h = h32(x, r, 0.1, 3, 4)
    for got, t in ((run_norm(x, w, b, "f32"), x), (run_fused(x, r, w, b, 0.1, 3, 4, "f32"), h)):
        y, mean, rstd = ref.forward(t.double(), w.double(), b.double(), EPS)[:3]
        size = (t.double() - mean[:, None]) * rstd[:, None] * w.double()
        assert rms(got[0].double() - y) <= 4 * ref.U * rms(size.abs() + b.double().abs())
        assert rms(got[1].double() - mean) <= 4 * ref.U * rms(t) and rms(got[2].double() / rstd - 1) <= 4 * ref.U
    mean, rstd = saved(h)
    dh, dw, db = ref.backward(h.double(), dy.double(), mean.double(), rstd.double(), w.double())[:3]
    xhat, g = (h.double() - mean.double()[:, None]) * rstd.double()[:, None], dy.double() * w.double()
    size = rstd.double()[:, None] * (g.abs() + g.mean(1, keepdim=True).abs() + (xhat * (g * xhat).mean(1, keepdim=True)).abs())
    keep = ref.keep_mask(rows, cols, 0.1, 3, 4).double() * 65536 / (65536 - ref.threshold(0.1))
    one, two = run_norm_backward(h, dy, mean, rstd, w, "f32"), run_fused_backward(h, dy, None, mean, rstd, w, 0.1, 3, 4, "f32")
    for got, want in ((one[0], dh), (two[1], dh), (two[0], dh * keep)):
        assert rms(got.double() - want) <= 4 * ref.U * rms(size * (keep if want is not dh else 1.0))
    for dwk, dbk in ((one[1], one[2]), (two[2], two[3])):
        assert rms(dwk.double() - dw) <= 8 * ref.U * rms((dy.double() * xhat).square().sum(0).sqrt())
        assert rms(dbk.double() - db) <= 8 * ref.U * rms(dy.double().square().sum(0).sqrt())


# ---- tensors of one call that lie differently -----------------------------------------------------------------------------


MIXED = [((0, 0), (1, 1), (2, 3), (0, 0), (3, 0)), ((1, 2), (0, 0), (0, 0), (2, 1), (0, 0)), ((3, 1), (2, 1), (1, 0), (0, 8), (5, 2)),
         ((0, 8), (0, 0), (1, 0), (1, 0), (0, 16)), ((2, 5), (2, 3), (6, 1), (7, 0), (4, 4))]


def whole_rows(t):
    """Every tensor aligned: rows padded to whole granules."""
    return 0, -t.shape[1] % 8


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("rows,cols", [(3, 5), (70, 64), (41, 203), (50, 260), (300, 511), (33, 1024), (29, 1913), (2400, 1283), (9, 4093), (7, 8200),
                                       (5, 13001), (3, 20001)])
def test_every_tensor_has_its_own_alignment(rows, cols, kind):
    """Offsets and leading dimensions that differ from tensor to tensor of a call (aligned sources with ragged targets, two
    skews in one staged row) give the bits of the aligned layout."""
    gen = torch.Generator().manual_seed(rows * 11 + cols)
    dt, p, seed, offset = ref.KINDS[kind], 0.2, 17, 1 << 33
    x, r, dy, dh = (values(gen, rows, cols, kind) for _ in range(4))
    w, b = (t.to(DEV) for t in vectors(gen, cols))
    drop = qf.make_dropout(p, seed, offset)
    mean, rstd = (t.to(DEV) for t in saved(x))

    def passes(layout):
        """All outputs of every pass; layout: offset and padding of five tensors, inputs first."""
        put = lambda i, data=None: Buffer(rows, cols, kind, *layout[i], data)
        out = []
        bx, br, bo = put(0, x), put(1, r), put(3)
        qf.qfmt_dropout(bx.ptr, bx.ld, br.ptr, br.ld, bo.ptr, bo.ld, rows, cols, dt, drop)
        out += [bo.get(), bx.get(), br.get()]
        by, m, s = put(3), *torch.empty(2, rows, device=DEV).unbind(0)
        qf.qfmt_layer_norm(qf.make_norm(rows, cols, dt, EPS, ld_x=bx.ld, ld_y=by.ld), bx.ptr, w, b, by.ptr, m, s)
        out += [by.get(), m.cpu(), s.cpu()]
        bh, by = put(2), put(4)
        norm = qf.make_norm(rows, cols, dt, EPS, ld_x=bx.ld, ld_residual=br.ld, ld_h=bh.ld, ld_y=by.ld)
        qf.qfmt_dropout_add_layer_norm(norm, drop, bx.ptr, br.ptr, w, b, bh.ptr, by.ptr, m, s)
        out += [bh.get(), by.get(), m.cpu(), s.cpu()]
        bdy, bh, bdx = put(1, dy), put(0, x), put(3)
        norm = qf.make_norm(rows, cols, dt, EPS, ld_x=bh.ld, ld_dy=bdy.ld, ld_dx=bdx.ld)
        ws = torch.full((qf.qfmt_layer_norm_workspace_bytes(norm),), 0xFF, dtype=torch.uint8, device=DEV)
        dw, db = torch.empty(2, cols, device=DEV).unbind(0)
        qf.qfmt_layer_norm_backward(norm, bdy.ptr, bh.ptr, mean, rstd, w, bdx.ptr, dw, db, ws, ws.numel())
        out += [bdx.get(), dw.cpu(), db.cpu()]
        bdh, bdx, bdr = put(2, dh), put(3), put(4)
        norm = qf.make_norm(rows, cols, dt, EPS, ld_h=bh.ld, ld_dy=bdy.ld, ld_dh=bdh.ld, ld_dx=bdx.ld, ld_dresidual=bdr.ld)
        qf.qfmt_dropout_add_layer_norm_backward(norm, drop, bdy.ptr, bdh.ptr, bh.ptr, mean, rstd, w, bdx.ptr, bdr.ptr, dw, db, ws, ws.numel())
        return out + [bdx.get(), bdr.get(), dw.cpu(), db.cpu()]

    want = passes([whole_rows(x)] * 5)
    same_bits(want[0], expect_dropout(x, r, p, seed, offset, kind))
    for layout in MIXED:
        for u, v in zip(want, passes(layout)):
            assert torch.equal(u, v), layout


# ---- how calls sit in a program ---------------------------------------------------------------------------------------


def test_offsets_beyond_32_bits():
    """Three rows 2^30 + 8 codes apart: element offsets pass 2^31."""
    ld, rows, cols = (1 << 30) + 8, 3, 136
    wide = torch.empty(rows * ld, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator().manual_seed(3)
    x = values(gen, rows, cols, "bf16")
    w, b = vectors(gen, cols)
    view = wide.view(rows, ld)[:, :cols]
    view.copy_(x)
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    mean, rstd = torch.empty(2, rows, device=DEV).unbind(0)
    qf.qfmt_layer_norm(qf.make_norm(rows, cols, torch.bfloat16, EPS, ld_x=ld), wide, w.to(DEV), b.to(DEV), y, mean, rstd)
    check_norm((y.cpu(), mean.cpu(), rstd.cpu()), x, w, b, "bf16")
    qf.qfmt_dropout(wide, ld, None, 0, wide, ld, rows, cols, torch.bfloat16, qf.make_dropout(0.5, 1, 2))
    same_bits(view.cpu().contiguous(), expect_dropout(x, None, 0.5, 1, 2, "bf16"))
    norm = qf.make_norm(rows, cols, torch.bfloat16, EPS, ld_x=ld, ld_dx=ld)
    view.copy_(x)
    ws = torch.empty(qf.qfmt_layer_norm_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
    dw, db = torch.empty(2, cols, device=DEV).unbind(0)
    dy = values(gen, rows, cols, "bf16")
    mean, rstd = saved(x)
    dx = torch.empty_like(wide)
    qf.qfmt_layer_norm_backward(norm, dy.to(DEV), wide, mean.to(DEV), rstd.to(DEV), w.to(DEV), dx, dw, db, ws, ws.numel())
    want = ref.backward(x.double(), dy.double(), mean.double(), rstd.double(), w.double())
    ref.close(dx.view(rows, ld)[:, :cols].cpu(), want[0], want[3], "bf16")
    ref.close(dw, want[1], want[4])
    ref.close(db, want[2], want[5])


def test_column_sums_of_more_than_two_to_the_thirty_columns():
    """[dweight, dbias] side by side pass 2^31 places.  With one row dbias is dy and dweight is dy xhat, each rounding known."""
    cols = (1 << 30) + 8
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.empty(1, cols, dtype=torch.bfloat16, device=DEV).normal_(generator=gen) for _ in range(2))
    norm = qf.make_norm(1, cols, torch.bfloat16, EPS)
    ws = torch.empty(qf.qfmt_layer_norm_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
    grads = torch.full((2 * cols + 24,), SENTINEL, device=DEV)
    dw, db = grads[8:8 + cols], grads[16 + cols:16 + 2 * cols]
    mean, rstd = torch.tensor([0.25], device=DEV), torch.tensor([1.5], device=DEV)
    qf.qfmt_layer_norm_backward(norm, dy, x, mean, rstd, None, None, dw, db, ws, ws.numel())
    for i in range(0, cols, 1 << 28):
        part = slice(i, min(cols, i + (1 << 28)))
        assert torch.equal(db[part], dy[0, part].float())
        assert torch.equal(dw[part], dy[0, part].float() * ((x[0, part].float() - mean) * rstd))
    for edge in (grads[:8], grads[8 + cols:16 + cols], grads[16 + 2 * cols:]):
        assert torch.all(edge == SENTINEL)


def test_passes_over_a_row_of_more_than_two_to_the_thirty_columns():
    """Every pass over one row of 2^30 + 8 columns (byte offsets pass 2^31): results by chunks against 64 bits, masks against the
    generator at both ends and around 2^29 and 2^30."""
    cols, kind, p, seed, offset = (1 << 30) + 8, torch.bfloat16, 0.25, 5, 1 << 40
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, r = (torch.empty(cols, dtype=kind, device=DEV).normal_(generator=gen) for _ in range(2))
    h, y = torch.empty_like(x), torch.empty_like(x)
    drop = qf.make_dropout(p, seed, offset)
    scale = 65536 / (65536 - ref.threshold(p))

    def chunks(*tensors):
        for i in range(0, cols, 1 << 27):
            yield [t[i:i + (1 << 27)].double() for t in tensors]

    def near(got, want, extra):
        """Within one rounding to bfloat16 and `extra`."""
        return bool(torch.all((got - want).abs() <= ref.UNIT["bf16"] * (want.abs() + extra) + extra))

    def kept(i, n):
        """The mask of columns i .. i + n (i a multiple of 8)."""
        words = ref.philox((np.arange(i // 8, (i + n) // 8, dtype=np.uint64),) + tuple(np.full(n // 8, v, dtype=np.uint64)
                           for v in (0, offset & 0xFFFFFFFF, offset >> 32)), (seed, 0))
        bits = np.stack([v for w in words for v in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=1).reshape(-1)
        return torch.from_numpy(bits >= ref.threshold(p)).to(DEV)

    y.fill_(1.0)
    qf.qfmt_dropout(y, 0, None, 0, y, 0, 1, cols, kind, drop)
    mask = y != 0
    for i in (0, (1 << 29) - 64, (1 << 30) - 1024, cols - 4096):
        assert torch.equal(mask[i:i + 4096], kept(i, min(4096, cols - i)))
    qf.qfmt_dropout(x, 0, None, 0, y, 0, 1, cols, kind, drop)
    assert all(near(d, v * m * scale, 2.0 ** -20) for d, v, m in chunks(y, x, mask))
    norm = qf.make_norm(1, cols, kind, EPS)
    stat = torch.empty(2, device=DEV)
    qf.qfmt_dropout_add_layer_norm(norm, drop, x, r, None, None, h, y, stat[:1], stat[1:])
    total = square = 0.0
    for v, u, m in chunks(x, r, mask):
        t = u + v * m * scale
        total, square = total + float(t.sum()), square + float(t.square().sum())
    mean = total / cols
    rstd = (square / cols - mean * mean + EPS) ** -0.5
    assert abs(float(stat[0]) - mean) < 1e-6 and abs(float(stat[1]) / rstd - 1) < 1e-6
    for v, u, m, hh, yy in chunks(x, r, mask, h, y):
        t = u + v * m * scale
        assert near(hh, t, 2.0 ** -20) and near(yy, (t - mean) * rstd, 2.0 ** -18)
    qf.qfmt_layer_norm(norm, h, None, None, y, stat[:1], stat[1:])
    mean, rstd = float(stat[0]), float(stat[1])
    assert all(near(yy, (hh - mean) * rstd, 2.0 ** -18) for yy, hh in chunks(y, h))
    dy, dres = r, x                                            # the residual serves as a gradient; dresidual takes x's place
    c1 = c2 = 0.0
    for g, hh in chunks(dy, h):
        c1, c2 = c1 + float(g.sum()) / cols, c2 + float((g * (hh - mean)).sum()) * rstd / cols
    qf.qfmt_dropout_add_layer_norm_backward(norm, drop, dy, None, h, stat[:1], stat[1:], None, y, dres, None, None, None, 0)
    for g, hh, m, dx, dr in chunks(dy, h, mask, y, dres):
        want = rstd * (g - c1 - (hh - mean) * rstd * c2)
        assert near(dr, want, 2.0 ** -18) and near(dx, want * m * scale, 2.0 ** -17)


def test_column_sums_of_no_rows_of_the_widest_matrix():
    cols = (1 << 31) - 1
    norm = qf.make_norm(0, cols, torch.bfloat16, EPS)
    ws = torch.empty(qf.qfmt_layer_norm_workspace_bytes(norm), dtype=torch.uint8, device=DEV)
    grads = torch.full((2 * cols + 16,), SENTINEL, device=DEV)
    dw, db = grads[:cols], grads[8 + cols:8 + 2 * cols]
    qf.qfmt_layer_norm_backward(norm, None, None, None, None, None, None, dw, db, ws, ws.numel())
    for t in (dw, db):
        assert all(float(t[i:i + (1 << 28)].abs().max()) == 0.0 for i in range(0, cols, 1 << 28))
    assert torch.all(grads[cols:cols + 8] == SENTINEL) and torch.all(grads[8 + 2 * cols:] == SENTINEL)


def test_long_single_row_dropout():
    """A flat tensor as one row: granule numbers beyond 2^16."""
    n = (1 << 22) + 3
    x = torch.randn(1, n, generator=torch.Generator().manual_seed(1))
    same_bits(run_dropout(x, None, 0.1, 3, 4, "f32"), expect_dropout(x, None, 0.1, 3, 4, "f32"))


def test_another_stream_and_back_to_back_calls():
    """Calls on a side stream, one reading what the one before wrote, without a synchronisation in between."""
    gen = torch.Generator().manual_seed(9)
    rows, cols = 4096, 1024
    x, r = (values(gen, rows, cols, "f32").to(DEV) for _ in range(2))
    w, b = (t.to(DEV) for t in vectors(gen, cols))
    norm, drop = qf.make_norm(rows, cols, torch.float32, EPS), qf.make_dropout(0.1, 1, 1)
    ws = torch.empty(qf.qfmt_layer_norm_workspace_bytes(norm), dtype=torch.uint8, device=DEV)

    def chain(stream):
        h, y, dx, dr = (torch.empty(rows, cols, device=DEV) for _ in range(4))
        mean, rstd = torch.empty(2, rows, device=DEV).unbind(0)
        grads = torch.empty(3, 2, cols, device=DEV)
        cur = x
        torch.cuda.synchronize()
        for k in range(3):
            qf.qfmt_dropout_add_layer_norm(norm, drop, cur, r, w, b, h, y, mean, rstd, stream=stream)
            qf.qfmt_dropout_add_layer_norm_backward(norm, drop, y, None, h, mean, rstd, w, dx, dr, grads[k, 0], grads[k, 1], ws,
                                                    ws.numel(), stream=stream)
            qf.qfmt_dropout(dx, cols, dr, cols, y, cols, rows, cols, torch.float32, drop, stream=stream)
            cur = y.clone() if stream is None else y
        torch.cuda.synchronize()
        return [t.cpu() for t in (h, y, mean, rstd, dx, dr, grads)]

    side = torch.cuda.Stream()
    # the side stream's chain reads y while it is overwritten only in place, which is allowed
    for u, v in zip(chain(None), chain(side)):
        assert torch.equal(u, v)


def test_nothing_to_do():
    empty = torch.empty(0, device=DEV)
    drop = qf.make_dropout(0.5, 1)
    qf.qfmt_dropout(empty, 0, None, 0, empty, 0, 0, 8, torch.float32, drop)
    qf.qfmt_dropout(empty, 0, None, 0, empty, 0, 8, 0, torch.float32, drop)
    fmt = qf.make_format(6, 9)
    for rows, cols in ((0, 8), (8, 0)):
        stats = torch.full((qf.STATS_WORDS,), 5, dtype=torch.int64, device=DEV)
        qf.qfmt_layer_norm(qf.make_norm(rows, cols, torch.float32), empty, None, None, empty, None, None, fmt, stats)
        assert torch.all(stats == 0)
        stats.fill_(5)
        dw = torch.full((9,), SENTINEL, device=DEV)
        norm = qf.make_norm(rows, cols, torch.float32)
        ws = torch.empty(max(16, qf.qfmt_layer_norm_workspace_bytes(norm)), dtype=torch.uint8, device=DEV)
        qf.qfmt_layer_norm_backward(norm, empty, empty, empty, empty, None, empty, dw, None, ws, ws.numel(), fmt, stats)
        assert torch.all(stats == 0) and torch.all(dw[:cols] == 0) and torch.all(dw[cols:] == SENTINEL)
