"""Global norm of a list of tensors and clipping, against 64 bits."""
import math

import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import TYPES, close, half_step, randn, workspace

pytestmark = pytest.mark.gpu


class List:
    def __init__(self, tensors, outs="new"):
        self.tensors = tensors
        self.outs = [torch.full_like(t, float("nan")) for t in tensors] if outs == "new" else outs
        host = qf.make_tensors(tensors, self.outs)
        self.count, self.chunks = len(tensors), qf.qfmt_plan_tensors(host, len(host)) if len(host) else 0
        self.records = torch.frombuffer(host, dtype=torch.uint8).cuda() if len(host) else None
        self.ws = workspace(qf.qfmt_grad_norm_workspace_bytes(self.count, self.chunks))
        self.norm = torch.full((2,), -1, dtype=torch.int64, device="cuda")

    def run(self, most, dls=None, stats=None, clip=True):
        qf.qfmt_grad_norm(self.records, self.count, self.chunks, most, dls, self.norm, stats, self.ws, self.ws.numel())
        if clip:
            qf.qfmt_grad_clip(self.records, self.count, self.chunks, self.norm)
        norm, factor = self.norm.view(torch.float32)[:2].tolist()
        return norm, factor, int(self.norm[1])


def dls(scale):
    t = torch.zeros(14, device="cuda")
    t[0] = scale
    return t


def check(tensors, most, scale=None):
    l = List(tensors)
    norm, factor, bad = l.run(most, None if scale is None else dls(scale))
    s = 1.0 if scale is None else scale
    want = math.sqrt(sum(float(t.double().square().sum()) for t in tensors)) / s
    # norm and factor are rounded to 32 bits once: half a step of the value, or of the denormals (2^-149 apart); a norm beyond the
    # largest 32-bit number is infinite
    assert bad == 0 and (abs(norm - want) <= want * 2.0 ** -23 + 2.0 ** -150 if want < 2.0 ** 128 else norm == math.inf)
    f = min(1.0, most / want) / s if want > 0 else 1.0 / s
    assert abs(factor - f) <= f * 2.0 ** -23 + 2.0 ** -150
    for t, o in zip(tensors, l.outs):
        y = t.double() * f
        close(o, y, y.abs() * 2.0 ** -23 + t.double().abs() * 2.0 ** -150 + half_step(y, t.dtype))
    return l


SIZES = [[1], [7], [8192], [8193], [1000003], [1, 0, 3, 0, 0, 70000, 5, 8192, 16384, 2], [0, 5], [5, 0], [129] * 700, [1 << 22, 1, 1 << 20]]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: str(s[:4]))
def test_norm_and_clipping(sizes, dtype):
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    tensors = [randn(gen, n).to(TYPES[dtype]) for n in sizes]
    check(tensors, 0.5)
    check(tensors, 1e6, 2.0 ** 9)
    check(tensors, float("inf"), 2.0 ** -3)


def test_mixed_types_and_alignments():
    gen = torch.Generator(device="cuda").manual_seed(1)
    tensors, outs = [], []
    for i, t in enumerate((torch.float32, torch.bfloat16, torch.float16) * 5):
        n = 5000 * i + i
        buf, out = torch.empty(n + 32, device="cuda", dtype=t), torch.full((n + 32,), float("nan"), device="cuda", dtype=t)
        tensors.append(buf[i:i + n])
        tensors[-1].copy_(randn(gen, n))
        outs.append(out[(3 * i) % 16:][:n])
    want = check(tensors, 1.0)
    got = List(tensors, outs)
    assert got.run(1.0) == want.run(1.0)
    for a, b in zip(got.outs, want.outs):
        assert torch.equal(a, b)
    for o in outs:  # nothing around them
        base = o._base
        assert int(torch.isnan(base).sum()) == base.numel() - o.numel()


@pytest.mark.parametrize("value", [1e-30, 1e-44, 1e25, 3e38])
def test_squares_beyond_32_bits(value):
    t = torch.full((5000,), value, device="cuda")
    check([t], 1.0)


def test_zeros():
    l = check([torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")], 1.0, 4.0)
    assert not l.outs[0].any()


def test_an_empty_list():
    l = List([])
    assert l.run(1.0) == (0.0, 1.0, 0)
    l = List([torch.zeros(0, device="cuda")])
    assert l.run(1.0, dls(2.0)) == (0.0, 0.5, 0)


def test_in_place_and_norm_only():
    gen = torch.Generator(device="cuda").manual_seed(4)
    t = [randn(gen, 9000), randn(gen, 77)]
    keep = [x.clone() for x in t]
    want = check(keep, 2.0)
    l = List(t, t)
    l.run(2.0)
    for a, b in zip(t, want.outs):
        assert torch.equal(a, b)
    l = List(keep, None if False else [None, None])
    l.run(2.0)
    assert all(torch.isfinite(x).all() for x in keep)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_infinities_and_nan(dtype):
    """The step is to be skipped: counts go to the controller, nothing is clipped."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    t = TYPES[dtype]
    tensors = [randn(gen, 20001).to(t), randn(gen, 300).to(t)]
    tensors[0][7], tensors[0][9000], tensors[1][299], tensors[1][0] = float("inf"), float("-inf"), float("nan"), float("inf")
    stats = torch.full((qf.STATS_WORDS,), 9, dtype=torch.int64, device="cuda")
    state = torch.zeros(7, dtype=torch.int64, device="cuda")
    rec = qf.qfmt_dls_t(2.0 ** 10, 2.0, 0.5, 1.0, 2.0 ** 20, 100, 5, 0, 0, 0, 0)
    state.copy_(torch.frombuffer(bytearray(bytes(rec)), dtype=torch.int64))
    l = List(tensors)
    norm, factor, bad = l.run(1.0, state, stats)
    assert not math.isfinite(norm) and factor == 1.0 and bad == 4
    for a, b in zip(tensors, l.outs):
        assert torch.equal(a.nan_to_num(1.5), b.nan_to_num(1.5))
    s = stats.cpu()
    assert int(s[qf.ST_TOTAL]) == 20301 and int(s[qf.ST_NAN]) == 1 and int(s[qf.ST_INF_IN]) == 3
    assert int(s.sum()) == 20301 + 4
    qf.qfmt_dls_update(state, stats, 1)
    after = qf.qfmt_dls_t.from_buffer_copy(state.cpu().numpy().tobytes())
    assert after.skip == 1 and after.scale == 2.0 ** 9
    tensors[0][7], tensors[0][9000], tensors[1][299], tensors[1][0] = 0.0, 0.0, 0.0, 0.0
    l.run(1.0, state, stats)
    qf.qfmt_dls_update(state, stats, 1)
    after = qf.qfmt_dls_t.from_buffer_copy(state.cpu().numpy().tobytes())
    assert after.skip == 0 and after.clean_steps == 1


def test_the_sum_repeats():
    gen = torch.Generator(device="cuda").manual_seed(8)
    tensors = [randn(gen, 300001) for _ in range(40)]
    l = List(tensors)
    first = l.run(1.0)
    assert all(l.run(1.0) == first for _ in range(5))


def test_captured():
    gen = torch.Generator(device="cuda").manual_seed(9)
    tensors = [randn(gen, 30000), randn(gen, 50).bfloat16()]
    l, state = List(tensors), dls(4.0)
    graph = torch.cuda.CUDAGraph()
    l.run(1.0, state)
    with torch.cuda.graph(graph):
        qf.qfmt_grad_norm(l.records, l.count, l.chunks, 1.0, state, l.norm, None, l.ws, l.ws.numel())
        qf.qfmt_grad_clip(l.records, l.count, l.chunks, l.norm)
    for scale in (1.0, 8.0):
        state[0] = scale
        tensors[0].mul_(3.0)
        graph.replay()
        got = [o.clone() for o in l.outs]
        l.run(1.0, state)
        for a, b in zip(got, l.outs):
            assert torch.equal(a, b)
