"""Products with an epilogue on every path they may take, each named by its test: a pass over the weights, tiles on single CTAs, tiles on
CTA pairs, and tiles whose K is shared with the epilogue in a pass of its own.  Against the formulas in 64 bits."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import workspace
from test_linear_act_gpu import code

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
