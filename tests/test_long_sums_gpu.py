"""Products over a long K, on every path they may take.

A tensor core truncates each of its additions of 16 products, always towards zero, so a sum of one sign drifts by its length.  Sums are closed
after 8192 elements and the closed ones added up, rounded to nearest, so whatever K none is off by more than
(min(K, 8192) / 16 + K / 16384 + 24) 2^-23 of sum |a||b|, the last for the few additions around it."""
import pytest
import torch

import paper_2103_15940_b200 as qf
from step_reference import TYPES, close, half_step, workspace

pytestmark = pytest.mark.gpu


def ceil(a, b):
    return -(-a // b)


def limit_of(k):
    return (min(k, 8192) / 16 + k / 16384 + 24) * 2.0 ** -23


def one_sign(gen, rows, cols, t):
    return (0.5 + torch.rand(rows, cols, generator=gen, device="cuda")).to(t)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k,ta,tb,shared", [(130, 72, 1 << 17, False, False, False), (130, 72, 1 << 17, True, True, False),
                                                (70, 264, 100000, False, True, True), (300, 264, 65539, True, False, False),
                                                (3, 520, 1 << 17, False, True, True), (32, 100, 65536, False, True, True), (32, 100, 65544, False, True, True),
                                                (5, 72, 1 << 17, False, False, True), (2, 64, 32768, False, False, True), (2400, 2049, 20001, False, True, True),
                                                (130, 72, 8192, False, False, False), (130, 72, 8193, False, False, False)])
def test_sums_of_one_sign_over_a_long_contraction(m, n, k, ta, tb, shared, dtype):
    gen, t = torch.Generator(device="cuda").manual_seed(k), TYPES[dtype]
    pad = lambda v: (v + 7) // 8 * 8
    x = one_sign(gen, *((k, pad(m)) if ta else (m, pad(k))), t)[:, :m if ta else k]
    w = one_sign(gen, *((n, pad(k)) if tb else (k, pad(n))), t)[:, :k if tb else n]
    w.mul_(2.0 ** -8)  # sums stay within binary16
    A, B = qf.make_matrix(x, ta), qf.make_matrix(w, tb)
    full = qf.qfmt_linear_act_workspace_bytes(A, B)
    sums = max(ceil(m, 256) * 8, min(592 // ceil(n, 256), ceil(m, 8))) * pad(n) * 4  # the column sums' place, behind the status area
    ws = workspace(full if shared else 256 + sums)
    y, db = torch.empty(m, n, device="cuda", dtype=t), torch.empty(n, device="cuda")
    want = (x.t() if ta else x).double() @ (w.t() if tb else w).double()
    limit = limit_of(k)
    qf.qfmt_linear_act(A, B, qf.make_epilogue(), y, n, t, ws, ws.numel())
    close(y, want, want * limit + half_step(want * (1 + limit), t))
    qf.qfmt_linear_act_backward(A, B, qf.make_epilogue(), y, n, db, t, ws, ws.numel())
    close(y, want, want * limit + half_step(want * (1 + limit), t))
    total = want.sum(dim=0)
    close(db, total, total * (limit + (ceil(m, 256) + 40) * 2.0 ** -24))
    assert qf.qfmt_device_status(ws) == qf.QFMT_OK
