"""Argument checks of products with an epilogue, cross entropy and clipping: everything is refused on the host before any device
call (no GPU needed)."""
import ctypes

import pytest

import paper_2103_15940_b200 as qf
from paper_2103_15940_b200 import build as qbuild

P, BAD = 0x10000, qf.QFMT_ERR_BAD_ARG
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return qf.lib()


def status(call, *args, **kw):
    with pytest.raises(qf.QfmtError) as e:
        call(*args, stream=0, **kw)
    return e.value.status


def matrix(rows, cols, ld=None, trans=0, ptr=P):
    return qf.qfmt_matrix_t(ptr, rows, cols, cols if ld is None else ld, trans)


def linear(A=None, B=None, e=None, y=P, ldy=24, dtype=qf.QFMT_BF16, ws=P, size=BIG):
    return status(qf.qfmt_linear_act, A or matrix(8, 16), B or matrix(16, 24), e or qf.make_epilogue(), y, ldy, dtype, ws, size)


def linear_backward(A=None, B=None, e=None, y=P, ldy=24, dtype=qf.QFMT_BF16, ws=P, size=BIG, db=P):
    return status(qf.qfmt_linear_act_backward, A or matrix(8, 16), B or matrix(16, 24), e or qf.make_epilogue(), y, ldy, db, dtype, ws, size)


@pytest.mark.parametrize("call", [linear, linear_backward])
def test_products(call):
    for kw in (dict(A=matrix(8, 15, 16)), dict(A=matrix(-1, 16)), dict(A=matrix(8, 16, 8)), dict(A=matrix(8, 16, 20)), dict(A=matrix(8, 16, ptr=P + 8)),
               dict(A=matrix(8, 16, ptr=None)), dict(B=matrix(16, 24, 16)), dict(B=matrix(16, 24, 28)), dict(B=matrix(16, 24, ptr=P + 2)),
               dict(B=matrix(16, 24, ptr=None)), dict(B=matrix(16, 24, trans=1)), dict(A=matrix(1 << 31, 16), ldy=24), dict(y=None), dict(y=P + 1),
               dict(ldy=23), dict(dtype=qf.QFMT_F32), dict(dtype=3), dict(ws=None), dict(ws=P + 8), dict(size=255),
               dict(e=qf.make_epilogue(5)), dict(e=qf.make_epilogue(-1)), dict(e=qf.make_epilogue(0, P + 2)), dict(e=qf.make_epilogue(0, None, P + 1)),
               dict(e=qf.make_epilogue(0, None, P, 23)), dict(e=qf.make_epilogue(0, None, None, 0, P + 1)), dict(e=qf.make_epilogue(0, None, None, 0, P, 8)),
               dict(A=matrix(1 << 30, 16), B=matrix(16, 1 << 30), ldy=1 << 30)):
        assert call(**kw) == BAD, kw


def test_backward_needs_z_and_room_for_its_sums():
    assert linear_backward(e=qf.make_epilogue(qf.QFMT_ACT_GELU)) == BAD
    assert linear_backward(db=P + 2) == BAD
    need = qf.qfmt_linear_act_workspace_bytes(matrix(8, 16), matrix(16, 24))
    assert linear_backward(size=need - 1) == BAD and need > 256


def test_workspaces_of_products():
    ws = qf.qfmt_linear_act_workspace_bytes
    assert ws(matrix(8, 16), matrix(17, 24)) == 0 and ws(matrix(-8, 16), matrix(16, 24)) == 0
    small, shared = ws(matrix(8192, 1024), matrix(1024, 4096)), ws(matrix(1, 4096), matrix(4096, 1024))
    assert 256 < small <= 256 + 8192 // 32 * 4096 * 4            # column sums of groups of 32 rows
    assert shared > 256 + 2 * 1024 * 4                           # and the parts of a shared K


def test_records_of_another_type_are_refused():
    a, b, e = matrix(8, 16), matrix(16, 24), qf.make_epilogue()
    for args in ((e, b, e), (a, e, e), (a, b, a), (P, b, e), (a, b, P)):
        with pytest.raises(TypeError):
            qf.qfmt_linear_act(*args, P, 24, qf.QFMT_F16, P, BIG, stream=0)
    kind = qf.make_cross_entropy(qf.QFMT_F16)
    for args in ((kind, b, kind), (a, kind, kind), (a, b, e)):
        with pytest.raises(TypeError):
            qf.qfmt_linear_cross_entropy(*args, None, P, P, P, None, P, BIG, stream=0)
    with pytest.raises(KeyError):
        qf.make_cross_entropy("torch.float64")
    assert ctypes.sizeof(qf.qfmt_epilogue_t) == 48 and ctypes.sizeof(qf.qfmt_cross_entropy_t) == 16
    assert ctypes.sizeof(qf.qfmt_tensor_t) == 40 and ctypes.sizeof(qf.qfmt_grad_norm_t) == 16


def act(dy=P, ld_dy=16, z=P, ld_z=16, dz=P, ld_dz=16, db=P, rows=4, cols=16, dtype=qf.QFMT_F32, act=qf.QFMT_ACT_GELU, ws=P, size=BIG):
    return status(qf.qfmt_act_backward, dy, ld_dy, z, ld_z, dz, ld_dz, db, rows, cols, dtype, act, ws, size)


def test_act_backward():
    for kw in (dict(dy=None), dict(z=None), dict(dy=P + 2), dict(z=P + 2), dict(dz=P + 2), dict(db=P + 2), dict(ld_dy=15), dict(ld_z=15), dict(ld_dz=-16),
               dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31, ld_dy=0, ld_z=0, ld_dz=0), dict(dtype=3), dict(act=5), dict(act=-1),
               dict(ws=None), dict(ws=P + 4), dict(size=0), dict(dtype=qf.QFMT_F16, dy=P + 1)):
        assert act(**kw) == BAD, kw
    assert qf.qfmt_act_backward_workspace_bytes(-1, 4) == 0 == qf.qfmt_act_backward_workspace_bytes(4, 1 << 31)


def loss(H=None, W=None, kind=None, bias=P, targets=P, loss=P, lse=P, mean=P, ws=P, size=BIG):
    return status(qf.qfmt_linear_cross_entropy, H or matrix(8, 16), W or matrix(100, 16, trans=1), kind or qf.make_cross_entropy(qf.QFMT_BF16), bias,
                  targets, loss, lse, mean, ws, size)


def loss_backward(H=None, W=None, kind=None, bias=P, targets=P, lse=P, dloss=P, dls=P, dh=P, ld_dh=16, dw=P, ld_dw=16, db=P, ws=P, size=BIG):
    return status(qf.qfmt_linear_cross_entropy_backward, H or matrix(8, 16), W or matrix(100, 16, trans=1), kind or qf.make_cross_entropy(qf.QFMT_BF16),
                  bias, targets, lse, dloss, dls, dh, ld_dh, dw, ld_dw, db, ws, size)


@pytest.mark.parametrize("call", [loss, loss_backward])
def test_cross_entropy(call):
    kind = qf.make_cross_entropy
    for kw in (dict(H=matrix(16, 8, trans=1)), dict(H=matrix(8, 16, ptr=None)), dict(H=matrix(8, 16, ptr=P + 8)), dict(H=matrix(8, 16, 20)),
               dict(H=matrix(8, 17, 24)), dict(H=matrix(-1, 16)), dict(H=matrix((1 << 24) + 1, 16)), dict(H=matrix(8, 0, 8), W=matrix(100, 0, 8, 1)),
               dict(W=matrix(100, 16, 8, 1)), dict(W=matrix(0, 16, trans=1)), dict(W=matrix(100, 16, ptr=None, trans=1)), dict(W=matrix(16, 100, 101)),
               dict(W=matrix(100, 16, ptr=P + 4, trans=1)), dict(W=matrix((1 << 28) + 1, 16, trans=1)), dict(kind=kind(qf.QFMT_F32)),
               dict(kind=qf.qfmt_cross_entropy_t(0, 7, 0)), dict(kind=qf.qfmt_cross_entropy_t(0, 1, 2)), dict(bias=P + 2), dict(targets=None),
               dict(targets=P + 4), dict(lse=P + 2), dict(ws=None), dict(ws=P + 8), dict(size=256)):
        assert call(**kw) == BAD, kw


def test_cross_entropy_outputs():
    assert loss(loss=P + 2) == BAD == loss(mean=P + 1)
    for kw in (dict(lse=None), dict(dloss=P + 2), dict(dls=P + 4), dict(dh=P + 1), dict(dw=P + 1), dict(db=P + 2), dict(ld_dh=15), dict(ld_dw=15)):
        assert loss_backward(**kw) == BAD, kw


def test_workspaces_of_the_loss():
    ws = qf.qfmt_linear_cross_entropy_workspace_bytes
    H, W = matrix(8192, 1024), matrix(30522, 1024, trans=1)
    forward, backward = ws(H, W, False), ws(H, W, True)
    logits = 8192 * 30522 * 4
    assert 0 < forward < logits // 16 and forward < backward < logits // 4  # neither holds the logits
    assert ws(H, matrix(30522, 1000, trans=1), False) == 0
    for fn, size in ((loss, forward), (loss_backward, backward)):
        kw = dict(ld_dh=1024, ld_dw=1024) if fn is loss_backward else {}
        assert fn(H=H, W=W, size=size - 1, **kw) == BAD


def tensors(*rows):
    a = (qf.qfmt_tensor_t * len(rows))()
    for r, (src, dst, n, dtype) in zip(a, rows):
        r.src, r.dst, r.n, r.dtype = src, dst, n, dtype
    return a


def test_lists():
    a = tensors((P, P, 8192, 0), (None, None, 0, 2), (P + 2, None, 8193, 1), (P, P, 1, 2))
    assert qf.qfmt_plan_tensors(a, 4) == 4 and [r.first_chunk for r in a] == [0, 1, 1, 3]
    for bad in ((None, P, 1, 0), (P + 2, P, 1, 0), (P, P + 2, 1, 0), (P + 1, P, 1, 1), (P, P + 1, 1, 2), (P, P, -1, 0), (P, P, 1, 3), (P, P, (1 << 46) + 1, 0)):
        with pytest.raises(qf.QfmtError):
            qf.qfmt_plan_tensors(tensors((P, P, 4, 0), bad), 2)
    lib = qf.lib()
    assert lib.qfmt_plan_tensors(None, 1) == BAD == lib.qfmt_plan_tensors(None, -1) and lib.qfmt_plan_tensors(None, 0) == 0


def norm(d=P, count=2, chunks=3, most=1.0, dls=P, out=P, stats=P, ws=P, size=BIG):
    return status(qf.qfmt_grad_norm, d, count, chunks, most, dls, out, stats, ws, size)


def test_norm_and_clipping():
    for kw in (dict(d=None), dict(d=P + 4), dict(count=-1), dict(chunks=-1), dict(count=0), dict(count=1 << 31), dict(most=0.0), dict(most=-1.0),
               dict(most=float("nan")), dict(dls=P + 4), dict(out=None), dict(out=P + 4), dict(stats=P + 4), dict(ws=None), dict(ws=P + 8), dict(size=0)):
        assert norm(**kw) == BAD, kw
    for kw in (dict(d_tensors=None), dict(count=-1), dict(d_norm=None), dict(d_norm=P + 4), dict(chunks=-2)):
        assert status(qf.qfmt_grad_clip, **{**dict(d_tensors=P, count=1, chunks=1, d_norm=P), **kw}) == BAD, kw


def test_lists_of_tensors():
    import torch
    a, b = torch.zeros(10), torch.zeros(4, 4, dtype=torch.bfloat16)
    rec = qf.make_tensors([a, b, torch.zeros(0)], [a, torch.empty_like(b), None])
    assert [r.n for r in rec] == [10, 16, 0] and rec[0].src == rec[0].dst == a.data_ptr() and rec[2].src is None
    assert [r.dtype for r in rec] == [qf.QFMT_F32, qf.QFMT_BF16, qf.QFMT_F32]
    for args in (([b.t()[:2]],), ([a], [b]), ([a], [a.double()]), ([a], [a[:5]]), ([a], [])):
        with pytest.raises(ValueError):
            qf.make_tensors(*args)
    with pytest.raises(KeyError):
        qf.make_tensors([a.double()])
