"""Argument checks of the sub-layer output operators: everything is refused on the host before any device call (no GPU
needed)."""
import ctypes

import pytest

import paper_2103_15940_b200 as qf
from paper_2103_15940_b200 import build as qbuild

P, BAD, FMT = 0x10000, qf.QFMT_ERR_BAD_ARG, qf.QFMT_ERR_BAD_FORMAT


@pytest.fixture(scope="module", autouse=True)
def lib():
    qbuild.build()
    return qf.lib()


def status(call, *args, **kw):
    with pytest.raises(qf.QfmtError) as e:
        call(*args, stream=0, **kw)
    return e.value.status


NORM = dict(rows=4, cols=16, dtype=qf.QFMT_F32)


def forward(norm=None, x=P, w=P, b=P, y=P, mean=P, rstd=P, **kw):
    return status(qf.qfmt_layer_norm, qf.make_norm(**{**NORM, **(norm or {})}), x, w, b, y, mean, rstd, **kw)


def backward(norm=None, dy=P, x=P, mean=P, rstd=P, w=P, dx=P, dw=P, db=P, ws=P, size=1 << 30, **kw):
    return status(qf.qfmt_layer_norm_backward, qf.make_norm(**{**NORM, **(norm or {})}), dy, x, mean, rstd, w, dx, dw, db, ws, size, **kw)


def fused(norm=None, drop=None, x=P, r=P, h=P, y=P, **kw):
    return status(qf.qfmt_dropout_add_layer_norm, qf.make_norm(**{**NORM, **(norm or {})}), drop or qf.make_dropout(0.1, 1), x, r, P, P,
                  h, y, P, P, **kw)


def fused_backward(norm=None, drop=None, dy=P, dh=None, h=P, dx=P, dr=P + 0x1000, ws=P, size=1 << 30, **kw):
    return status(qf.qfmt_dropout_add_layer_norm_backward, qf.make_norm(**{**NORM, **(norm or {})}), drop or qf.make_dropout(0.1, 1), dy,
                  dh, h, P, P, P, dx, dr, P, P, ws, size, **kw)


CALLS = [forward, backward, fused, fused_backward]


def dropout(drop, x=P, ld_x=16, r=None, ld_r=0, out=P, ld_out=16, rows=4, cols=16, dtype=0):
    return status(qf.qfmt_dropout, x, ld_x, r, ld_r, out, ld_out, rows, cols, dtype, drop)


@pytest.mark.parametrize("p", [-0.1, 1.5, float("nan"), float("inf")])
def test_probability(p):
    assert dropout(qf.make_dropout(p, 1)) == BAD
    assert fused(drop=qf.make_dropout(p, 1)) == BAD and fused_backward(drop=qf.make_dropout(p, 1)) == BAD


def test_dropout_arguments():
    ok = qf.make_dropout(0.1, 1)
    assert dropout(None) == BAD
    assert dropout(qf.make_dropout(0.1, 1, 0, P + 4)) == BAD          # the offset's address
    for kw in (dict(x=None), dict(out=None), dict(x=P + 2), dict(out=P + 1), dict(r=P + 2, ld_r=16), dict(ld_x=15), dict(ld_out=8),
               dict(r=P, ld_r=15), dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31, ld_x=1 << 31, ld_out=1 << 31),
               dict(dtype=3), dict(dtype=-1), dict(x=P + 1, dtype=1), dict(out=P + 1, dtype=2)):
        assert dropout(ok, **kw) == BAD, kw


@pytest.mark.parametrize("call", CALLS)
def test_geometry(call):
    for norm in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31), dict(dtype=3), dict(dtype=-1), dict(eps=-1e-5),
                 dict(eps=float("nan")), dict(eps=float("inf")), dict(ld_x=15), dict(ld_residual=1), dict(ld_h=-16), dict(ld_y=15),
                 dict(ld_dy=15), dict(ld_dh=15), dict(ld_dx=15), dict(ld_dresidual=15)):
        assert call(norm) == BAD, norm


def test_null_and_misaligned_pointers():
    for kw in (dict(x=None), dict(y=None), dict(x=P + 2), dict(y=P + 1), dict(w=P + 2), dict(b=P + 1), dict(mean=P + 2), dict(rstd=P + 1)):
        assert forward(**kw) == BAD, kw
    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dy=P + 2), dict(x=P + 2), dict(dx=P + 2), dict(dw=P + 2),
               dict(db=P + 1), dict(w=P + 2), dict(ws=None), dict(ws=P + 8), dict(size=16), dict(size=0)):
        assert backward(**kw) == BAD, kw
    for kw in (dict(x=None), dict(y=None), dict(r=P + 2), dict(h=P + 1)):
        assert fused(**kw) == BAD, kw
    for kw in (dict(dy=None), dict(h=None), dict(dh=P + 2), dict(dx=P + 2), dict(dr=P + 2), dict(dx=P, dr=P), dict(ws=None), dict(size=0)):
        assert fused_backward(**kw) == BAD, kw
    lib = qf.lib()
    assert lib.qfmt_layer_norm(None, P, None, None, P, None, None, None, None, 0, None) == BAD
    assert lib.qfmt_layer_norm_workspace_bytes(None) == 0
    assert qf.qfmt_layer_norm_workspace_bytes(qf.make_norm(-1, 4, 0)) == 0


@pytest.mark.parametrize("call", CALLS)
def test_formats(call):
    for fmt in (qf.make_format(9, 9), qf.make_format(6, 24), qf.make_format(6, 9, loss_scale=2.0), qf.make_format(6, 9, denormals=2)):
        assert call(fmt=fmt) == FMT
    for dtype, fmt in ((qf.QFMT_F16, (6, 9)), (qf.QFMT_F16, (8, 7)), (qf.QFMT_BF16, (5, 10)), (qf.QFMT_BF16, (6, 9))):
        assert call(dict(dtype=dtype), fmt=qf.make_format(*fmt)) == FMT
    assert call(d_stats=P) == BAD                                       # statistics of no format
    assert call(fmt=qf.make_format(6, 9), d_stats=P + 4) == BAD
    assert call(fmt=qf.make_format(6, 9), d_stats=P, accumulate=2) == BAD


def test_statistics_of_a_gradient_that_is_not_wanted():
    assert backward(dx=None, fmt=qf.make_format(6, 9), d_stats=P) == BAD
    assert fused_backward(dx=None, fmt=qf.make_format(6, 9), d_stats=P) == BAD


def test_records():
    assert ctypes.sizeof(qf.qfmt_dropout_t) == 32 and ctypes.sizeof(qf.qfmt_norm_t) == 88
    with pytest.raises(KeyError):
        qf.make_norm(1, 1, "torch.float64")


def test_argument_types():
    """Addresses come as integers, tensors or None; anything else, or another number of arguments, is a TypeError."""
    norm = qf.make_norm(4, 16, qf.QFMT_F32)
    for bad in ("text", 1.5, b"bytes", [P]):
        with pytest.raises(TypeError):
            qf.qfmt_layer_norm(norm, bad, P, P, P, stream=0)
    with pytest.raises(TypeError):
        qf.qfmt_layer_norm("norm", P, P, P, P, stream=0)
    with pytest.raises(TypeError):
        qf._calls.dropout(P, 16)
    assert qf._calls.dropout(P, 16, None, 0, P, 16, 4, 16, 3, None, None) == BAD


def test_records_of_another_type_are_refused():
    """A call copies a record of the type it expects: a shorter one in its place would be read beyond its end."""
    norm, drop, fmt = qf.make_norm(4, 16, qf.QFMT_F32), qf.make_dropout(0.1, 1), qf.make_format(6, 9)
    for n, d, f in ((drop, drop, fmt), (norm, norm, fmt), (norm, drop, drop), (drop, norm, None), (fmt, drop, None), (norm, fmt, None),
                    (norm, drop, norm), (P, drop, None), (norm, P, None), (norm, drop, P)):
        with pytest.raises(TypeError):
            qf.qfmt_dropout_add_layer_norm(n, d, None, None, P, P, None, None, fmt=f, stream=0)
        with pytest.raises(TypeError):
            qf.qfmt_dropout_add_layer_norm_backward(n, d, None, None, None, P, P, P, None, None, P, P, None, 0, fmt=f, stream=0)
    for n, f in ((drop, fmt), (fmt, None), (norm, drop), (norm, norm)):
        with pytest.raises(TypeError):
            qf.qfmt_layer_norm(n, None, P, P, None, fmt=f, stream=0)
        with pytest.raises(TypeError):
            qf.qfmt_layer_norm_backward(n, None, None, P, P, P, None, P, P, None, 0, fmt=f, stream=0)
    for d in (norm, fmt, P):
        with pytest.raises(TypeError):
            qf.qfmt_dropout(None, 16, None, 0, None, 16, 4, 16, 0, d, stream=0)
    for n in (drop, fmt, P):
        with pytest.raises(TypeError):
            qf.qfmt_layer_norm_workspace_bytes(n)
    assert qf.qfmt_layer_norm_workspace_bytes(None) == 0


def test_tensors_pass_their_address():
    """A tensor stands for its data_ptr(): a misaligned one is refused as its address is."""
    import torch
    buf = torch.zeros(64, dtype=torch.uint8)
    odd = buf[1:] if buf.data_ptr() % 2 == 0 else buf
    assert odd.data_ptr() % 2 == 1
    assert forward(x=odd) == BAD == forward(x=odd.data_ptr())


@pytest.fixture
def seen(lib):
    """What the C side of qfmt_dropout and qfmt_layer_norm_backward is called with, instead of the library."""
    calls = []
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    dropout = ctypes.CFUNCTYPE(ctypes.c_int, vp, i64, vp, i64, vp, i64, i64, i64, ctypes.c_int32, vp, vp)(lambda *a: calls.append(a) or 0)
    backward = ctypes.CFUNCTYPE(ctypes.c_int, *[vp] * 11, ctypes.c_int, vp, ctypes.c_size_t, vp)(lambda *a: calls.append(a) or 0)
    fake = [ctypes.cast(f, vp).value for f in (dropout, backward)]
    qf._calls.bind(fake[0], 0, fake[1], 0, 0)
    yield calls
    qf._bind_calls(lib)


def test_sizes_are_numbers_and_never_addresses(seen):
    """Sizes convert as in the library's other calls (numpy integers, tensors of one integer); a tensor among them stands for
    its value, not for its address."""
    import numpy as np
    import torch
    drop, norm = qf.make_dropout(0.1, 1), qf.make_norm(4, 16, qf.QFMT_F32)
    one = torch.tensor
    for kind in (int, np.int64, np.uint32, one):
        qf.qfmt_dropout(P, kind(24), P, kind(32), P, kind(40), kind(3), kind(17), qf.QFMT_F16, drop, stream=0)
        assert seen.pop()[:9] == (P, 24, P, 32, P, 40, 3, 17, qf.QFMT_F16)
        qf.qfmt_layer_norm_backward(norm, P, P, P, P, P, P, P, P, P, kind(4096), accumulate=kind(1), stream=0)
        assert seen.pop()[11:14] == (1, P, 4096)
    for bad in (None, "8", 8.0, torch.zeros(2), torch.zeros(1)):
        with pytest.raises((TypeError, ValueError)):
            qf.qfmt_dropout(P, bad, None, 0, P, 16, 4, 16, 0, drop, stream=0)
        with pytest.raises((TypeError, ValueError)):
            qf.qfmt_layer_norm_backward(norm, P, P, P, P, P, P, P, P, P, bad, stream=0)
    assert not seen
