"""Plain forms in 64 bits, and the error bounds of the kernels, for products with an epilogue, cross entropy and clipping.

Bounds.  A product's 32-bit sum over K loses at most one unit in the last place, 2^-23 of sum |a||b|, per 16 products (the tensor
core truncates) and as much for each of the few additions around it: ``sum_bound``.  Activations and exponentials add relative
errors of at most 2^-18.  A result is rounded to its type once: half a step of its value (finfo.eps / 2), or of the smallest
denormal (``half_step``).
"""
import math

import torch

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def act64(act, z):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(act, z):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act64(act, z).sum(), z)[0]


def half_step(value, dtype):
    info = torch.finfo(dtype)
    return value.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def sum_bound(a, b, k):
    """a, b in 64 bits; additions of partial sums included (at most 16 splits)."""
    return (a.abs() @ b.abs()) * ((k / 16 + 24) * 2.0 ** -23)


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def operand(t, dtype, pad=0):
    """A matrix whose rows start on 16 bytes; NaN between the rows."""
    ld = (t.shape[1] + 7) // 8 * 8 + pad
    wide = torch.full((t.shape[0], ld), float("nan"), device="cuda", dtype=dtype)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def placed(shape, dtype, pad=0, shift=0, fill=None):
    """A rows x cols view `shift` elements into a buffer of NaN with `pad` elements between rows, and the buffer."""
    rows, cols = shape
    buf = torch.full((rows * (cols + pad) + shift + 16,), float("nan"), device="cuda", dtype=dtype)
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if fill is not None:
        view.copy_(fill)
    return view, buf


def untouched(view, buf):
    """Whether everything of the buffer around the view still is NaN."""
    outside = torch.ones(buf.numel(), dtype=torch.bool, device="cuda")
    outside.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool(torch.isnan(buf[outside]).all())


def close(got, want, bound):
    """Elementwise within the bound; infinities and NaN where they should be."""
    if got.dtype == torch.float16:
        # what is rounded beyond 65504 is infinite, from 65520 (half a step further) on; within the bound of that both are right
        edge = want.abs() + bound >= 65520.0
        over = edge & (torch.isinf(got) | (want.abs() - bound >= 65520.0))
        want = torch.where(over, torch.copysign(torch.full_like(want, math.inf), want), want)
    got, want, bound = got.double(), want.double(), bound.double()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN"
    assert torch.equal(got[~finite].nan_to_num(), want[~finite].nan_to_num()), "infinities"
    err, most = (got - want)[finite].abs(), bound.expand_as(want)[finite]
    worst = float((err / most.clamp(min=1e-300)).max()) if err.numel() else 0.0
    assert worst <= 1.0, "error %.3g of the bound" % worst


def workspace(n):
    return torch.full((max(256, n),), 0xA5, dtype=torch.uint8, device="cuda")
