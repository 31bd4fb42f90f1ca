"""Plain 64-bit forms of the sub-layer output operators (dropout, layer normalisation, their fusion) for the tests:
the mask by unsigned integers, everything else in float64 on the CPU."""
import numpy as np
import torch

KINDS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a last place, relative
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # half the smallest denormal
U = 2.0 ** -24


def philox(c, k):
    """The 128-bit block of counter words c (four arrays of uint64 holding 32-bit values) under key words k."""
    c, k, low = list(c), list(k), np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return int(float(np.float32(p)) * 65536.0 + 0.5)


def keep_mask(rows, cols, p, seed, offset):
    groups = (cols + 7) // 8
    g, r = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    words = philox((g, r, np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.empty((rows, groups, 8), dtype=np.uint64)
    for j in range(4):
        bits[:, :, 2 * j], bits[:, :, 2 * j + 1] = words[j] & np.uint64(0xFFFF), words[j] >> np.uint64(16)
    return torch.from_numpy(bits.reshape(rows, groups * 8)[:, :cols] >= threshold(p))


def drop32(x, keep, p):
    """D(x) of a tensor of any storage type, in single precision: one multiplication, rounded, or zero."""
    t = threshold(p)
    scale = np.float32(65536.0 / (65536.0 - t)) if t < 65536 else np.float32(0)
    return torch.where(keep, x.float() * (torch.tensor(scale) if t else torch.tensor(np.float32(1))), torch.zeros(()))


def forward(h, weight, bias, eps):
    """y, mean, rstd of float64 rows, and a bound on a single-precision evaluation's error in y."""
    n = h.shape[1]
    mean = h.mean(dim=1, keepdim=True)
    var = ((h - mean) ** 2).mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xhat = (h - mean) * rstd
    y = xhat * weight + bias
    # a sum of n terms in a tree over threads of sequential pieces: at most k roundings on any path
    k = roundings(n)
    d_mean = (k + 1) * U * h.abs().mean(dim=1, keepdim=True)
    d_centred = d_mean + U * (h - mean).abs() + d_mean * U
    d_rel = 0.5 * ((k + 4) * U + 4.0 * d_mean * rstd) + 6 * U + (d_mean * rstd) ** 2   # of rstd
    tol = weight.abs() * (d_centred * rstd + xhat.abs() * (d_rel + 2 * U)) + 2 * U * (y.abs() + bias.abs())
    return y, mean[:, 0], rstd[:, 0], 1.01 * tol, d_mean[:, 0], (d_rel * rstd)[:, 0]


def roundings(n):
    """Roundings on one path of a sum over n columns: eight in a granule, one per further granule of a thread
    (32 threads at least share a row), five or ten in the tree, a few at the end."""
    return 8 * (1 + n // 4096) + 20 + 8 * 8


def backward(h, dy, mean, rstd, weight):
    """dh, dweight, dbias in float64 from the given mean and rstd, and bounds on single precision's errors."""
    rows, n = h.shape
    mean, rstd = mean[:, None], rstd[:, None]
    xhat = (h - mean) * rstd
    g = dy * weight
    c1, c2 = g.mean(dim=1, keepdim=True), (g * xhat).mean(dim=1, keepdim=True)
    dh = rstd * (g - c1 - xhat * c2)
    k = roundings(n)
    d_c1 = (k + 2) * U * g.abs().mean(dim=1, keepdim=True)
    d_c2 = (k + 6) * U * (g * xhat).abs().mean(dim=1, keepdim=True)
    tol = rstd * (d_c1 + xhat.abs() * d_c2 + 6 * U * (g.abs() + c1.abs() + (xhat * c2).abs()))
    kr = 8 + rows + 16 if rows < 256 else 256 + 24 + rows // 64     # rows a thread adds up, then the joins
    d_dw = (kr + 4) * U * (dy * xhat).abs().sum(dim=0)
    d_db = kr * U * dy.abs().sum(dim=0)
    return dh, (dy * xhat).sum(dim=0), dy.sum(dim=0), 1.01 * tol, 1.01 * d_dw, 1.01 * d_db


def close(got, ref, tol, kind="f32"):
    """Every element within tol plus the one rounding to its storage type; NaN and infinities in the same places."""
    got, ref = got.double().cpu(), ref.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    both = fine & torch.isfinite(got)
    assert torch.equal(fine, torch.isfinite(got))
    err = (got - ref).abs()[both]
    lim = (tol.expand_as(ref) + UNIT[kind] * (ref.abs() + tol) + TINY[kind])[both]
    if err.numel():
        worst = float((err / lim.clamp_min(1e-300)).max())
        assert worst <= 1.0, worst
