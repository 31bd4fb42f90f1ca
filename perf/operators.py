"""Cases of the sub-layer output operators: dropout, layer normalisation, and the two fused with the residual addition.

A transformer layer ends each of its two halves with y = LN(residual + D(x)): D drops elements of the product's output and
LN normalises every row.  The cases are the forward and backward passes of D, of LN and of the fused form, on fp32 containers
and on binary16 / bfloat16 codes, from a single token to 64 Mi elements, aligned and odd row lengths, dense rows and rows that
are a slice of wider ones.

``own`` selects the library's kernels; without it every pass is written in elementary torch operations in 32 bits, rounded
once at the end.

The mask.  Element (row, col) is dropped when its 16 random bits are below round(p * 65536).  They are bits
16 * (col % 8) ... of the 128-bit Philox4x32-10 block (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
1, 2, 3", SC 2011) with key = seed and counter words (col / 8, row, offset low, offset high).  What is kept is multiplied by
65536 / (65536 - round(p * 65536)).
"""
import numpy as np
import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
PHILOX_M = (0xD2511F53, 0xCD9E8D57)
PHILOX_W = (0x9E3779B9, 0xBB67AE85)
LOW32 = 0xFFFFFFFF

DROPOUT, NORM, NORM_BWD, SUBLAYER, SUBLAYER_BWD = "dropout", "norm", "norm_bwd", "sublayer", "sublayer_bwd"
OPS = (DROPOUT, NORM, NORM_BWD, SUBLAYER, SUBLAYER_BWD)


def _case(name, op, rows, cols, dtype, p=0.0, residual=False, pad=0):
    """``pad``: elements between the end of a row of the inputs and the start of the next one."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual, "pad": pad}


def listed():
    return [
        # one token's hidden vector: what a fine-tuning step on a single position pays for the launch
        _case("dropout one token f32", DROPOUT, 1, 1000, "f32", p=0.1),
        # the activation between the two feed-forward products of the BERT-large-shaped stack, on codes
        _case("dropout ffn bf16", DROPOUT, 8192, 4096, "bf16", p=0.1),
        # a residual branch of odd width cut out of a wider tensor
        _case("dropout add ragged f32", DROPOUT, 4099, 1021, "f32", p=0.25, residual=True, pad=3),
        # the normalisation of one token at inference
        _case("norm one token bf16", NORM, 1, 1024, "bf16"),
        # BERT-base-shaped layer (batch 32 x 128 tokens) on fp32 containers
        _case("norm base f32", NORM, 4096, 768, "f32"),
        # a long batch of wide rows, the largest tensor of the rounding sweep (64 Mi elements), on codes
        _case("norm wide bf16", NORM, 16384, 4096, "bf16"),
        # BERT-base-shaped layer's backward pass on binary16 codes
        _case("norm backward base f16", NORM_BWD, 4096, 768, "f16"),
        # few long rows of odd length
        _case("norm backward ragged f32", NORM_BWD, 331, 10007, "f32"),
        # the sub-layer output of the BERT-large-shaped stack (batch 16 x 512 tokens), forward on codes
        _case("sublayer large bf16", SUBLAYER, 8192, 1024, "bf16", p=0.1),
        # an odd batch of odd rows inside padded buffers
        _case("sublayer ragged f16", SUBLAYER, 777, 1913, "f16", p=0.1, pad=7),
        # the same sub-layer's backward pass on fp32 containers
        _case("sublayer backward large f32", SUBLAYER_BWD, 8192, 1024, "f32", p=0.1),
        # backward pass of wide rows on codes
        _case("sublayer backward wide bf16", SUBLAYER_BWD, 8192, 4096, "bf16", p=0.1),
    ]


def draw(rng):
    most = 1 << 25
    rows = int(round(2.0 ** rng.uniform(0, 16)))
    cols = int(round(2.0 ** rng.uniform(5, 14)))
    while rows * cols > most:
        rows = max(1, rows // 2)
    step = rng.choice((64, 64, 8, 1))  # widths are mostly round numbers; some are not
    cols = max(step, cols // step * step)
    op = rng.choice(OPS)
    return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(tuple(DTYPES)),
            "p": 0.0 if op in (NORM, NORM_BWD) else rng.choice((0.05, 0.1, 0.2, 0.5)),
            "residual": op == DROPOUT and rng.random() < 0.5, "pad": rng.choice((0, 0, 0, 8, 5))}


def work(case):
    n, size = case["rows"] * case["cols"], 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    tensors = {DROPOUT: 3 if case["residual"] else 2, NORM: 2, NORM_BWD: 3, SUBLAYER: 4, SUBLAYER_BWD: 4}[op]
    other = {DROPOUT: 0, NORM: 8 * (case["cols"] + case["rows"]), SUBLAYER: 8 * (case["cols"] + case["rows"]),
             NORM_BWD: 12 * case["cols"] + 8 * case["rows"], SUBLAYER_BWD: 12 * case["cols"] + 8 * case["rows"]}[op]
    flops = {DROPOUT: 2, NORM: 8, SUBLAYER: 10, NORM_BWD: 16, SUBLAYER_BWD: 18}[op]
    return {"bytes": n * size * tensors + other, "flops": n * flops}


def prepare(case, seed):
    rows, cols, pad, dtype = case["rows"], case["cols"], case["pad"], DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)

    def hold(t):
        wide = torch.zeros(rows, cols + pad, device="cuda", dtype=dtype)
        wide[:, :cols] = t
        return wide[:, :cols]

    def empty(kind=dtype):
        return torch.empty(rows, cols, device="cuda", dtype=kind)

    op = case["op"]
    s = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "p": case["p"], "seed": (seed * 0x9E3779B97F4A7C15 + 1) & (2 ** 62 - 1),
         "offset": 1 + seed % 1000}

    def activations():  # rows differ in size and centre, a few channels stand out
        t = randn(rows, cols) * torch.exp2(randn(rows, 1)) + 0.5 * randn(rows, 1)
        return t * (1.0 + 8.0 * (torch.rand(1, cols, generator=gen, device="cuda") < 0.01))

    if op != DROPOUT:
        s["weight"], s["bias"] = 1.0 + 0.1 * randn(cols), 0.1 * randn(cols)
    if op in (NORM_BWD, SUBLAYER_BWD):
        h = hold(activations())
        s["h"], s["dy"] = h, hold(randn(rows, cols) * 2.0 ** -4)
        s["mean"] = h.float().mean(dim=1)
        s["rstd"] = torch.rsqrt(h.float().var(dim=1, unbiased=False) + EPS)
        s["dx"] = empty()
        s["dweight"], s["dbias"] = torch.empty(2, cols, device="cuda").unbind(0)
        if op == SUBLAYER_BWD:
            s["dresidual"] = empty()
        return s
    s["x"] = hold(activations())
    if op == SUBLAYER or case["residual"]:
        s["residual"] = hold(randn(rows, cols))
    s["y"] = empty()
    if op != DROPOUT:
        s["mean"], s["rstd"] = torch.empty(2, rows, device="cuda").unbind(0)
    if op == SUBLAYER:
        s["h"] = empty()
    return s


# ---- the library's calls ----------------------------------------------------------------------------------------------


def _norm(qf, s):
    """The geometry a program sets up once for a layer."""
    if "norm" not in s:
        lds = {"ld_" + k: s[k].stride(0) for k in ("x", "residual", "dy") if k in s}  # everything else is dense
        if "dy" in s:
            lds["ld_x" if s["op"] == NORM_BWD else "ld_h"] = s["h"].stride(0)
        s["norm"] = qf.make_norm(s["rows"], s["cols"], s["dtype"], EPS, **lds)
        if s["op"] in (NORM_BWD, SUBLAYER_BWD):
            s["workspace"] = torch.empty(qf.qfmt_layer_norm_workspace_bytes(s["norm"]), dtype=torch.uint8, device="cuda")
    return s["norm"]


def _framework(s):
    import paper_2103_15940_b200 as qf
    op = s["op"]
    if op == DROPOUT:
        r = s.get("residual")
        qf.qfmt_dropout(s["x"], s["x"].stride(0), r, 0 if r is None else r.stride(0), s["y"], s["cols"], s["rows"], s["cols"],
                        s["dtype"], qf.make_dropout(s["p"], s["seed"], s["offset"]))
        return s["y"]
    norm = _norm(qf, s)
    if op == NORM:
        qf.qfmt_layer_norm(norm, s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if op == NORM_BWD:
        qf.qfmt_layer_norm_backward(norm, s["dy"], s["h"], s["mean"], s["rstd"], s["weight"], s["dx"], s["dweight"], s["dbias"],
                                    s["workspace"], s["workspace"].numel())
        return s["dx"], s["dweight"], s["dbias"]
    drop = qf.make_dropout(s["p"], s["seed"], s["offset"])
    if op == SUBLAYER:
        qf.qfmt_dropout_add_layer_norm(norm, drop, s["x"], s["residual"], s["weight"], s["bias"], s["h"], s["y"], s["mean"], s["rstd"])
        return s["y"], s["h"], s["mean"], s["rstd"]
    qf.qfmt_dropout_add_layer_norm_backward(norm, drop, s["dy"], None, s["h"], s["mean"], s["rstd"], s["weight"], s["dx"],
                                            s["dresidual"], s["dweight"], s["dbias"], s["workspace"], s["workspace"].numel())
    return s["dx"], s["dresidual"], s["dweight"], s["dbias"]


# ---- the plain forms --------------------------------------------------------------------------------------------------


def _threshold(p):
    return int(p * 65536.0 + 0.5)


def _keep(s):
    """The mask by the paper's rounds on int64 words (a product of two 32-bit words has the right bits modulo 2^64)."""
    rows, cols = s["rows"], s["cols"]
    groups = (cols + 7) // 8
    keys = torch.tensor([[((s["seed"] >> (32 * i)) + r * PHILOX_W[i]) & LOW32 for i in (0, 1)] for r in range(10)], device="cuda")
    mult = torch.tensor(PHILOX_M, device="cuda")[:, None, None]
    even, odd = torch.empty(2, 2, rows, groups, dtype=torch.int64, device="cuda").unbind(0)  # words 0 and 2, words 1 and 3
    even[0], even[1] = torch.arange(groups, device="cuda"), s["offset"] & LOW32
    odd[0], odd[1] = torch.arange(rows, device="cuda")[:, None], s["offset"] >> 32
    for key in keys[:, :, None, None].unbind(0):
        product = (even * mult).flip(0)
        even, odd = ((product >> 32) & LOW32) ^ odd ^ key, product & LOW32
    words = torch.stack((even[0], odd[0], even[1], odd[1]), dim=2)
    bits = torch.stack((words & 0xFFFF, words >> 16), dim=3).reshape(rows, groups * 8)[:, :cols]
    return bits >= _threshold(s["p"])


def _drop(s, t):
    return torch.where(_keep(s), t * (65536.0 / (65536 - _threshold(s["p"]))), torch.zeros_like(t))


def _plain_norm(s, h):
    mean = h.mean(dim=1)
    centred = h - mean[:, None]
    rstd = 1.0 / torch.sqrt((centred * centred).mean(dim=1) + EPS)
    return (centred * rstd[:, None] * s["weight"] + s["bias"]).to(s["dtype"]), mean, rstd


def _plain_norm_bwd(s):
    xhat = (s["h"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dh = s["rstd"][:, None] * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return dh, (dy * xhat).sum(dim=0), dy.sum(dim=0)


def _plain(s):
    op, dtype = s["op"], s["dtype"]
    if op == DROPOUT:
        y = _drop(s, s["x"].float())
        return (y + s["residual"].float() if "residual" in s else y).to(dtype)
    if op == NORM:
        return _plain_norm(s, s["x"].float())
    if op == SUBLAYER:
        h = s["residual"].float() + _drop(s, s["x"].float())
        y, mean, rstd = _plain_norm(s, h)
        return y, h.to(dtype), mean, rstd
    dh, dweight, dbias = _plain_norm_bwd(s)
    if op == NORM_BWD:
        return dh.to(dtype), dweight, dbias
    return _drop(s, dh).to(dtype), dh.to(dtype), dweight, dbias


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------


def _exact_keep(s):
    """The mask again, row block by row block on the host with unsigned 64-bit words."""
    rows, cols, groups = s["rows"], s["cols"], (s["cols"] + 7) // 8
    m32, out = np.uint64(LOW32), np.empty((rows, cols), dtype=bool)
    per = max(1, (1 << 18) // groups)
    for r0 in range(0, rows, per):
        r1 = min(rows, r0 + per)
        ctr = [np.broadcast_to(np.arange(groups, dtype=np.uint64), (r1 - r0, groups)),
               np.broadcast_to(np.arange(r0, r1, dtype=np.uint64)[:, None], (r1 - r0, groups)),
               np.full((r1 - r0, groups), s["offset"] & LOW32, dtype=np.uint64), np.full((r1 - r0, groups), s["offset"] >> 32, dtype=np.uint64)]
        for r in range(10):
            key = [np.uint64(((s["seed"] >> (32 * i)) + r * PHILOX_W[i]) & LOW32) for i in (0, 1)]
            p0, p1 = ctr[0] * np.uint64(PHILOX_M[0]), ctr[2] * np.uint64(PHILOX_M[1])
            ctr = [(p1 >> np.uint64(32)) ^ ctr[1] ^ key[0], p1 & m32, (p0 >> np.uint64(32)) ^ ctr[3] ^ key[1], p0 & m32]
        lanes = np.stack(ctr, axis=-1).astype("<u4").view("<u2").reshape(r1 - r0, groups * 8)
        out[r0:r1] = lanes[:, :cols] >= round(s["p"] * 65536)
    return torch.from_numpy(out).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    op, n = s["op"], s["cols"]
    d = {k: v.double() for k, v in s.items() if k in ("x", "residual", "weight", "bias", "dy", "mean", "rstd")
         or (k == "h" and op in (NORM_BWD, SUBLAYER_BWD))}
    keep = None
    if op in (DROPOUT, SUBLAYER, SUBLAYER_BWD):
        keep = _exact_keep(s).double() / (1.0 - round(s["p"] * 65536) / 65536)
    if op in (DROPOUT, NORM, SUBLAYER):
        h = d["x"] if keep is None else d["x"] * keep + d.get("residual", 0.0)
        if op == DROPOUT:
            return h
        mean = h.sum(dim=1) / n
        var = (h - mean[:, None]).square().sum(dim=1) / n
        y = (h - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * d["weight"] + d["bias"]
        rstd = (var + EPS) ** -0.5
        return (y, mean, rstd) if op == NORM else (y, h, mean, rstd)
    # dL/dh_j = sum_i dL/dxhat_i dxhat_i/dh_j with xhat_i = (h_i - mean) rstd, from the given mean and rstd
    xhat = (d["h"] - d["mean"][:, None]) * d["rstd"][:, None]
    gx = d["dy"] * d["weight"]
    dh = (gx - (gx.sum(dim=1, keepdim=True) + xhat * (gx * xhat).sum(dim=1, keepdim=True)) / n) * d["rstd"][:, None]
    dweight, dbias = torch.einsum("rc,rc->c", d["dy"], xhat), d["dy"].sum(dim=0)
    return (dh, dweight, dbias) if op == NORM_BWD else (dh * keep, dh, dweight, dbias)
