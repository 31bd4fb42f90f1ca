"""Cases of the operators around a training step's last products: a product with bias, activation and residual in its epilogue
and its backward pass, softmax cross entropy over a large vocabulary on top of the product that makes the logits, with its
gradients, and the global norm of all gradients with clipping.

Operands are binary16 / bfloat16 codes.  ``own`` selects the library's kernels; without it every pass is written in elementary
torch operations in 32 bits, rounded once at the end.

    linear       z = X W + bias,  y = act(z) + residual
    linear_bwd   dz = (dY W^T + add) act'(z),  dbias = column sums of dz
    act_bwd      the same where dY is there already
    ce           logits = H W + bias,  lse = log sum exp(logits),  loss = lse - logit of the target, 0 in rows that do not count
    ce_bwd       dlogits = g (exp(logits - lse) - onehot),  dH = dlogits W^T,  dW = H^T dlogits,  dbias = column sums of dlogits,
                 g = loss scale / number of rows that count
    clip         norm = |gradients / loss scale|,  every gradient times min(1, most / norm) / loss scale
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LINEAR, LINEAR_BWD, ACT_BWD, CE, CE_BWD, CLIP = "linear", "linear_bwd", "act_bwd", "ce", "ce_bwd", "clip"
OPS = (LINEAR, LINEAR_BWD, ACT_BWD, CE, CE_BWD, CLIP)
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
IGNORED = -100
MOST = 1.0  # the norm that gradients are clipped to


def _product(name, op, rows, k, n, dtype, act, trans, residual=False, keep=True):
    """``trans``: the weight is stored with its outputs as rows.  ``keep``: z is stored for the backward pass."""
    return {"name": name, "op": op, "rows": rows, "k": k, "n": n, "dtype": dtype, "act": act, "trans": trans, "residual": residual,
            "keep": keep}


def _act(name, rows, n, dtype, act, pad=0):
    return {"name": name, "op": ACT_BWD, "rows": rows, "n": n, "dtype": dtype, "act": act, "pad": pad}


def _loss(name, op, rows, hidden, vocab, dtype, trans, ignored=0.0, bias=True):
    """``ignored``: the part of the rows whose target does not count."""
    return {"name": name, "op": op, "rows": rows, "hidden": hidden, "vocab": vocab, "dtype": dtype, "trans": trans, "ignored": ignored,
            "bias": bias}


def _clip(name, layers, hidden, vocab, dtype):
    return {"name": name, "op": CLIP, "layers": layers, "hidden": hidden, "vocab": vocab, "dtype": dtype}


def listed():
    return [
        # one token through a layer's first feed-forward product, at inference
        _product("linear one token bf16", LINEAR, 1, 1024, 4096, "bf16", "gelu", True, keep=False),
        # the first feed-forward product of the BERT-large-shaped stack (batch 16 x 512 tokens), in training
        _product("linear large bf16", LINEAR, 8192, 1024, 4096, "bf16", "gelu", False),
        # an odd batch through layers of odd width, with the gradient of the residual path added
        _product("linear backward ragged f16", LINEAR_BWD, 777, 1913, 1001, "f16", "gelu_tanh", True, residual=True),
        # gradient of the second feed-forward product's input, through the activation
        _product("linear backward large bf16", LINEAR_BWD, 8192, 1024, 4096, "bf16", "gelu", False),
        # bias gradient of a product of odd width on fp32 containers
        _act("act backward ragged f32", 777, 1913, "f32", "none", pad=3),
        # an activation whose output's gradient comes from elsewhere
        _act("act backward large bf16", 8192, 4096, "bf16", "gelu"),
        # the loss of one token: what evaluating position by position pays
        _loss("ce one token f16", CE, 1, 1024, 30522, "f16", True),
        # masked language model: 15 % of the tokens count
        _loss("ce masked bf16", CE, 8192, 1024, 30522, "bf16", True, ignored=0.85),
        # a small odd vocabulary and an odd batch
        _loss("ce backward ragged f16", CE_BWD, 333, 520, 10007, "f16", False, ignored=0.1),
        # every token counts: the largest
        _loss("ce backward large bf16", CE_BWD, 8192, 1024, 30522, "bf16", True),
        # a small model of odd widths on fp32 containers
        _clip("clip odd f32", 3, 129, 1009, "f32"),
        # all gradients of a BERT-large-shaped model
        _clip("clip large bf16", 24, 1024, 30522, "bf16"),
    ]


def draw(rng):
    def size(lo, hi):  # mostly round numbers, some odd ones
        v = 2.0 ** rng.uniform(lo, hi)
        step = rng.choice((64, 8, 1))
        return max(1, int(v)) if v < 2 * step else int(v) // step * step

    op, dtype = rng.choice(OPS), rng.choice(("f16", "bf16"))
    if op in (LINEAR, LINEAR_BWD):
        rows, k, n = size(0, 13), size(5, 12), size(5, 12)
        while rows * k * n > 1 << 35:
            rows //= 2
        return {"op": op, "rows": rows, "k": k, "n": n, "dtype": dtype, "act": rng.choice(ACTS), "trans": rng.random() < 0.5,
                "residual": rng.random() < 0.5, "keep": rng.random() < 0.5}
    if op == ACT_BWD:
        return {"op": op, "rows": size(0, 13), "n": size(5, 12), "dtype": rng.choice(tuple(DTYPES)), "act": rng.choice(ACTS),
                "pad": rng.choice((0, 0, 8, 5))}
    if op == CLIP:
        return {"op": op, "layers": rng.randint(1, 24), "hidden": size(4, 10), "vocab": size(8, 15), "dtype": rng.choice(tuple(DTYPES))}
    rows, hidden, vocab = size(0, 13), size(5, 11), size(8, 17)
    while rows * vocab > 1 << 27 or rows * hidden * vocab > 1 << 37:
        rows //= 2
    return {"op": op, "rows": rows, "hidden": hidden, "vocab": vocab, "dtype": dtype, "trans": rng.random() < 0.5,
            "ignored": rng.choice((0.0, 0.0, 0.1, 0.85)), "bias": rng.random() < 0.5}


def _sizes(case):
    """Shapes of a model's gradients: four attention and two feed-forward products a layer, their biases, the norms, one embedding."""
    h = case["hidden"]
    layer = [(h, h), (h,)] * 4 + [(h, 4 * h), (4 * h,), (4 * h, h), (h,)] + [(h,)] * 4
    return [(case["vocab"], h)] + layer * case["layers"]


def _counted(case):
    return case["rows"] - round(case["rows"] * case["ignored"])


def work(case):
    op, size = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == CLIP:
        n = sum(math.prod(s) for s in _sizes(case))
        return {"bytes": 2 * n * size + 4, "flops": 3 * n}
    rows = case["rows"]
    if op in (LINEAR, LINEAR_BWD, ACT_BWD):
        n = case["n"]
        out = rows * n * size
        if op == ACT_BWD:
            tensors = 1 if case["act"] == "none" else 3  # without an activation only the column sums are new
            return {"bytes": out * tensors + 4 * n, "flops": rows * n}
        k = case["k"]
        tensors = 1 + case["residual"] + (case["keep"] if op == LINEAR else case["act"] != "none")
        return {"bytes": (rows * k + k * n) * size + out * tensors + 4 * n, "flops": 2 * rows * k * n}
    d, v, m = case["hidden"], case["vocab"], _counted(case)
    weight, tokens = v * d * size, m * d * size
    if op == CE:
        return {"bytes": weight + tokens + 4 * v * case["bias"] + 16 * rows, "flops": 2 * m * d * v}
    return {"bytes": 2 * weight + tokens + rows * d * size + 4 * v * (1 + case["bias"]) + 12 * rows, "flops": 6 * m * d * v}


def prepare(case, seed):
    op, dtype = case["op"], DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)

    def operand(t, pad=None):  # rows of an operand start on 16 bytes
        pad = -t.shape[1] % 8 if pad is None else pad
        wide = torch.zeros(t.shape[0], t.shape[1] + pad, device="cuda", dtype=dtype)
        wide[:, :t.shape[1]] = t
        return wide[:, :t.shape[1]]

    def empty(*shape, kind=dtype):
        return torch.empty(*shape, device="cuda", dtype=kind)

    s = {k: v for k, v in case.items() if k != "name"}
    s["type"] = dtype
    # a loss scale as a step in progress holds it: the record's first word, the rest is the controller's
    s["dls"] = torch.zeros(14, device="cuda", dtype=torch.float32)
    s["dls"][0] = 2.0 ** 10
    if op == CLIP:
        shapes = _sizes(case)
        total = sum(math.prod(v) for v in shapes)
        s["flat"], s["out"] = empty(total), empty(total)  # the gradients lie in one buffer, as buckets of a reduction do
        flat = s["flat"]
        for at in range(0, total, 1 << 26):
            part = flat[at:at + (1 << 26)]
            part.copy_(randn(part.numel()))
        s["grads"], s["outs"], at = [], [], 0
        for v in shapes:
            n = math.prod(v)
            s["grads"].append(flat[at:at + n].view(v))
            s["grads"][-1].mul_(2.0 ** 10 * 2.0 ** float(-6 - 4 * (len(v) > 1)))  # matrices have the smaller gradients
            s["outs"].append(s["out"][at:at + n].view(v))
            at += n
        s["record"] = torch.zeros(2, dtype=torch.int64, device="cuda")
        return s
    rows = case["rows"]
    if op in (LINEAR, LINEAR_BWD, ACT_BWD):
        n, pad = case["n"], case.get("pad", 0)
        if op != ACT_BWD:
            k = case["k"]
            grad = 1.0 if op == LINEAR else 2.0 ** -4
            s["x"] = operand(randn(rows, k) * grad * (1.0 + 8.0 * (torch.rand(1, k, generator=gen, device="cuda") < 0.01)))
            w = randn(k, n) * k ** -0.5
            s["w"] = operand(w.t() if case["trans"] else w)
        if op == LINEAR:
            s["bias"] = 0.1 * randn(n)
            s["y"], s["z"] = empty(rows, n), empty(rows, n) if case["keep"] else None
        else:
            s["z"] = None if case["act"] == "none" else operand(randn(rows, n) * 1.5, pad)
            s["dbias"] = empty(n, kind=torch.float32)
            if op == ACT_BWD:
                s["dy"] = operand(randn(rows, n) * 2.0 ** -4, pad)
                s["dz"] = None if case["act"] == "none" else empty(rows, n)
            else:
                s["dz"] = empty(rows, n)
        s["extra"] = operand(randn(rows, n) * (1.0 if op == LINEAR else 2.0 ** -4)) if case.get("residual") else None
        return s
    d, v = case["hidden"], case["vocab"]
    s["h"] = operand(randn(rows, d))
    w = randn(v, d) * (2.0 * d ** -0.5)  # logits of standard deviation two
    s["w"] = operand(w if case["trans"] else w.t())
    s["bias"] = randn(v) if case["bias"] else None
    # few words make up most of a text
    s["targets"] = (v * torch.rand(rows, generator=gen, device="cuda") ** 3).long().clamp_(max=v - 1)
    s["targets"][torch.randperm(rows, generator=gen, device="cuda")[:rows - _counted(case)]] = IGNORED
    if op == CE:
        s["loss"], s["lse"] = empty(2, rows, kind=torch.float32).unbind(0)
        s["mean"] = empty(1, kind=torch.float32)
    else:
        s["lse"] = _plain_logits(s).logsumexp(dim=1) * (s["targets"] != IGNORED)
        s["dh"], s["dw"], s["dbias"] = empty(rows, d), empty(*s["w"].shape), empty(v, kind=torch.float32)
    return s


# ---- the library's calls ----------------------------------------------------------------------------------------------


def _setup(qf, s):
    """What a program sets up once for a layer: descriptors, and a workspace of the recommended size."""
    op, act = s["op"], getattr(qf, "QFMT_ACT_" + s.get("act", "none").upper())
    if op == CLIP:
        host = qf.make_tensors(s["grads"], s["outs"])
        s["chunks"] = qf.qfmt_plan_tensors(host, len(host))
        s["tensors"], s["count"] = torch.frombuffer(host, dtype=torch.uint8).cuda(), len(host)
        need = qf.qfmt_grad_norm_workspace_bytes(s["count"], s["chunks"])
    elif op == ACT_BWD:
        s["act_code"] = act
        need = qf.qfmt_act_backward_workspace_bytes(s["rows"], s["n"])
    elif op in (LINEAR, LINEAR_BWD):
        s["a"] = qf.make_matrix(s["x"])
        s["b"] = qf.make_matrix(s["w"], s["trans"])
        extra, z = s["extra"], s["z"]
        s["epilogue"] = qf.make_epilogue(act, s.get("bias"), extra, 0 if extra is None else extra.stride(0), z, 0 if z is None else z.stride(0))
        need = qf.qfmt_linear_act_workspace_bytes(s["a"], s["b"])
    else:
        s["a"], s["b"] = qf.make_matrix(s["h"]), qf.make_matrix(s["w"], s["trans"])
        s["kind"] = qf.make_cross_entropy(s["type"], IGNORED, mean=True)
        need = qf.qfmt_linear_cross_entropy_workspace_bytes(s["a"], s["b"], op == CE_BWD)
    s["workspace"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")


def _framework(s):
    import paper_2103_15940_b200 as qf
    if "workspace" not in s:
        _setup(qf, s)
    op, ws = s["op"], s["workspace"]
    if op == LINEAR:
        qf.qfmt_linear_act(s["a"], s["b"], s["epilogue"], s["y"], s["n"], s["type"], ws, ws.numel())
        return (s["y"], s["z"]) if s["keep"] else s["y"]
    if op == LINEAR_BWD:
        qf.qfmt_linear_act_backward(s["a"], s["b"], s["epilogue"], s["dz"], s["n"], s["dbias"], s["type"], ws, ws.numel())
        return s["dz"], s["dbias"]
    if op == ACT_BWD:
        z, dy = s["z"], s["dy"]
        qf.qfmt_act_backward(dy, dy.stride(0), z, 0 if z is None else z.stride(0), s["dz"], s["n"], s["dbias"], s["rows"], s["n"], s["type"],
                             s["act_code"], ws, ws.numel())
        return s["dbias"] if z is None else (s["dz"], s["dbias"])
    if op == CE:
        qf.qfmt_linear_cross_entropy(s["a"], s["b"], s["kind"], s["bias"], s["targets"], s["loss"], s["lse"], s["mean"], ws, ws.numel())
        return s["loss"], s["lse"], s["mean"]
    if op == CE_BWD:
        qf.qfmt_linear_cross_entropy_backward(s["a"], s["b"], s["kind"], s["bias"], s["targets"], s["lse"], None, s["dls"], s["dh"],
                                              s["hidden"], s["dw"], s["dw"].stride(0), s["dbias"], ws, ws.numel())
        return s["dh"], s["dw"], s["dbias"]
    qf.qfmt_grad_norm(s["tensors"], s["count"], s["chunks"], MOST, s["dls"], s["record"], None, ws, ws.numel())
    qf.qfmt_grad_clip(s["tensors"], s["count"], s["chunks"], s["record"])
    return s["out"], s["record"].view(torch.float32)[:1]


# ---- the plain forms --------------------------------------------------------------------------------------------------


def _plain_act(act, z):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -(0.5 ** 0.5))
    if act == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _plain_slope(act, z):
    if act == "relu":
        return (z > 0.0).float()
    if act == "gelu":
        return 0.5 * torch.erfc(z * -(0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = 2.0 * (2.0 / math.pi) ** 0.5
        p = 1.0 / (1.0 + torch.exp(-c * (z + 0.044715 * z * z * z)))
        return p + z * p * (1.0 - p) * c * (1.0 + 3.0 * 0.044715 * z * z)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p + z * p * (1.0 - p)


def _plain_weight(s):
    w = s["w"].float()
    return w.t() if s["trans"] else w


def _plain_logits(s):
    logits = s["h"].float() @ _plain_weight(s)
    return logits if s["bias"] is None else logits.add_(s["bias"])


def _plain(s):
    op, dtype = s["op"], s["type"]
    if op == CLIP:
        scale = s["dls"][0]
        grads = s["flat"].float()
        norm = torch.sqrt(torch.sum(grads * grads, dtype=torch.float64)) / scale
        return (grads * (torch.clamp(MOST / norm, max=1.0) / scale).float()).to(dtype), norm.float().view(1)
    if op == LINEAR:
        z = s["x"].float() @ _plain_weight(s) + s["bias"]
        y = _plain_act(s["act"], z)
        y = (y if s["extra"] is None else y + s["extra"].float()).to(dtype)
        return (y, z.to(dtype)) if s["keep"] else y
    if op in (LINEAR_BWD, ACT_BWD):
        dz = s["dy"].float() if op == ACT_BWD else s["x"].float() @ _plain_weight(s)
        if s["extra"] is not None:
            dz = dz + s["extra"].float()
        if s["act"] != "none":
            dz = dz * _plain_slope(s["act"], s["z"].float())
        dbias = dz.sum(dim=0)
        return dbias if op == ACT_BWD and s["act"] == "none" else (dz.to(dtype), dbias)
    counts = s["targets"] != IGNORED
    picked = s["targets"].clamp(min=0)[:, None]
    logits = _plain_logits(s)
    if op == CE:
        most = logits.amax(dim=1, keepdim=True)
        lse = (torch.log(torch.exp(logits - most).sum(dim=1)) + most[:, 0]) * counts
        loss = (lse - logits.gather(1, picked)[:, 0]) * counts
        return loss, lse, (loss.sum() / counts.sum().clamp(min=1)).view(1)
    p = logits.sub_(s["lse"][:, None]).exp_()
    p.scatter_add_(1, picked, torch.full_like(picked, -1.0, dtype=torch.float32))
    p.mul_((counts * (s["dls"][0] / counts.sum().clamp(min=1)))[:, None])
    dw = p.t() @ s["h"].float() if s["trans"] else s["h"].float().t() @ p
    return (p @ _plain_weight(s).t()).to(dtype), dw.to(dtype), p.sum(dim=0)


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------


def _exact_act(act, z):
    phi = torch.special.ndtr(z)
    if act == "gelu":
        return z * phi
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return {"none": z, "relu": torch.relu(z), "silu": z * torch.sigmoid(z)}[act]


def _exact_slope(act, z):
    """By differentiating the activation."""
    with torch.enable_grad():
        z = z.detach().requires_grad_()
        return torch.autograd.grad(_exact_act(act, z).sum(), z)[0]


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == CLIP:
        flat = torch.cat([g.reshape(-1) for g in s["grads"]])  # from the single gradients
        scale = float(s["dls"][0])
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(p.double())) ** 2 for p in flat.split(1 << 26))) / scale
        return flat.double() * (min(1.0, MOST / norm) / scale), torch.tensor([norm], device="cuda", dtype=torch.float64)
    w = None if op == ACT_BWD else (s["w"].double().t() if s["trans"] else s["w"].double())
    if op == LINEAR:
        z = torch.addmm(s["bias"].double(), s["x"].double(), w)
        y = _exact_act(s["act"], z)
        if s["extra"] is not None:
            y = y + s["extra"].double()
        return (y, z) if s["keep"] else y
    if op in (LINEAR_BWD, ACT_BWD):
        dz = s["dy"].double() if op == ACT_BWD else torch.mm(s["x"].double(), w)
        if s["extra"] is not None:
            dz += s["extra"].double()
        if s["act"] != "none":
            dz *= _exact_slope(s["act"], s["z"].double())
        ones = torch.ones(s["rows"], device="cuda", dtype=torch.float64)
        return ones @ dz if op == ACT_BWD and s["act"] == "none" else (dz, ones @ dz)
    h, rows = s["h"].double(), s["rows"]
    bias = torch.zeros(s["vocab"], device="cuda", dtype=torch.float64) if s["bias"] is None else s["bias"].double()
    scale = float(s["dls"][0]) / max(1, _counted(case))
    loss, lse = torch.zeros(2, rows, device="cuda", dtype=torch.float64).unbind(0)
    dh, dw, dbias = torch.zeros_like(h), torch.zeros_like(w), torch.zeros_like(bias)
    per = max(1, (1 << 27) // s["vocab"])
    counted = (s["targets"] != IGNORED).nonzero()[:, 0]
    for at in counted.split(per):  # rows that count, a gigabyte of logits at a time
        logits, t = torch.addmm(bias, h[at], w), s["targets"][at]
        each = torch.arange(len(at), device="cuda")
        if op == CE:
            lse[at] = torch.logsumexp(logits, dim=1)
            loss[at] = lse[at] - logits[each, t]
            continue
        d = torch.exp(logits - s["lse"][at].double()[:, None])
        d[each, t] -= 1.0
        d *= scale
        dh[at] = d @ w.t()
        dw += h[at].t() @ d
        dbias += d.sum(dim=0)
    if op == CE:
        return loss, lse, (loss.sum() / max(1, len(counted))).view(1)
    return dh, dw.t().contiguous() if s["trans"] else dw, dbias
