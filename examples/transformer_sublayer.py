"""Trains one transformer sub-layer, y = LN(x + D(x W + b)), in emulated 16-bit arithmetic on one GPU.

The product's operands, its output, the normalised output and the gradient that the two backward products read are
rounded to the format (1/6/9 by default) with their statistics recorded; the residual, the row statistics and the
master weights are fp32.  Dropout's mask is recomputed from (seed, step) in the backward pass.  The target is what
another sub-layer of the same shape gives, so the loss has somewhere to go.

    python examples/transformer_sublayer.py --rows 8192 --hidden 1024 --steps 20
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_15940_b200 as qf  # noqa: E402


class SubLayer:
    """Parameters, buffers and the two passes of one sub-layer for a fixed number of rows (tokens)."""

    def __init__(self, rows, hidden, p, fmt, seed, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.rows, self.hidden, self.p, self.fmt, self.seed = rows, hidden, p, fmt, seed
        self.weight = torch.randn(hidden, hidden, generator=gen, device=device) * hidden ** -0.5
        self.bias = torch.randn(hidden, generator=gen, device=device) * 0.1
        self.gamma = 1.0 + 0.3 * torch.randn(hidden, generator=gen, device=device)
        self.beta = 0.3 * torch.randn(hidden, generator=gen, device=device)
        tensor = lambda *shape: torch.empty(*shape, device=device)
        self.xq, self.out, self.h, self.y, self.dx, self.dresidual, self.dinput = (tensor(rows, hidden) for _ in range(7))
        self.wq, self.dweight = tensor(hidden, hidden), tensor(hidden, hidden)
        self.dbias, self.dgamma, self.dbeta = (tensor(hidden) for _ in range(3))
        self.mean, self.rstd = tensor(rows), tensor(rows)
        self.stats = torch.zeros(5, qf.STATS_WORDS, dtype=torch.int64, device=device)  # x, weight, product, y, dx
        self.norm = qf.make_norm(rows, hidden, torch.float32)
        self.ws_norm = torch.empty(qf.qfmt_layer_norm_workspace_bytes(self.norm), dtype=torch.uint8, device=device)
        x, w, g = qf.make_matrix(self.xq), qf.make_matrix(self.wq), qf.make_matrix(self.dx)
        wt, xt = qf.make_matrix(self.wq, True), qf.make_matrix(self.xq, True)
        need = max(qf.qfmt_linear_forward_workspace_bytes(x, w), qf.qfmt_gemm_workspace_bytes(g, wt), qf.qfmt_gemm_workspace_bytes(xt, g))
        self.ws = torch.empty(max(256, need), dtype=torch.uint8, device=device)
        self.matrices = x, w, g, wt, xt

    def forward(self, x, step):
        """y for the input x (fp32, rows x hidden); step selects the mask."""
        n, hidden = self.rows, self.hidden
        mx, mw = self.matrices[:2]
        qf.qfmt_quantize_stats(x, self.xq, x.numel(), self.fmt, self.stats[0])
        qf.qfmt_quantize_stats(self.weight, self.wq, self.weight.numel(), self.fmt, self.stats[1])
        qf.qfmt_linear_forward(mx, mw, self.bias, self.out, hidden, self.fmt, self.stats[2], 0, self.ws, self.ws.numel())
        self.drop = qf.make_dropout(self.p, self.seed, step)
        qf.qfmt_dropout_add_layer_norm(self.norm, self.drop, self.out, x, self.gamma, self.beta, self.h, self.y, self.mean, self.rstd,
                                       self.fmt, self.stats[3])
        return self.y

    def backward(self, dy):
        """Gradients of the parameters, in self.d*, and of the input, from dy = dL/dy."""
        hidden = self.hidden
        g, wt, xt = self.matrices[2:]
        qf.qfmt_dropout_add_layer_norm_backward(self.norm, self.drop, dy, None, self.h, self.mean, self.rstd, self.gamma, self.dx,
                                                self.dresidual, self.dgamma, self.dbeta, self.ws_norm, self.ws_norm.numel(), self.fmt,
                                                self.stats[4])
        qf.qfmt_gemm(xt, g, self.dweight, hidden, self.fmt, self.ws, self.ws.numel())
        torch.sum(self.dx, dim=0, out=self.dbias)
        qf.qfmt_gemm(g, wt, self.dinput, hidden, self.fmt, self.ws, self.ws.numel())
        return self.dinput.add_(self.dresidual)

    def update(self, rate):
        for value, grad in ((self.weight, self.dweight), (self.bias, self.dbias), (self.gamma, self.dgamma), (self.beta, self.dbeta)):
            value.sub_(grad, alpha=rate)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rows", type=int, default=8192, help="tokens in a batch")
    ap.add_argument("--hidden", type=int, default=1024, help="a multiple of 4 (the products' operands are fetched by the copy engine)")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--rate", type=float, default=0.2)
    ap.add_argument("--loss-scale", type=float, default=2.0 ** 10)
    ap.add_argument("--format", type=int, nargs=2, default=(6, 9), metavar=("E", "M"))
    a = ap.parse_args(argv)
    fmt = qf.make_format(*a.format)
    gen = torch.Generator(device="cuda").manual_seed(0)
    model, teacher = SubLayer(a.rows, a.hidden, a.dropout, fmt, 1), SubLayer(a.rows, a.hidden, 0.0, fmt, 2)
    losses = []
    for step in range(a.steps):
        x = torch.randn(a.rows, a.hidden, generator=gen, device="cuda")
        error = model.forward(x, step) - teacher.forward(x, 0)
        losses.append((error * error).mean())
        model.backward(error * (2.0 * a.loss_scale / a.rows))
        model.update(a.rate / a.loss_scale)
    torch.cuda.synchronize()
    losses = [float(v) for v in losses]
    st = model.stats.cpu()
    for name, row in zip(("x", "weight", "product", "y", "dx"), st):
        print("%-8s denormal fraction %.2e, underflow %d, overflow %d of %d" % (
            name, int(row[qf.ST_DENORMAL]) / max(1, int(row[qf.ST_TOTAL])), int(row[qf.ST_UNDERFLOW]), int(row[qf.ST_OVERFLOW]),
            int(row[qf.ST_TOTAL])))
    print("loss %.4f -> %.4f in %d steps" % (losses[0], losses[-1], a.steps))
    return losses, st, model


if __name__ == "__main__":
    main()
