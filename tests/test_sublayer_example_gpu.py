"""examples/transformer_sublayer.py: the sub-layer's passes together with the rounding pass and the products, as a training
step uses them."""
import importlib.util
import os

import pytest
import torch

import paper_2103_15940_b200 as qf
import sublayer_reference as ref

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "transformer_sublayer.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("transformer_sublayer", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", [("6", "9"), ("5", "10")])
def test_the_loss_falls(example, fmt):
    losses, stats, model = example.main(["--rows", "512", "--hidden", "128", "--steps", "30", "--format", *fmt])
    assert losses[-1] < 0.6 * losses[0]
    assert [int(r[qf.ST_TOTAL]) for r in stats] == [512 * 128, 128 * 128, 512 * 128, 512 * 128, 512 * 128]


def test_gradients_of_one_step(example):
    """Every gradient against automatic differentiation of the same step in 64 bits from the rounded operands.  Wide
    formats (1/8/10) leave only rounding errors of 2^-11 in the product's operands and output, in y and in dx."""
    rows, hidden = 256, 64
    layer = example.SubLayer(rows, hidden, 0.2, qf.make_format(8, 10), 5)
    gen = torch.Generator().manual_seed(1)
    x, dy = torch.randn(rows, hidden, generator=gen), torch.randn(rows, hidden, generator=gen)
    layer.forward(x.cuda(), 3)
    dinput = layer.backward(dy.cuda())
    t = [v.detach().double().cpu().requires_grad_() for v in (layer.xq, layer.wq, layer.bias, layer.gamma, layer.beta)]
    residual = x.double().requires_grad_()
    keep = ref.keep_mask(rows, hidden, 0.2, 5, 3).double() * 65536 / (65536 - ref.threshold(0.2))
    h = residual + keep * (t[0] @ t[1] + t[2])
    y = torch.nn.functional.layer_norm(h, (hidden,), t[3], t[4], 1e-5)
    (y * dy.double()).sum().backward()
    want = {"dweight": t[1].grad, "dbias": t[2].grad, "dgamma": t[3].grad, "dbeta": t[4].grad, "dresidual": residual.grad}
    for name, grad in want.items():
        got = getattr(layer, name).double().cpu()
        assert float((got - grad).norm() / grad.norm()) < 4 * 2.0 ** -11, name  # a few roundings of 2^-11 each, adding in squares
    total = t[0].grad + residual.grad
    assert float((dinput.double().cpu() - total).norm() / total.norm()) < 4 * 2.0 ** -11
