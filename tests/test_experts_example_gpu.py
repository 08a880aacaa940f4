"""The example of a layer of experts, at small sizes."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "experts.py")


def _load():
    spec = importlib.util.spec_from_file_location("experts_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("sizes", [
    dict(experts=8, choices=2, prompt=60, hidden=256, inner=96, requests=3, shares=2),
    dict(experts=20, choices=4, prompt=300, hidden=512, inner=160, requests=16, shares=4),
])
def test_layer(sizes):
    """The results' and the sum's rounding to bf16 (2^-8 each at most, relative to values
    whose weighted sum of squares they are), and fp32 sums; the shares round once each."""
    _, errors, apart = _load().main(steps=5, **sizes)
    assert len(errors) == 2 and max(errors) <= 2 * 2.0 ** -8 + 2.0 ** -12
    assert apart <= 3 * 2.0 ** -8


def test_router_gradient():
    """Against the formula in 64 bits: d w_j = dout . z, through the softmax over the chosen
    logits, times x.  fp32 sums over at most 256 channels and 40 tokens, the logits' rounding
    to fp32 (256 terms) in the weights: 2^-24 (256 + 256 + 40 + 64) of the sums' amounts."""
    module = _load()
    layer = module.Experts(10, 3, 256, 64)
    x, dout = (torch.randn((40, 256), device="cuda").bfloat16() for _ in range(2))
    grad, z, plan = module.router_gradient(layer, x, dout)
    l = x.double() @ layer.router.double().T
    v, i = torch.topk(l, 3, dim=1)
    w = torch.softmax(v, 1)
    dw = (z.double()[plan.slots.long()] * dout.double()[:, None]).sum(-1)
    amount = (z.double()[plan.slots.long()] * dout.double()[:, None]).abs().sum(-1)

    def back(d):
        return torch.zeros_like(l).scatter_(1, i, d)
    want = back(w * (dw - (w * dw).sum(1, keepdim=True))).T @ x.double()
    size = back(w * (amount + (w * amount).sum(1, keepdim=True))).T @ x.double().abs()
    assert ((grad.double() - want).abs() <= 2.0 ** -24 * 616 * size).all()
