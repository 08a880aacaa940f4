"""The router's weights and gradient where the logits of a token lie far apart: from where an
exponential leaves the normal numbers (87) past where it is zero (110) to differences that
are infinite in fp32.  Every finite row is compared.

Tolerance of a weight e^d / sum, d = l - m, relative, in units of 2^-24.  The exponential
2^(d log2 e): d is rounded (|d| units), the power of two is within a unit in the last place (2), the
product's rounding error is multiplied back in (1 for the result; what is neglected is below
2^-34): |d| + 3.  The sum: its terms' errors are sum_i p_i (|d_i| + 3) with sum_i p_i |d_i| at most
the logarithm of up to 1024 terms (7), so 10, and 16 + 6 additions; the division 1.  Together
below |d| + 40.  Absolute: an exponential below the normal numbers may be zero, 2^-126; with |d|
above 110 both sides are below that.

The gradient [i chosen] g - p s, g = w dw, s = sum g: p as a weight (one more product), g and s
products and sums of up to 16 terms in 6 steps, one subtraction, so (|d_i| + 50) units of p_i sum |g|
+ |g_i|; the rounding to the logits' type; and 2^-126 (1 + sum |g|)."""
import math

import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SPREADS = (79.0, 85.0, 87.0, 87.3, 87.5, 88.0, 95.0, 100.0, 103.0, 104.0, 109.0, 110.0, 110.5,
           111.0, 128.0, 200.0, 1e4, 1e30, 1e38, 3.3e38)
MOST = torch.finfo(torch.bfloat16).max


def logits(E, dtype):
    """For each spread s: one largest logit and the others s below it, all; spread evenly from
    0 to s below; half of them beside the largest.  The largest is 0, 3 or, where s is far
    larger, s / 2, so that both ends are finite."""
    g = torch.Generator().manual_seed(E)
    rows = []
    for n, s in enumerate(SPREADS):
        m = s / 2 if s >= 1e4 else (0.0, 3.0)[n % 2]
        below = torch.full((3, E), s, dtype=torch.float64)
        below[1] = torch.linspace(0, s, E, dtype=torch.float64)
        below[2, :E // 2] = torch.rand(E // 2, generator=g).double()
        below[:, 0] = 0
        rows.append((m - below)[:, torch.randperm(E, generator=g)])
    ends = torch.full((2, E), -MOST, dtype=torch.float64)
    ends[:, E // 3] = MOST
    ends[1, E // 2:] = -math.inf
    return torch.cat((*rows, ends)).to(TYPES[dtype]).cuda()


def distances(l):
    l = l.double().cpu()
    return (l.amax(1, keepdim=True) - l).clamp(max=110.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("E,k", [(4, 4), (16, 16), (60, 6), (128, 8), (300, 5), (1024, 16)])
def test_weights(E, k, renormalize, dtype):
    l = logits(E, dtype)
    w, x = rfq.rfq_route(l, k, renormalize)
    rw, rx, _ = ref.route(l, k, renormalize)
    assert torch.equal(x.cpu().long(), rx) and torch.isfinite(rw).all()
    d = torch.where(rx >= 0, distances(l).gather(1, rx.clamp(min=0)), 0.0)
    tol = rw * (d + 40) * ULP + 2.0 ** -126
    assert ((w.double().cpu() - rw).abs() <= tol).all()
    # (The tolerance leaves no room for a lost weight where the exponential is normal.)
    assert (w.cpu()[(rx >= 0) & (rw > 2.0 ** -120)] > 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("E,k", [(4, 4), (60, 6), (300, 5), (1024, 16)])
def test_gradient(E, k, renormalize, dtype):
    l = logits(E, dtype)
    w, x = rfq.rfq_route(l, k, renormalize)
    dw = torch.randn((len(l), k), generator=torch.Generator().manual_seed(k))
    got = rfq.rfq_route_backward(dw.cuda(), l, w, x, renormalize).double().cpu()
    x = x.cpu().long()
    ok, at = x >= 0, torch.where(x >= 0, x, E)
    g = torch.where(ok, w.double().cpu() * dw.double(), 0.0)

    def spread(v):
        return torch.zeros((len(l), E + 1), dtype=torch.float64).scatter_add(1, at, v)[:, :E]
    if renormalize:
        p = spread(torch.where(ok, w.double().cpu(), 0.0))
    else:
        p = torch.softmax(l.double().cpu(), 1)
    size = g.abs().sum(1, keepdim=True)
    want = spread(g) - p * g.sum(1, keepdim=True)
    tol = ((distances(l) + 50) * ULP * (p * size + spread(g.abs())) + HALF[l.dtype] * want.abs()
           + 2.0 ** -126 * (1 + size))
    assert ((got - want).abs() <= tol).all()
