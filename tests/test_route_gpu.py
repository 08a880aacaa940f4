"""The router: choices against the definition (ties, masks, NaN, infinities), weights and
gradients against 64 bits and against differences, autograd, streams and graphs.

Tolerance of a weight, relative: l - m is rounded (|l - m| 2^-24 in the exponent), expf to
2 units (2^-22), a sum of up to 1024 positive terms in a lane's 16 and 6 steps of pairs
(22 roundings), the division to 1: with s the largest |l - m|, numerator and denominator
together at most (2 s + 8 + 8 + 22 + 2) 2^-24 < (2 s + 40) 2^-24."""
import math

import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def logits(T, E, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (3.0 * torch.randn((T, E), generator=g)).to(TYPES[dtype]).cuda()


def check(l, k, renormalize):
    w, x = rfq.rfq_route(l, k, renormalize)
    assert w.dtype == torch.float32 and x.dtype == torch.int32 and w.shape == x.shape == (len(l), k)
    rw, rx, s = ref.route(l, k, renormalize)
    assert torch.equal(x.cpu().long(), rx)
    w = w.double().cpu()
    assert torch.equal(torch.isnan(w), torch.isnan(rw))
    tol = rw * ((2 * s + 40) * ULP)[:, None]
    assert (((w - rw).abs() <= tol) | torch.isnan(rw)).all()
    return w, x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k", [
    (1, 1, 1), (3, 8, 2), (5, 16, 16), (1, 17, 4), (33, 31, 3), (17, 32, 8), (129, 60, 4),
    (64, 64, 6), (7, 100, 1), (13, 90, 5), (11, 96, 6), (50, 128, 8), (21, 160, 6), (7, 157, 5), (8, 192, 8), (5, 186, 16), (16, 255, 9), (9, 256, 8), (6, 257, 8),
    (5, 511, 16), (5, 512, 2), (4, 1000, 10), (3, 1024, 16)])
def test_choices_and_weights(T, E, k, renormalize, dtype):
    check(logits(T, E, dtype, T * E + k), k, renormalize)


@pytest.mark.parametrize("E,k", [(8, 8), (60, 7), (128, 8), (300, 16)])
def test_ties_go_to_the_lowest_index(E, k):
    g = torch.Generator().manual_seed(E)
    l = torch.randint(0, 3, (40, E), generator=g).float()
    l[0] = 1.0
    l[1, ::2], l[1, 1::2] = 0.0, -0.0
    for t in (l, l.bfloat16()):
        check(t.cuda(), k, True)
        check(t.cuda(), k, False)
    _, x = rfq.rfq_route(l.cuda(), k)
    assert x[0].tolist() == list(range(k)) and x[1].tolist() == list(range(k))


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("dtype", TYPES)
def test_masked_experts_infinities_and_nan(dtype, renormalize):
    E, k = 60, 6
    l = logits(12, E, "f32", 5).cpu()
    l[0] = -math.inf                                   # a padded token
    l[1, 3:] = -math.inf                               # three experts left
    l[2, :k] = -math.inf
    l[3, 7] = math.nan
    l[4, [0, 59]] = math.nan
    l[5, 11] = math.inf
    l[6, [1, 2]] = math.inf
    l[7] = math.nan
    l[8, :] = torch.finfo(torch.bfloat16).min
    l[9, 5] = torch.finfo(torch.bfloat16).max
    l[9, 6:] = torch.finfo(torch.bfloat16).min
    l[10, 4] = -math.nan
    for t in (l, torch.full((3, E), -math.inf)):
        rw, rx, s = ref.route(t.to(TYPES[dtype]), k, renormalize)
        w, x = rfq.rfq_route(t.to(TYPES[dtype]).cuda(), k, renormalize)
        assert torch.equal(x.cpu().long(), rx)
        w = w.double().cpu()
        # A row with +infinity: NaN where it counts, and zeros or NaN elsewhere.
        odd = torch.isnan(rw).any(1)
        assert torch.isnan(w[odd]).any(1).all() and not torch.isnan(w[~odd]).any()
        fine = s < 80
        tol = rw * ((2 * s + 40) * ULP)[:, None] + 2.0 ** -126
        assert ((w - rw).abs() <= tol)[~odd & fine].all()
        assert (w[~odd].sum(1) <= 1.0 + 64 * ULP).all()


def test_rows_that_do_not_start_aligned():
    g = torch.Generator().manual_seed(2)
    for dtype in TYPES.values():
        flat = torch.randn(1 + 20 * 64, generator=g).to(dtype).cuda()
        check(flat[1:].view(20, 64), 8, True)


def gradient(l, d, w, x, renormalize):
    """The formula in 64 bits, and the sum of what its terms amount to."""
    l, d, w = l.double().cpu(), d.double().cpu(), w.double().cpu()
    x = x.cpu().long()
    E = l.shape[1]
    ok = (x >= 0) & (x < E)
    at = torch.where(ok, x, E)
    g = torch.where(ok, w * d, 0.0)
    one = torch.zeros((len(l), E + 1), dtype=torch.float64)
    s, sa = g.sum(1, keepdim=True), g.abs().sum(1, keepdim=True)
    chosen = one.scatter_add(1, at, g)[:, :E]
    if renormalize:
        p = one.scatter_add(1, at, w)[:, :E]
    else:
        p = torch.where((l > -math.inf).any(1, keepdim=True), torch.softmax(l, 1), 0.0)
    return chosen - p * s, one.scatter_add(1, at, g.abs())[:, :E] + p * sa


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 8, 2), (33, 60, 4), (70, 128, 8), (9, 161, 6),
                                   (4, 256, 16), (3, 700, 3), (2, 1024, 8)])
def test_gradient_matches_the_formula(T, E, k, renormalize, dtype):
    l = logits(T, E, dtype, E)
    if T > 3:
        l[0] = -math.inf
        l[1, 1:] = -math.inf
    w, x = rfq.rfq_route(l, k, renormalize)
    d = torch.randn((T, k), generator=torch.Generator().manual_seed(3)).cuda()
    got = rfq.rfq_route_backward(d, l, w, x, renormalize)
    assert got.dtype == l.dtype
    want, size = gradient(l, d, w, x, renormalize)
    # Products and sums of up to 16 terms, and p as above (|l - m| below 30 here).
    tol = 128 * ULP * size + HALF[l.dtype] * want.abs() + 2.0 ** -126
    assert ((got.double().cpu() - want).abs() <= tol).all()


def test_gradient_of_experts_outside_and_named_twice():
    l = logits(3, 20, "f32", 1)
    x = torch.tensor([[4, 4, -1], [19, 25, 0], [-7, -1, -1]], dtype=torch.int32).cuda()
    w = torch.tensor([[.5, .3, .2], [.6, .2, .2], [.4, .3, .3]]).cuda()
    d = torch.tensor([[1., 2., 3.], [-1., 5., 2.], [1., 1., 1.]]).cuda()
    for renormalize in (True, False):
        want, size = gradient(l, d, w, x, renormalize)
        got = rfq.rfq_route_backward(d, l, w, x, renormalize).double().cpu()
        assert ((got - want).abs() <= 128 * ULP * size).all()


@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_matches_differences(renormalize):
    """Central differences of f = sum c_j w_j with a step h = 2^-6: the choice stays (logits
    are multiples of 1/4), third derivatives are at most sum |c| (so h^2 / 6 of that), and
    the weights' rounding (relative (2 s + 40) 2^-24 with s < 4: below 2^-18) divides by h."""
    E, k, h = 12, 4, 2.0 ** -6
    g = torch.Generator().manual_seed(4)
    base = torch.randperm(E, generator=g).float() / 4
    c = torch.randn(k, generator=g)
    both = base.repeat(2 * E, 1)
    both[torch.arange(E), torch.arange(E)] += h
    both[E + torch.arange(E), torch.arange(E)] -= h
    f = rfq.rfq_route(both.cuda(), k, renormalize)[0].double().cpu() @ c.double()
    diff = (f[:E] - f[E:]) / (2 * h)
    l = base[None].cuda().requires_grad_()
    w, x = rfq.rfq_route(l, k, renormalize)
    assert w.requires_grad and not x.requires_grad
    (w[0] @ c.cuda()).backward()
    tol = (h * h / 6 + 2.0 ** -18 / h) * c.abs().sum()
    assert (l.grad[0].double().cpu() - diff).abs().max() <= tol


def test_autograd_on_strided_gradients_and_streams():
    l = logits(6, 40, "f32", 9)
    want, _ = gradient(l, torch.ones(6, 3), *rfq.rfq_route(l, 3), True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (None, s):
        a = l.clone().requires_grad_()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        w, x = rfq.rfq_route(a, 3, stream=stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        w.sum().backward()                              # an expanded gradient
        torch.cuda.synchronize()
        assert (a.grad.double().cpu() - want).abs().max() <= 256 * ULP


def test_captured_and_replayed():
    l = logits(100, 128, "bf16", 1)
    for _ in range(2):
        rfq.rfq_route(l, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w, x = rfq.rfq_route(l, 8)
        d = rfq.rfq_route_backward(w, l, w, x)
    for seed in (2, 3, 4):
        l.copy_(logits(100, 128, "bf16", seed))
        graph.replay()
        ew, ex = rfq.rfq_route(l, 8)
        torch.cuda.synchronize()
        assert torch.equal(w, ew) and torch.equal(x, ex)
        assert torch.equal(d, rfq.rfq_route_backward(ew, l, ew, ex))


def test_empty_and_refusals():
    w, x = rfq.rfq_route(torch.empty((0, 8), device="cuda"), 2)
    assert w.shape == x.shape == (0, 2)
    l = logits(4, 8, "f32", 0)
    for k in (0, 9, 17, -1):
        with pytest.raises(ValueError, match="k must be"):
            rfq.rfq_route(l, k)
    with pytest.raises(TypeError):
        rfq.rfq_route(l.half(), 2)
    with pytest.raises(ValueError, match="contiguous"):
        rfq.rfq_route(l.T, 2)
    with pytest.raises(ValueError, match="2-D"):
        rfq.rfq_route(l[0], 2)
    with pytest.raises(ValueError, match="device tensor"):
        rfq.rfq_route(l.cpu(), 2)
    with pytest.raises(rfq.RfqError, match="RFQ_ERR_SHAPE"):
        rfq.rfq_route(torch.zeros((1, 1025), device="cuda"), 2)
    w, x = rfq.rfq_route(l, 2)
    with pytest.raises(ValueError):
        rfq.rfq_route_backward(w[:2], l, w, x)
    with pytest.raises(TypeError):
        rfq.rfq_route_backward(w, l, w, x.long())
