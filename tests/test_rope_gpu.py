"""Rotary positions with several axes against the formula: bit for bit in fp32
arithmetic, near it in 64 bits, and the gradient against differences."""
import numpy as np
import pytest
import torch

import paper_2608_26581_amd as rfq
import kv_util as ku

pytestmark = pytest.mark.gpu


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _case(T, H, D, rotary, n_axes, seed, max_pos=97):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, H, D)).astype(np.float32)
    pos = rng.integers(0, max_pos, (n_axes, T)).astype(np.int32)
    axes = bytes(int(a) for a in rng.integers(0, n_axes, rotary // 2))
    return x, pos, axes, ku.table(max_pos, rotary)


def _bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


SHAPES = [(1, 1, 16, 16), (1, 40, 128, 128), (3, 5, 96, 64), (7, 1, 64, 32), (33, 24, 128, 64),
          (130, 8, 256, 256), (5, 3, 512, 512), (17, 9, 48, 16), (2100, 12, 64, 64), (2049, 7, 80, 48)]


@pytest.mark.parametrize("T,H,D,rotary", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("backward", [False, True])
def test_matches_the_formula(T, H, D, rotary, interleaved, dtype, backward):
    n_axes = 1 + (T + H) % 4
    x, pos, axes, cs = _case(T, H, D, rotary, n_axes, T + D)
    xd = _dev(x).to(dtype)
    x = xd.float().cpu().numpy()
    print("rope T=%d H=%d D=%d rotary=%d axes=%d" % (T, H, D, rotary, n_axes), flush=True)
    f = rfq.rfq_rope_backward if backward else rfq.rfq_rope
    y = f(xd, _dev(pos), _dev(cs), axes, interleaved=interleaved)
    ref32 = ku.rotate(x, pos, cs, axes, interleaved, backward, np.float32)
    want = _dev(ref32).to(dtype)
    assert np.array_equal(_bits(y), _bits(want))
    # fp32 products and sums: a few 2^-24 of |a| + |b|; the bf16 rounding: 2^-9.
    ref = ku.rotate(x, pos, cs, axes, interleaved, backward)
    top = np.abs(x).max() * 2
    tol = 3 * 2.0 ** -24 * top + (2.0 ** -8 * np.abs(ref) if dtype == torch.bfloat16 else 0)
    assert np.all(np.abs(y.float().cpu().numpy() - ref) <= tol)


def test_gradient_against_differences():
    """<dy, (rope(x + h e) - rope(x - h e)) / 2h> is the gradient's component along e
    (the rotation is linear: differences are exact but for fp32 rounding, 2^-20 of
    the norms here)."""
    T, H, D = 6, 2, 64
    x, pos, axes, cs = _case(T, H, D, 48, 3, 1)
    rng = np.random.default_rng(2)
    dy = rng.standard_normal((T, H, D)).astype(np.float32)
    args = (_dev(pos), _dev(cs), axes)
    for interleaved in (False, True):
        dx = rfq.rfq_rope_backward(_dev(dy), *args, interleaved=interleaved).cpu().numpy()
        for k in range(20):
            e = rng.standard_normal((T, H, D)).astype(np.float32)
            up, down = (rfq.rfq_rope(_dev(x + s * e), *args, interleaved=interleaved).cpu().numpy()
                        .astype(np.float64) for s in (0.5, -0.5))
            slope = np.sum(dy * (up - down))
            norm = np.linalg.norm(dy) * (np.linalg.norm(x) + np.linalg.norm(e))
            assert abs(slope - np.sum(dx.astype(np.float64) * e)) <= 2.0 ** -20 * norm


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward_undoes_forward(dtype):
    x, pos, axes, cs = _case(50, 4, 128, 128, 2, 3)
    xd = _dev(x).to(dtype)
    y = rfq.rfq_rope(xd, _dev(pos), _dev(cs), axes)
    z = rfq.rfq_rope_backward(y, _dev(pos), _dev(cs), axes)
    tol = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -21
    assert (z.float() - xd.float()).abs().max().item() <= tol * np.abs(x).max() * 2


def test_positions_outside_the_table_give_nan():
    x, pos, _, cs = _case(5, 3, 64, 32, 2, 4)
    pos[0] = [0, 96, 97, -1, 2 ** 31 - 1]
    axes = bytes([0] * 8 + [1] * 8)
    y = rfq.rfq_rope(_dev(x), _dev(pos), _dev(cs), axes).cpu().numpy()
    bad = np.zeros((5, 3, 64), bool)
    bad[2:, :, 0:8] = bad[2:, :, 16:24] = True
    assert np.array_equal(np.isnan(y), bad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [9, 2050])
def test_strides_and_in_place(dtype, T):
    """Slices of a joint tensor, heads before tokens, a broadcast head, and y = x;
    nothing beside the rotated heads is written."""
    x, pos, axes, cs = _case(T, 6, 128, 64, 2, 5)
    xd = _dev(x).to(dtype)
    args = (_dev(pos), _dev(cs), axes)
    ref = rfq.rfq_rope(xd, *args)
    joint = torch.full((T, 10, 144), 3.0, dtype=dtype, device="cuda")
    view = joint[:, 2:8, 8:136] if dtype == torch.bfloat16 else joint[:, 2:8, 4:132]
    view.copy_(xd)
    assert torch.equal(rfq.rfq_rope(view, *args), ref)
    out = rfq.rfq_rope(view, *args, out=view)
    assert torch.equal(out, ref)
    view.fill_(3.0)
    assert torch.all(joint == 3.0)
    turned = xd.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(rfq.rfq_rope(turned, *args), ref)
    one = xd[:, :1].expand(-1, 6, -1)
    assert torch.equal(rfq.rfq_rope(one, *args), rfq.rfq_rope(one.contiguous(), *args))


def test_empty_and_refused():
    x, pos, axes, cs = _case(4, 2, 64, 64, 1, 6)
    xd, p, c = _dev(x), _dev(pos), _dev(cs)
    assert rfq.rfq_rope(xd[:0], p[:, :0], c).shape == (0, 2, 64)
    assert rfq.rfq_rope(xd[:, :0], p, c).shape == (4, 0, 64)
    assert torch.equal(rfq.rfq_rope(xd, p[0], c), rfq.rfq_rope(xd, p, c, bytes(32)))
    with pytest.raises(ValueError, match="per rotated pair"):
        rfq.rfq_rope(xd, p, c, bytes(31))
    with pytest.raises(rfq.RfqError, match="SHAPE"):
        rfq.rfq_rope(xd, p, c, bytes([1] * 32))                       # one axis only
    with pytest.raises(rfq.RfqError, match="SHAPE"):
        rfq.rfq_rope(xd[..., :32], p, c)                              # more channels than D
    with pytest.raises(TypeError, match="int32"):
        rfq.rfq_rope(xd, p.long(), c)
    with pytest.raises(TypeError):
        rfq.rfq_rope(xd.half(), p, c)
    with pytest.raises(ValueError, match="per token"):
        rfq.rfq_rope(xd, p[:, :3], c)
    with pytest.raises(ValueError, match="shape"):
        rfq.rfq_rope(xd, p, c, out=xd[:3])
    with pytest.raises(ValueError, match="contiguous"):
        rfq.rfq_rope(xd.transpose(1, 2), p, c)
    with pytest.raises(rfq.RfqError, match="ALIGN"):
        rfq.rfq_rope(torch.zeros(4 * 2 * 65, device="cuda").view(4, 2, 65)[..., 1:], p, c)


def test_rope_table_helper():
    t = rfq.rope_table(33, 64, 500000.0)
    assert np.array_equal(t.cpu().numpy(), ku.table(33, 64, 500000.0))
    assert rfq.rope_axes((2, 0, 3)) == bytes([0, 0, 2, 2, 2])


@pytest.mark.parametrize("f,g", [(rfq.rfq_rope, rfq.rfq_rope_backward),
                                 (rfq.rfq_rope_backward, rfq.rfq_rope)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_autograd(f, g, interleaved, dtype):
    """A result of x that asks for a gradient has one: the rotation by the opposite angle, of
    gradients with any strides, and its own gradient in turn."""
    x, pos, axes, cs = _case(23, 4, 64, 48, 3, 8)
    args = (_dev(pos), _dev(cs), list(axes))
    kw = dict(interleaved=interleaved)
    xd = _dev(x).to(dtype).requires_grad_()
    with torch.no_grad():
        plain = f(xd, *args, **kw)
    assert not plain.requires_grad and not f(xd.detach(), *args, **kw).requires_grad
    y = f(xd, *args, **kw)
    assert y.requires_grad and torch.equal(y.detach(), plain)
    rng = np.random.default_rng(9)
    dy = _dev(rng.standard_normal(x.shape).astype(np.float32)).to(dtype)
    want = g(dy, *args, **kw)
    for grad in (dy, dy.transpose(0, 2).contiguous().transpose(0, 2),
                 torch.cat((dy.flatten()[:1], dy.flatten()))[1:].view(dy.shape)):
        dx, = torch.autograd.grad(y, xd, grad, retain_graph=True)
        assert torch.equal(dx, want)
    dx, = torch.autograd.grad(y.float().sum(), xd, retain_graph=True)      # (a broadcast 1)
    assert torch.equal(dx, g(torch.ones_like(dy), *args, **kw))
    v = dy.clone().requires_grad_()
    dx, = torch.autograd.grad(y, xd, v, create_graph=True)
    assert torch.equal(dx.detach(), want)
    again, = torch.autograd.grad(dx, v, xd.detach())
    assert torch.equal(again, plain)


def test_autograd_on_a_given_stream():
    x, pos, axes, cs = _case(50, 4, 64, 64, 2, 10)
    args = (_dev(pos), _dev(cs), axes)
    xd = _dev(x).requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = rfq.rfq_rope(xd, *args, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    y.backward(y.detach())
    torch.cuda.synchronize()
    assert torch.equal(xd.grad, rfq.rfq_rope_backward(y.detach(), *args))


def test_out_and_gradients():
    """out cannot carry a gradient."""
    x, pos, axes, cs = _case(9, 4, 64, 64, 2, 11)
    args = (_dev(pos), _dev(cs), axes)
    xd = _dev(x).requires_grad_()
    with pytest.raises(ValueError, match="out"):
        rfq.rfq_rope(xd, *args, out=torch.empty_like(x_ := xd.detach()))
    with torch.no_grad():
        assert torch.equal(rfq.rfq_rope(xd, *args, out=torch.empty_like(x_)), rfq.rfq_rope(x_, *args))


def test_what_is_written_in_place_is_noticed():
    """A tensor saved for a backward pass and then given as out makes that pass fail."""
    x, pos, axes, cs = _case(9, 4, 64, 64, 2, 11)
    args, x_ = (_dev(pos), _dev(cs), axes), _dev(x)
    for f in (rfq.rfq_rope, rfq.rfq_rope_backward):
        for stream in (None, torch.cuda.current_stream()):
            w = torch.ones_like(x_, requires_grad=True)
            h = x_.clone()
            z = (w * h).sum()
            assert f(h, *args, out=h, stream=stream) is h
            with pytest.raises(RuntimeError, match="inplace"):
                z.backward()
    with torch.inference_mode():
        h = x_.clone()
        assert torch.equal(rfq.rfq_rope(h, *args, out=h), rfq.rfq_rope(x_, *args))


def test_refused_arguments_of_a_differentiable_call():
    """The same errors as without a gradient."""
    x, pos, axes, cs = _case(4, 2, 64, 64, 1, 12)
    xd, p, c = _dev(x).requires_grad_(), _dev(pos), _dev(cs)
    for bad, error in (((None, c), ValueError), ((p.long(), c), TypeError), ((p, None), ValueError),
                       ((p[:, :3], c), ValueError), ((p, c, bytes(31)), ValueError),
                       ((p, c, bytes([1] * 32)), rfq.RfqError)):
        for a in (xd, xd.detach()):
            with pytest.raises(error):
                rfq.rfq_rope(a, *bad)
