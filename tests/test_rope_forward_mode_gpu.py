"""Forward-mode differentiation of the rotation: it has reverse mode only, and a tangent that
comes in is refused as torch refuses it for such functions, on the native calls and on the
binding's Python path (which an explicit stream takes), never dropped."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("name", ["rfq_rope", "rfq_rope_backward"])
def test_a_tangent_is_refused(name, path):
    f = getattr(rfq, name)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((5, 4, 64), generator=g, device="cuda").bfloat16()
    rest = torch.arange(5, device="cuda").int(), rfq.rope_table(9, 64)
    s = None if path == "native" else torch.cuda.current_stream()
    want = f(x, *rest, stream=s)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                with pytest.raises(NotImplementedError, match="jvp"):
                    f(dual, *rest, stream=s)
                with pytest.raises(ValueError, match="out takes no gradient"):
                    f(dual, *rest, out=torch.empty_like(x), stream=s)
                with pytest.raises(ValueError, match="out takes no gradient"):
                    f(x, *rest, out=forward_ad.make_dual(torch.empty_like(x), x), stream=s)
        # A tensor without a tangent is an ordinary one, also inside a level.
        assert torch.equal(f(x, *rest, stream=s), want)
    assert torch.equal(f(dual, *rest, stream=s), want)  # the level has ended


@pytest.mark.parametrize("name", ["rfq_rope", "rfq_rope_backward"])
def test_a_tangent_of_the_gradient_is_refused(name):
    """Forward mode over reverse: the gradient that comes to the backward pass has a tangent."""
    x = torch.ones((5, 4, 64), device="cuda", requires_grad=True)
    y = getattr(rfq, name)(x, torch.arange(5, device="cuda").int(), rfq.rope_table(9, 64))
    with forward_ad.dual_level():
        c = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(NotImplementedError, match="jvp"):
            torch.autograd.grad((y * c).sum(), x)
