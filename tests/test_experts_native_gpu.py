"""The native calls around a layer of experts against the binding's Python path (which an
explicit stream takes): the same results, the caller's own outputs returned, and tensors that
are not the common form left to the Python path."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq
from paper_2608_26581_amd import experts as module
from paper_2608_26581_amd import rfq as binding

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    pass


def _same(a, b):
    a, b = [x if isinstance(x, tuple) else (x,) for x in (a, b)]
    assert len(a) == len(b)
    for s, t in zip(a, b):
        assert s.dtype == t.dtype and s.shape == t.shape and s.stride() == t.stride()
        assert torch.equal(s, t)


def _served(monkeypatch, names):
    """Fails where one of these calls goes on in Python."""
    binding.load()
    assert binding._calls
    real = module._native

    def native(func, *args):
        r = real(func, *args)
        assert r is not None or func not in names, func
        return r
    monkeypatch.setattr(module, "_native", native)


def _inputs(T=40, E=8, k=3, N=64, K=96):
    g = torch.Generator(device="cuda").manual_seed(1)
    l = torch.randn((T, E), generator=g, device="cuda")
    x = torch.randn((T, N), generator=g, device="cuda").bfloat16()
    z = torch.randn((T * k, N), generator=g, device="cuda").bfloat16()
    return l, x, z, ref.codes((T,), K, 1), ref.codes((E, N), K, 2, None)


def test_results_match(monkeypatch):
    _served(monkeypatch, ("route", "route_backward", "expert_sort", "expert_gather",
                          "expert_combine", "expert_combine_backward", "gemm_experts"))
    l, x, z, a, w = _inputs()
    s = torch.cuda.current_stream()
    for renormalize in (True, False):
        r = rfq.rfq_route(l, 3, renormalize)
        _same(r, rfq.rfq_route(l, 3, renormalize, stream=s))
        _same(rfq.rfq_route_backward(r[0], l, *r, renormalize),
              rfq.rfq_route_backward(r[0], l, *r, renormalize, stream=s))
    plan = rfq.rfq_expert_sort(r[1], 8)
    assert isinstance(plan, rfq.ExpertPlan)
    _same(plan, rfq.rfq_expert_sort(r[1], 8, stream=s))
    _same(rfq.rfq_expert_sort(r[1], 4, first=2), rfq.rfq_expert_sort(r[1], 4, first=2, stream=s))
    many = ref.choices(3000, 64, 4, 1).cuda()
    work = torch.empty(rfq.rfq_expert_sort_workspace_bytes(3000, 4, 64), dtype=torch.uint8, device="cuda")
    _same(rfq.rfq_expert_sort(many, 64), rfq.rfq_expert_sort(many, 64, workspace=work, stream=s))
    _same(rfq.rfq_expert_sort(many, 64, workspace=work), rfq.rfq_expert_sort(many, 64, stream=s))
    _same(rfq.rfq_expert_gather(x, plan), rfq.rfq_expert_gather(x, plan, stream=s))
    for weights in (r[0], None):
        _same(rfq.rfq_expert_combine(z, weights, plan), rfq.rfq_expert_combine(z, weights, plan, stream=s))
        _same(rfq.rfq_expert_combine_backward(x, z, weights, plan),
              rfq.rfq_expert_combine_backward(x, z, weights, plan, stream=s))
    for rows in (plan.rows, None):
        b = a if rows is not None else ref.codes((120,), 96, 3, False)
        for dt in (torch.float32, torch.bfloat16):
            _same(rfq.rfq_gemm_experts(*b, *w, plan.offsets, rows=rows, out_dtype=dt),
                  rfq.rfq_gemm_experts(*b, *w, plan.offsets, rows=rows, out_dtype=dt, stream=s))


def test_given_outputs_are_returned_and_marked_written(monkeypatch):
    _served(monkeypatch, ("expert_gather", "expert_combine", "gemm_experts"))
    l, x, z, a, w = _inputs()
    weights, experts = rfq.rfq_route(l, 3)
    plan = rfq.rfq_expert_sort(experts, 8)
    for call, like in ((lambda o: rfq.rfq_expert_gather(x, plan, out=o), z),
                       (lambda o: rfq.rfq_expert_combine(z, weights, plan, out=o), x),
                       (lambda o: rfq.rfq_gemm_experts(*a, *w, plan.offsets, rows=plan.rows, out=o), z)):
        out = torch.empty_like(like)
        before = out._version
        assert call(out) is out and out._version > before


def test_other_forms_go_through_python(monkeypatch):
    l, x, z, a, w = _inputs()
    weights, experts = rfq.rfq_route(l, 3)
    plan = rfq.rfq_expert_sort(experts, 8)
    called = []
    real = module._native
    monkeypatch.setattr(module, "_native", lambda f, *r: called.append((f, real(f, *r))) or called[-1][1])
    _same(rfq.rfq_route(l.as_subclass(Sub), 3), (weights, experts))
    _same(tuple(rfq.rfq_expert_sort(experts.as_subclass(Sub), 8)), tuple(plan))
    _same(rfq.rfq_expert_gather(x.as_subclass(Sub), list(plan)), rfq.rfq_expert_gather(x, plan))
    assert [r for f, r in called[:3]] == [None] * 3
    for bad in (lambda: rfq.rfq_expert_gather(x, plan, out=z[1:]),
                lambda: rfq.rfq_expert_combine(z, weights, plan, out=x[1:]),
                lambda: rfq.rfq_gemm_experts(*a, *w, plan.offsets, rows=plan.rows, out=z[1:]),
                lambda: rfq.rfq_expert_gather(x, (plan.offsets.float(), *plan[1:])),
                lambda: rfq.rfq_expert_gather(x, (plan.offsets, plan.rows[1:], plan.slots)),
                lambda: rfq.rfq_expert_combine(z, weights.double(), plan),
                lambda: rfq.rfq_gemm_experts(*a, *w, plan.offsets, rows=plan.rows.long()),
                lambda: rfq.rfq_gemm_experts(*a, w[0].int(), w[1], plan.offsets, rows=plan.rows),
                lambda: rfq.rfq_route(l.double(), 3)):
        with pytest.raises((TypeError, ValueError)):
            bad()


def test_without_the_native_module(monkeypatch):
    l, x, z, a, w = _inputs()
    want = rfq.rfq_route(l, 3)
    binding.load()
    monkeypatch.setattr(binding, "_calls", False)
    monkeypatch.setattr(module, "_bound", None)
    _same(rfq.rfq_route(l, 3), want)
