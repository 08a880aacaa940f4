"""The calls around a layer of experts on a stream that is not torch's current one: the memory
that they take belongs to that stream's order, so that nothing on the current stream
gets it while the call still works on it, and results are the current stream's."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu

T, E, k, N, K = 2000, 16, 8, 64, 128            # (more pairs than one workgroup sorts)


def _calls():
    """{name: f(stream)} of every call (all rows of the product belong to an expert)."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    l, x, z, d = randn(T, E), randn(T, N).bfloat16(), randn(T * k, N).bfloat16(), randn(T, k)
    w, experts = rfq.rfq_route(l, k)
    plan = rfq.rfq_expert_sort(experts, E)
    assert rfq.rfq_expert_sort_workspace_bytes(T, k, E) > 0
    a, we = ref.codes((T,), K, 1), ref.codes((E, N), K, 2, None)
    return {
        "route": lambda s: rfq.rfq_route(l, k, stream=s),
        "route_backward": lambda s: rfq.rfq_route_backward(d, l, w, experts, stream=s),
        "expert_sort": lambda s: rfq.rfq_expert_sort(experts, E, stream=s),
        "expert_gather": lambda s: rfq.rfq_expert_gather(x, plan, stream=s),
        "expert_combine": lambda s: rfq.rfq_expert_combine(z, w, plan, stream=s),
        "expert_combine_backward": lambda s: rfq.rfq_expert_combine_backward(x, z, w, plan, stream=s),
        "gemm_experts": lambda s: rfq.rfq_gemm_experts(*a, *we, plan.offsets, rows=plan.rows, stream=s),
    }


def _grad_calls():
    """{name: f(stream)} of the differentiable calls, with their results detached."""
    g = torch.Generator(device="cuda").manual_seed(4)
    l = torch.randn((T, E), generator=g, device="cuda", requires_grad=True)
    x = torch.randn((T, N), generator=g, device="cuda", requires_grad=True)
    z = torch.randn((T * k, N), generator=g, device="cuda", requires_grad=True)
    w, experts = rfq.rfq_route(l.detach(), k)
    plan = rfq.rfq_expert_sort(experts, E)
    return {
        "route": lambda s: tuple(t.detach() for t in rfq.rfq_route(l, k, stream=s)),
        "expert_gather": lambda s: rfq.rfq_expert_gather(x, plan, stream=s).detach(),
        "expert_combine": lambda s: rfq.rfq_expert_combine(z, w, plan, stream=s).detach(),
        "expert_combine of ones": lambda s: rfq.rfq_expert_combine(z, None, plan, stream=s).detach(),
    }


def _tensors(r):
    return r if isinstance(r, tuple) else (r,)


def _same(got, want):
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert a.shape == b.shape and a.dtype == b.dtype
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("name", [
    "route", "route_backward", "expert_sort", "expert_gather", "expert_combine",
    "expert_combine_backward", "gemm_experts"])
def test_memory_is_taken_on_the_calls_stream(name, monkeypatch):
    f = _calls()[name]
    want = [t.clone() for t in _tensors(f(None))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    taken, real = [], torch.empty

    def empty(*args, **kw):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return real(*args, **kw)
    monkeypatch.setattr(torch, "empty", empty)
    got = f(s)
    monkeypatch.setattr(torch, "empty", real)
    assert taken and set(taken) == {s.cuda_stream}
    s.synchronize()
    _same(_tensors(got), want)


@pytest.mark.parametrize("calls,name", [
    (_calls, "route"), (_calls, "expert_sort"), (_calls, "expert_combine_backward"),
    (_grad_calls, "route"), (_grad_calls, "expert_gather"), (_grad_calls, "expert_combine"),
    (_grad_calls, "expert_combine of ones")])
def test_a_waiting_call_keeps_its_memory(calls, name):
    """The stream is busy with something else when the call is made and the current stream
    takes as much memory as it can get of the sizes in question meanwhile."""
    f = calls()[name]
    want = [t.clone() for t in _tensors(f(None))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(5000000)
    got = _tensors(f(s))
    others = [torch.full((1 << n,), 255, dtype=torch.uint8, device="cuda")
              for n in range(9, 25) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.all(t == 255) for t in others)
    _same(got, want)
