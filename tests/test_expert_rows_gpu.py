"""Gather, combine and their gradients against 64 bits: types, row lengths, dropped pairs,
slots and rows that are none, autograd against the formula and against differences.

Tolerances: a sum of n products in fp32 differs by at most (n + 1) 2^-24 times the sum of
their amounts, a rounding to the output's type by half a step (2^-8 bf16, 2^-24 fp32)."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
# (T, experts, experts here, k, N)
SHAPES = [(1, 1, 1, 1, 1), (1, 8, 8, 2, 8), (3, 8, 4, 2, 5), (17, 16, 16, 3, 64), (40, 8, 2, 4, 100),
          (25, 60, 30, 5, 264), (33, 64, 64, 8, 1032), (9, 20, 20, 16, 2048), (12, 20, 10, 9, 4097),
          (5, 8, 8, 8, 12000)]


def randn(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(TYPES[dtype]).cuda()


def make(T, all_, E, k, N, dtype):
    plan = rfq.ExpertPlan(*ref.plan_tensors(ref.sort(ref.choices(T, all_, k, T + N), E)))
    return (plan, randn((T, N), dtype, 1), randn((T * k, N), dtype, 2),
            torch.softmax(randn((T, k), "f32", 3), 1))


def taken(z, slots):
    """float64 [T][k][N] rows of z, zeros for slots that are none."""
    s, z = slots.cpu().long(), z.double().cpu()
    ok = (s >= 0) & (s < len(z))
    return torch.where(ok[..., None], z[torch.where(ok, s, 0)], 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_gather(shape, dtype):
    plan, x, _, _ = make(*shape, dtype)
    got = rfq.rfq_expert_gather(x, plan)
    r = plan.rows.long()
    want = torch.where((r >= 0)[:, None], x[r.clamp(min=0)], 0)
    assert got.dtype == x.dtype and torch.equal(got, want)
    out = torch.full_like(want, 7.0)
    assert rfq.rfq_expert_gather(x, plan, out=out) is out and torch.equal(out, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_combine_and_gradient(shape, dtype):
    plan, d, z, w = make(*shape, dtype)
    T, _, _, k, N = shape
    rows = taken(z, plan.slots)
    w64, d64 = w.double().cpu()[..., None], d.double().cpu()[:, None]
    for weights, f in ((w, w64), (None, torch.ones_like(w64))):
        got = rfq.rfq_expert_combine(z, weights, plan)
        want, size = (rows * f).sum(1), (rows * f).abs().sum(1)
        tol = (k + 1) * ULP * size + HALF[z.dtype] * want.abs() + 2.0 ** -126
        assert got.dtype == z.dtype and ((got.double().cpu() - want).abs() <= tol).all()

        dz, dw = rfq.rfq_expert_combine_backward(d, z, weights, plan)
        want, size = (rows * d64).sum(-1), (rows * d64).abs().sum(-1)
        assert dw.dtype == torch.float32
        assert ((dw.double().cpu() - want).abs() <= (N + 1) * ULP * size).all()
        want = torch.zeros(z.shape, dtype=torch.float64)
        s = plan.slots.cpu().long().flatten()
        want[s[s >= 0]] = (f * d64).flatten(0, 1)[s >= 0]
        tol = (HALF[z.dtype] + ULP) * want.abs() + 2.0 ** -126
        assert dz.dtype == z.dtype and ((dz.double().cpu() - want).abs() <= tol).all()
        assert (dz[plan.rows < 0] == 0).all()


def test_slots_and_rows_that_are_none():
    x, z = randn((4, 40), "bf16", 1), randn((8, 40), "bf16", 2)
    rows = torch.tensor([0, 4, 3, 2 ** 31 - 1, 3, -1, -2 ** 31, 1], dtype=torch.int32).cuda()
    slots = torch.tensor([[0, 8], [-1, 7], [2 ** 31 - 1, -2 ** 31], [4, 2]], dtype=torch.int32).cuda()
    plan = (torch.tensor([0, 8], dtype=torch.int32).cuda(), rows, slots)
    got = rfq.rfq_expert_gather(x, plan)
    ok = (rows >= 0) & (rows < 4)
    assert torch.equal(got, torch.where(ok[:, None], x[torch.where(ok, rows, 0).long()], 0))
    got = rfq.rfq_expert_combine(z, None, plan).double().cpu()
    want = taken(z, slots).sum(1)
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs()).all()
    dz, dw = rfq.rfq_expert_combine_backward(x, z, None, plan)
    assert (dw[2] == 0).all() and dw[0, 1] == 0 and dw[1, 0] == 0
    assert torch.equal(dz, rfq.rfq_expert_gather(x, plan))
    # A slot that two choices name is read twice.
    slots[3, 1] = 4
    got = rfq.rfq_expert_combine(z, None, plan).double().cpu()
    want = taken(z, slots).sum(1)
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs()).all()


def test_masked_places_have_no_influence():
    """NaN and infinities in rows that no pair names."""
    plan, x, z, w = make(40, 8, 2, 4, 264, "bf16")
    want = rfq.rfq_expert_combine(z, w, plan)
    dz, dw = rfq.rfq_expert_combine_backward(x, z, w, plan)
    z[plan.rows < 0] = float("nan")
    assert torch.equal(rfq.rfq_expert_combine(z, w, plan), want)
    w2 = torch.where(plan.slots < 0, float("inf"), w)
    assert torch.equal(rfq.rfq_expert_combine(z, w2, plan), want)
    got = rfq.rfq_expert_combine_backward(x, z, w2, plan)
    assert torch.equal(got[0], dz) and torch.equal(got[1], dw)


@pytest.mark.parametrize("T,all_,E,k,N", [(7, 8, 8, 2, 24), (11, 8, 3, 4, 16)])
def test_autograd_matches_the_formula_and_differences(T, all_, E, k, N):
    """f = sum c out over a step of gather, combine: linear in x, z and each weight, so central
    differences with any step are exact but for the sums' rounding: (k + 1) 2^-24 of sum |c w z|
    on either side, divided by the step."""
    plan, x, z, w = make(T, all_, E, k, N, "f32")
    c = randn((T, N), "f32", 9)
    a, b, v = (t.clone().requires_grad_() for t in (x, z, w))
    out = rfq.rfq_expert_combine(rfq.rfq_expert_gather(a, plan) * b, v, plan)
    (out * c).sum().backward()
    rows, xs = taken(z, plan.slots), x.double().cpu()[:, None]
    live = (plan.slots >= 0).cpu()[..., None]
    w64, c64 = w.double().cpu()[..., None], c.double().cpu()[:, None]
    dx = (c64 * w64 * rows * live).sum(1)
    dw = (c64 * xs * rows).sum(-1)
    assert (a.grad.double().cpu() - dx).abs().max() <= (k + 4) * ULP * (c64 * w64 * rows).abs().sum(1).max()
    assert (v.grad.double().cpu() - dw).abs().max() <= (N + 4) * ULP * (c64 * xs * rows).abs().sum(-1).max()
    assert (b.grad[plan.rows < 0] == 0).all()

    def f(x, z, w):
        o = rfq.rfq_expert_combine(rfq.rfq_expert_gather(x, plan) * z, w, plan)
        return float((o.double() * c.double()).sum())
    h = 0.5
    size = float((c64 * w64 * rows * xs).abs().sum()) + N * float(c.abs().max()) * 4
    for t, grad in ((x, a.grad), (z, b.grad), (w, v.grad)):
        for at in [(0, 0), (T - 1, t.shape[1] - 1), (T // 2, 1)]:
            up, down = t.clone(), t.clone()
            up[at] += h
            down[at] -= h
            step = float(up[at].double() - down[at].double())
            args = [[n if s is t else s for s in (x, z, w)] for n in (up, down)]
            diff = (f(*args[0]) - f(*args[1])) / step
            assert abs(diff - float(grad[at])) <= 2 * (k + 4) * ULP * size / h


def test_second_order_through_gather():
    plan, x, _, _ = make(9, 8, 4, 3, 16, "f32")
    a = x.clone().requires_grad_()
    y = (rfq.rfq_expert_gather(a, plan) ** 2).sum()
    g, = torch.autograd.grad(y, a, create_graph=True)
    (g ** 2).sum().backward()
    n = (plan.slots >= 0).sum(1, keepdim=True).float()
    assert torch.allclose(a.grad, 8 * n * n * x, rtol=16 * ULP, atol=0)


def test_gradients_of_expanded_and_shared_inputs():
    plan, x, z, _ = make(10, 8, 8, 2, 32, "f32")
    w = torch.ones(1, device="cuda", requires_grad=True)
    a = z.clone().requires_grad_()
    out = rfq.rfq_expert_combine(a, w.expand(10, 2).contiguous(), plan) + rfq.rfq_expert_combine(a, None, plan)
    out.sum().backward()
    assert torch.equal(a.grad, torch.full_like(z, 2.0))
    want = z.double().sum()
    assert abs(float(w.grad) - float(want)) <= 64 * 20 * ULP * float(z.abs().sum())


def test_streams_and_only_the_wanted_gradient():
    plan, x, z, w = make(30, 8, 8, 4, 512, "bf16")
    want = rfq.rfq_expert_combine(z, w, plan)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    xs = rfq.rfq_expert_gather(x, plan, stream=s)
    got = rfq.rfq_expert_combine(z, w, plan, stream=s)
    a = w.clone().requires_grad_()
    s.wait_stream(torch.cuda.current_stream())
    y = rfq.rfq_expert_combine(z, a, plan, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want) and torch.equal(y, want)
    assert torch.equal(xs, rfq.rfq_expert_gather(x, plan))
    y.backward(x)
    torch.cuda.synchronize()
    assert torch.equal(a.grad, rfq.rfq_expert_combine_backward(x, z, w, plan)[1])


def test_captured_training_pass():
    plan, x, z, w = make(64, 16, 16, 4, 256, "bf16")
    x.requires_grad_(), w.requires_grad_()

    def step():
        xs = rfq.rfq_expert_gather(x, plan)
        return torch.autograd.grad(rfq.rfq_expert_combine(xs * z, w, plan), (x, w), z[:64])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (1, 2, 3):
        with torch.no_grad():
            x.copy_(randn(x.shape, "bf16", seed))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_empty_and_refusals():
    plan = rfq.ExpertPlan(*ref.plan_tensors((torch.zeros(9), torch.zeros(0), torch.zeros((0, 2)))))
    x = torch.empty((0, 16), device="cuda")
    assert rfq.rfq_expert_gather(x, plan).shape == (0, 16)
    assert rfq.rfq_expert_combine(x, None, plan).shape == (0, 16)
    dz, dw = rfq.rfq_expert_combine_backward(x, x, None, plan)
    assert dz.shape == (0, 16) and dw.shape == (0, 2)
    plan, x, z, w = make(6, 8, 8, 2, 32, "bf16")
    assert rfq.rfq_expert_gather(x[:, :0].contiguous(), plan).shape == (12, 0)
    assert (rfq.rfq_expert_combine_backward(x[:, :0].contiguous(), z[:, :0].contiguous(), w, plan)[1] == 0).all()
    with pytest.raises(ValueError, match="tokens"):
        rfq.rfq_expert_gather(x[:5], plan)
    with pytest.raises(ValueError, match="slots"):
        rfq.rfq_expert_combine(z[:11], w, plan)
    with pytest.raises(TypeError):
        rfq.rfq_expert_combine(z.half(), w, plan)
    with pytest.raises(TypeError):
        rfq.rfq_expert_combine(z, w.bfloat16(), plan)
    with pytest.raises(ValueError, match="contiguous"):
        rfq.rfq_expert_gather(z.T, plan)
    with pytest.raises(TypeError):
        rfq.rfq_expert_combine_backward(x.float(), z, w, plan)
    with pytest.raises(ValueError):
        rfq.rfq_expert_combine(z, w, plan, out=x[:5])
    with pytest.raises(ValueError, match="gradient"):
        rfq.rfq_expert_gather(x.clone().requires_grad_(), plan, out=torch.empty_like(z))
    with pytest.raises(rfq.RfqError, match="RFQ_ERR_ALIGN"):
        flat = torch.zeros(6 * 32 + 1, dtype=torch.bfloat16, device="cuda")
        rfq.rfq_expert_gather(flat[1:].view(6, 32), plan)
