"""A layer of experts as a program runs it: router, sort, quantized tokens, gate and up
products through the row map, SwiGLU and quantization, the down product on sorted rows,
and the weighted way back; against the same steps in 64 bits, eager and as a graph."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq
from gpu_util import TOL_SUM

pytestmark = pytest.mark.gpu


def layer(x, logits, k, w, first):
    E, Nh, half = w["gate"][0].shape
    weights, experts = rfq.rfq_route(logits, k)
    plan = rfq.rfq_expert_sort(experts, E, first=first)
    q = rfq.rfq_quantize_act(x)
    g, u = (rfq.rfq_gemm_experts(*q, *w[n], plan.offsets, rows=plan.rows, out_dtype=torch.bfloat16,
                                 out=torch.zeros((plan.rows.numel(), Nh), dtype=torch.bfloat16,
                                                 device="cuda")) for n in ("gate", "up"))
    h = rfq.rfq_swiglu_quantize_act(g, u)[:4]
    z = rfq.rfq_gemm_experts(*h, *w["down"], plan.offsets, out_dtype=torch.bfloat16)
    return weights, experts, plan, q, g, u, h, z, rfq.rfq_expert_combine(z, weights, plan)


def make(T, E, K, Nh, all_, seed):
    g = torch.Generator().manual_seed(seed)

    def weight(n, k):
        c, s = rfq.rfq_quantize_weight((0.05 * torch.randn((E * n, k), generator=g)).cuda())
        return c.view(E, n, k // 2), s.view(E, n, k // 32)
    w = {"gate": weight(Nh, K), "up": weight(Nh, K), "down": weight(K, Nh)}
    x = torch.randn((T, K), generator=g).bfloat16().cuda()
    return x, torch.randn((T, all_), generator=g).cuda(), w


@pytest.mark.parametrize("T,E,all_,first,k,K,Nh", [(1, 8, 8, 0, 2, 128, 64), (37, 8, 8, 0, 2, 256, 96),
                                                   (150, 8, 32, 16, 4, 512, 160),
                                                   (700, 4, 4, 0, 2, 256, 256)])
def test_layer(T, E, all_, first, k, K, Nh):
    x, logits, w = make(T, E, K, Nh, all_, T)
    weights, experts, plan, q, g, u, h, z, out = layer(x, logits, k, w, first)
    rw, rx, _ = ref.route(logits, k, True)
    assert torch.equal(experts.cpu().long(), rx)
    want = ref.sort(experts, E, first)
    assert all(torch.equal(a.cpu().long(), b) for a, b in zip(plan, want))
    # Each step against 64 bits from what the step before it gave.
    for z_, a, name, rows in ((g, q, "gate", plan.rows), (u, q, "up", plan.rows), (z, h, "down", None)):
        M = a[0].shape[0]
        v, bound, live = ref.product(a, w[name], plan.offsets, rows, M)
        err = (z_.double().cpu() - v).abs()
        assert (err <= TOL_SUM * bound + 2.0 ** -8 * v.abs())[live].all(), name
    s = plan.slots.cpu().long()
    taken = torch.where((s >= 0)[..., None], z.double().cpu()[s.clamp(min=0)], 0.0)
    f = weights.double().cpu()[..., None]
    v, size = (taken * f).sum(1), (taken * f).abs().sum(1)
    assert ((out.double().cpu() - v).abs() <= (k + 1) * 2.0 ** -24 * size + 2.0 ** -8 * v.abs()).all()


def test_layer_captured_with_new_inputs():
    x, logits, w = make(64, 8, 256, 96, 8, 3)
    layer(x, logits, 2, w, 0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(x, logits, 2, w, 0)[-1]
    for seed in (4, 5, 6):
        x2, logits2, _ = make(64, 8, 256, 96, 8, seed)
        x.copy_(x2)
        logits.copy_(logits2)
        graph.replay()
        want = layer(x, logits, 2, w, 0)[-1]
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_padded_tokens_and_masked_experts():
    """A padded token's row holds anything and its logits -infinity: its result is zeros, and
    nothing else changes.  A masked expert gets no token."""
    x, logits, w = make(50, 8, 256, 96, 8, 7)
    logits[:, 3] = -float("inf")
    _, first, plan1, q1, g1, *_ = layer(x, logits, 2, w, 0)
    pad = torch.tensor([0, 17, 49], device="cuda")
    x2, logits2 = x.clone(), logits.clone()
    x2[pad] = 3e38
    logits2[pad] = -float("inf")
    weights, experts, plan, _, g2, *_, out = layer(x2, logits2, 2, w, 0)
    assert (experts[pad] == -1).all() and (weights[pad] == 0).all() and (plan.slots[pad] == -1).all()
    assert (out[pad] == 0).all()
    keep = torch.ones(50, dtype=torch.bool, device="cuda")
    keep[pad] = False
    assert torch.equal(experts[keep], first[keep])
    # The slots move, and with them the order of the sums: either run's gate product is within
    # its sums' rounding and half a step of bf16 of the same value.
    s1, s2 = plan1.slots[keep].flatten().long(), plan.slots[keep].flatten().long()
    v, bound, _ = ref.product(q1, w["gate"], plan1.offsets, plan1.rows, 50)
    tol = 2 * (TOL_SUM * bound + 2.0 ** -8 * v.abs())
    assert ((g1[s1] - g2[s2]).abs().double().cpu() <= tol[s1.cpu()]).all()
    ends = plan.offsets.tolist()
    assert ends[3] == ends[4] and ends[8] == 94


def test_layer_of_one_token_and_one_expert():
    x, logits, w = make(1, 1, 64, 32, 1, 8)
    weights, experts, plan, q, g, u, h, z, out = layer(x, logits, 1, w, 0)
    assert weights.item() == 1.0 and experts.item() == 0 and plan.offsets.tolist() == [0, 1]
    assert torch.equal(out, z)
