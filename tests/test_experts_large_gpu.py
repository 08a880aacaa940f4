"""The calls around a layer of experts at sizes whose byte or element numbers pass 32 bits,
checked in the last rows and experts."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq
from gpu_util import TOL_SUM

pytestmark = pytest.mark.gpu


def _codes(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), generator=g, dtype=torch.uint8, device="cuda")
    s = torch.randint(125, 130, (*shape[:-1], shape[-1] // 32), generator=g, dtype=torch.uint8, device="cuda")
    return c, s


def test_product_with_weights_past_4_gib():
    E, N, K = 260, 16384, 2048                    # 4.4 GB of codes
    w = _codes((E, N, K), 1)
    lengths = [0] * E
    for e, n in ((0, 3), (E // 2, 20), (E - 2, 130), (E - 1, 7)):
        lengths[e] = n
    off = torch.tensor([0] + lengths).cumsum(0)
    P = int(off[-1])
    a = (*_codes((P, K), 2), *_codes((P, K), 3))
    z = rfq.rfq_gemm_experts(*a, *w, off.int().cuda())
    for e in (0, E // 2, E - 2, E - 1):
        i, j = int(off[e]), int(off[e + 1])
        part = [t[i:j] for t in a]
        sub = (w[0][e:e + 1, -300:], w[1][e:e + 1, -300:])
        want, bound, _ = ref.product(part, sub, torch.tensor([0, j - i]), None, j - i)
        assert ((z[i:j, -300:].double().cpu() - want).abs() <= TOL_SUM * bound).all(), e


@pytest.mark.parametrize("N,lengths", [(131073 + 64, [5, 0, 9]), (40000, [60000, 300])])
def test_product_with_wide_and_large_results(N, lengths):
    """More than 2048 column tiles; more than 2^31 results."""
    K = 64
    off = torch.tensor([0] + lengths).cumsum(0)
    P, E = int(off[-1]), len(lengths)
    a = (*_codes((P, K), 2), None, None)
    w = _codes((E, N, K), 1)
    z = rfq.rfq_gemm_experts(*a, *w, off.int().cuda(), out_dtype=torch.bfloat16)
    rows = torch.cat([torch.arange(max(int(off[e]), int(off[e + 1]) - 4), int(off[e + 1])) for e in range(E)])
    for r in rows.tolist():
        e = int((off[1:] <= r).sum())
        for n0 in (0, N // 2, N - 200):
            part = [t[r:r + 1] if t is not None else None for t in a]
            sub = (w[0][e:e + 1, n0:n0 + 200], w[1][e:e + 1, n0:n0 + 200])
            want, bound, _ = ref.product(part, sub, torch.tensor([0, 1]), None, 1)
            got = z[r:r + 1, n0:n0 + 200].double().cpu()
            assert ((got - want).abs() <= TOL_SUM * bound + 2.0 ** -8 * want.abs()).all(), (r, n0)


def test_rows_past_4_gib():
    T, E, k, N = 36000, 8, 8, 8192                # 2.4e9 elements in the slots
    experts = ref.choices(T, E, k, 1).cuda()
    plan = rfq.rfq_expert_sort(experts, E)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((T, N), generator=g, device="cuda", dtype=torch.bfloat16)
    xs = rfq.rfq_expert_gather(x, plan)
    for s in (0, T * k // 2, T * k - 3, T * k - 1):
        assert torch.equal(xs[s], x[plan.rows[s]])
    w = torch.softmax(torch.randn((T, k), generator=g, device="cuda"), 1)
    out = rfq.rfq_expert_combine(xs, w, plan)
    # Every slot of a token holds its row: the weights' sum (to 2^-23) times it.
    t = torch.tensor([0, T // 2, T - 1], device="cuda")
    want = x[t].double()
    assert ((out[t].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -20) * want.abs()).all()
    dz, dw = rfq.rfq_expert_combine_backward(x, xs, w, plan)
    norm = (x[t].double() ** 2).sum(1, keepdim=True)
    assert ((dw[t].double() - norm).abs() <= 2.0 ** -20 * norm).all()
    for i in t.tolist():
        got = dz[plan.slots[i].long()].double()
        want = w[i].double()[:, None] * x[i].double()
        assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all()


def test_router_past_4_gib():
    T, E, k = (1 << 22) + 5, 520, 3               # 2.2e9 logits
    l = torch.empty((T, E), dtype=torch.bfloat16, device="cuda").normal_()
    w, x = rfq.rfq_route(l, k, False)
    d = rfq.rfq_route_backward(w, l, w, x, False)
    for t in (0, T // 2, T - 1):
        rw, rx, _ = ref.route(l[t:t + 1], k, False)
        assert torch.equal(x[t].cpu().long(), rx[0])
        assert ((w[t].double().cpu() - rw[0]).abs() <= 2.0 ** -18 * rw[0]).all()
        p = torch.softmax(l[t].double(), 0)
        want = -p * (w[t].double() ** 2).sum()
        want[x[t].long()] += w[t].double() ** 2
        assert ((d[t].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * p).all()


def test_sort_of_many_pairs():
    T, k, E = 1 << 21, 8, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(-2, E + 2, (T, k), generator=g, device="cuda", dtype=torch.int32)
    plan = rfq.rfq_expert_sort(x, E)
    e = x.flatten().long()
    e = torch.where((e >= 0) & (e < E), e, E)
    order = torch.sort(e, stable=True).indices
    n = int((e < E).sum())
    assert torch.equal(plan.offsets.long(), torch.searchsorted(e[order], torch.arange(E + 1, device="cuda")))
    assert torch.equal(plan.rows[:n].long(), order[:n] // k) and (plan.rows[n:] == -1).all()
    slots = torch.full((T * k,), -1, device="cuda")
    slots[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(plan.slots.flatten().long(), slots)
