"""Pairs sorted by expert against the definition: whole layers and shares of them, dropped
pairs, one workgroup and several, graphs and streams."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu


def same(plan, want):
    assert all(t.dtype == torch.int32 for t in plan)
    for a, b, name in zip(plan, want, plan._fields):
        assert torch.equal(a.cpu().long(), b), name


def stable(x, E, first=0):
    """The definition through a stable sort, for many pairs."""
    T, k = x.shape
    e = x.cpu().long().flatten() - first
    e = torch.where((e >= 0) & (e < E), e, E)
    order = torch.sort(e, stable=True).indices
    key = e[order]
    slots = torch.empty_like(order)
    slots[order] = torch.where(key < E, torch.arange(T * k), -1)
    return (torch.searchsorted(key, torch.arange(E + 1)), torch.where(key < E, order // k, -1),
            slots.reshape(T, k))


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 8), (7, 3, 2), (64, 8, 1), (65, 60, 4),
                                   (200, 128, 8), (129, 1024, 7), (1000, 257, 3)])
def test_whole_layers(T, E, k):
    x = ref.choices(T, E, k, T)
    same(rfq.rfq_expert_sort(x.cuda(), E), ref.sort(x, E))


@pytest.mark.parametrize("T,E,k,all_,first", [(50, 16, 4, 64, 16), (33, 1, 2, 9, 8), (40, 8, 4, 64, 60),
                                              (40, 8, 4, 64, -3)])
def test_shares_of_layers_and_dropped_pairs(T, E, k, all_, first):
    x = ref.choices(T, all_, k, first + 10)
    x[3] = -1
    x[5, 0] = 2 ** 31 - 1
    x[6, 0] = -2 ** 31
    same(rfq.rfq_expert_sort(x.cuda(), E, first=first), ref.sort(x, E, first))


def test_one_expert_for_all_and_none():
    x = torch.full((300, 2), 5, dtype=torch.int32)
    same(rfq.rfq_expert_sort(x.cuda(), 8), ref.sort(x, 8))
    same(rfq.rfq_expert_sort(x.cuda(), 4), ref.sort(x, 4))         # all dropped
    x[:, 1] = torch.arange(300) % 8
    same(rfq.rfq_expert_sort(x.cuda(), 8), ref.sort(x, 8))         # a pair's expert twice


@pytest.mark.parametrize("T,E,k", [(1024, 8, 8), (1025, 64, 8), (8193, 128, 1), (5000, 1000, 3),
                                   (40000, 256, 8), (30011, 5, 16)])
def test_many_pairs_in_several_workgroups_and_in_one(T, E, k):
    x = ref.choices(T, max(E, k) + 3, k, T)
    want = stable(x, E)
    nbytes = rfq.rfq_expert_sort_workspace_bytes(T, k, E)
    assert (nbytes > 0) == (T * k > 8192)
    same(rfq.rfq_expert_sort(x.cuda(), E), want)
    # Too small a workspace: one workgroup.
    same(rfq.rfq_expert_sort(x.cuda(), E, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
         want)


def test_captured_graphs_share_a_workspace():
    T, E, k = 3000, 64, 4
    work = torch.empty(rfq.rfq_expert_sort_workspace_bytes(T, k, E), dtype=torch.uint8, device="cuda")
    xs = [ref.choices(T, E, k, s).cuda() for s in range(2)]
    rfq.rfq_expert_sort(xs[0], E, workspace=work)
    torch.cuda.synchronize()
    graphs = []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            plan = rfq.rfq_expert_sort(x, E, workspace=work)
        graphs.append((g, x, plan))
    for seed in (5, 6):
        for i, (g, x, plan) in enumerate(graphs):
            x.copy_(ref.choices(T, E, k, 10 * seed + i))
            g.replay()
            same(plan, stable(x, E))
            work.random_(0, 256)


def test_on_another_stream():
    x = ref.choices(3000, 64, 4, 8).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan = rfq.rfq_expert_sort(x, 64, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    same(plan, stable(x, 64))


def test_empty_and_refusals():
    plan = rfq.rfq_expert_sort(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 8)
    assert plan.offsets.tolist() == [0] * 9 and plan.rows.numel() == 0
    assert plan.slots.shape == (0, 4)
    x = ref.choices(4, 8, 2, 0).cuda()
    for E in (0, -1, 1025):
        with pytest.raises(ValueError, match="n_experts"):
            rfq.rfq_expert_sort(x, E)
    with pytest.raises(TypeError):
        rfq.rfq_expert_sort(x.long(), 8)
    with pytest.raises(ValueError, match="2-D"):
        rfq.rfq_expert_sort(x[0], 8)
    with pytest.raises(rfq.RfqError, match="RFQ_ERR_SHAPE"):
        rfq.rfq_expert_sort(torch.zeros((2, 17), dtype=torch.int32, device="cuda"), 8)
    with pytest.raises(rfq.RfqError, match="RFQ_ERR_SHAPE"):
        rfq.rfq_expert_sort(x, 8, first=2 ** 31)
