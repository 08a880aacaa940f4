"""Calls on a stream that is not torch's current one: the memory that they take belongs to
that stream's order, so that nothing on the current stream gets it while the call
still works on it, and results are the current stream's."""
import pytest
import torch

import paper_2608_26581_amd as rfq

pytestmark = pytest.mark.gpu


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _calls():
    """(name, f(stream)) of every call that takes memory of its own."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    x, w = randn(40, 2048).bfloat16(), randn(96, 2048)
    q, wq = rfq.rfq_quantize_act(x), rfq.rfq_quantize_weight(w)
    h, hw = rfq.rfq_hif4_quantize(x), rfq.rfq_hif4_quantize(w, residual=False)[:2]
    wgu = tuple(t[:64].contiguous() for t in wq)
    gate, up = randn(24, 64).bfloat16(), randn(24, 64).bfloat16()
    phi = rfq.rfq_fallback_map(q[2], q[1], rfq.RFQ_PHI_RESIDUAL_NONZERO)
    T, Hq, heads, D = 3, 8, 2, 128
    cache = rfq.kv_cache(200, heads, 16, D)
    for p in cache:
        p.random_(118, 126, generator=g)
    tables = torch.randperm(200, generator=g, device="cuda").int().view(1, 200)
    qh, kh = randn(T, Hq, D).bfloat16(), randn(T, heads, D).bfloat16()
    pos, cs = _ints(5, 6, 7), rfq.rope_table(9, D)
    slots, free, count = _ints(3197, 3198, 3199), torch.arange(9, device="cuda").int(), _ints(9)
    ctx, new, table, held = _ints(3), _ints(20), _ints(7, -1)[None], _ints(7, 8)[None]
    ended, left, w16 = torch.ones(1, dtype=torch.uint8, device="cuda"), _ints(7), w.bfloat16()
    lens, starts = _ints(3200), _ints(0, 3)

    return [
        ("quantize_act", lambda s: rfq.rfq_quantize_act(x, stream=s)),
        ("quantize_weight", lambda s: rfq.rfq_quantize_weight(w, stream=s)),
        ("gemm", lambda s: rfq.rfq_gemm(*q, *wq, stream=s)),
        ("gemm split", lambda s: rfq.rfq_gemm(*q, *wq, split=True, stream=s)),
        ("gemm_split_noalloc", lambda s: rfq.rfq_gemm_split_noalloc(*q, *wq, stream=s)),
        ("gemm_split", lambda s: rfq.rfq_gemm_split(*q, *wq, None, stream=s)),
        ("gemm_stream", lambda s: rfq.rfq_gemm_stream(x[:4], *wq, stream=s)),
        ("gemm_phi", lambda s: rfq.rfq_gemm_phi(*q, *wq, phi, stream=s)),
        ("fallback_map", lambda s: rfq.rfq_fallback_map(q[2], q[1], 0, stream=s)),
        ("dequant", lambda s: rfq.rfq_dequant(q[0], q[1], stream=s)),
        ("swiglu", lambda s: rfq.rfq_swiglu_quantize_act(gate, up, return_h=True, stream=s)),
        ("gemm_swiglu", lambda s: rfq.rfq_gemm_swiglu_quantize(*q, *wgu, return_h=True, stream=s)),
        ("hif4_quantize", lambda s: rfq.rfq_hif4_quantize(x, stream=s)),
        ("hif4_dequant", lambda s: rfq.rfq_hif4_dequant(*hw, stream=s)),
        ("hif4_gemm", lambda s: rfq.rfq_hif4_gemm(*h, *hw, stream=s)),
        ("hif4_gemm split", lambda s: rfq.rfq_hif4_gemm(*h, *hw, split=True, stream=s)),
        ("hif4_gemm_split", lambda s: rfq.rfq_hif4_gemm_split(*h, *hw, None, stream=s)),
        ("hif4_gemm_wbf16", lambda s: rfq.rfq_hif4_gemm_wbf16(*h, w16, stream=s)),
        ("block_assign", lambda s: rfq.rfq_block_assign(
            ctx, new, table, free, count, 16, 20, stream=s)),
        ("block_release", lambda s: rfq.rfq_block_release(
            new, ended, held, free, left, 16, stream=s)),
        ("rope", lambda s: rfq.rfq_rope(qh, pos, cs, stream=s)),
        ("rope_backward", lambda s: rfq.rfq_rope_backward(qh, pos, cs, stream=s)),
        ("kv_append", lambda s: rfq.rfq_kv_append(kh, kh, slots, cache, q=qh, positions=pos,
                                                  cos_sin=cs, stream=s)),
        ("kv_gather", lambda s: rfq.rfq_kv_gather(cache, slots, stream=s)),
        ("kv_attention", lambda s: rfq.rfq_kv_attention(
            qh, cache, tables, lens, starts, 3, 3200, return_lse=True, stream=s)),
    ]


def _tensors(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


def test_memory_is_taken_on_the_calls_stream(monkeypatch):
    calls = _calls()
    s = torch.cuda.Stream()
    taken = []
    real = torch.empty

    def empty(*args, **kw):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return real(*args, **kw)
    for name, f in calls:
        want = [t.clone() for t in _tensors(f(None))]
        s.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        monkeypatch.setattr(torch, "empty", empty)
        taken.clear()
        got = f(s)
        monkeypatch.setattr(torch, "empty", real)
        assert taken and set(taken) == {s.cuda_stream}, name
        s.synchronize()
        got = _tensors(got)
        assert len(got) == len(want), name
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name
    # The current stream's own handle, and a handle of another kind, work as well.
    for stream in (torch.cuda.current_stream(), torch.cuda.ExternalStream(s.cuda_stream)):
        s.wait_stream(torch.cuda.current_stream())
        assert len(_tensors(calls[0][1](stream))) == 4
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", ["kv_attention", "gemm split", "hif4_gemm split"])
def test_a_waiting_call_keeps_its_memory(name):
    """The stream is busy with something else when the call is made and the current stream
    takes as much memory as it can get of the sizes in question meanwhile."""
    f = dict(_calls())[name]
    want = [t.clone() for t in _tensors(f(None))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(5000000)
    got = _tensors(f(s))
    others = [torch.full((1 << k,), 255, dtype=torch.uint8, device="cuda")
              for k in range(9, 25) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.all(t == 255) for t in others)
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
