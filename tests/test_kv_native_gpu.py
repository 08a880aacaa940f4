"""The native calls of the key/value cache against the binding's Python path (which an
explicit stream takes): the same results, the caller's own outputs returned, and
tensors that are not the common form left to the Python path."""
import pytest
import torch

import paper_2608_26581_amd as rfq
from paper_2608_26581_amd import kv
from paper_2608_26581_amd import rfq as binding

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    pass


def _same(a, b):
    a, b = [x if isinstance(x, tuple) else (x,) for x in (a, b)]
    assert len(a) == len(b)
    for s, t in zip(a, b):
        assert (s is None) == (t is None)
        if s is not None:
            assert s.dtype == t.dtype and s.shape == t.shape and s.stride() == t.stride()
            assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))


def _served(monkeypatch, names):
    """Fails where one of these calls goes on in Python."""
    binding.load()
    assert binding._calls
    real = kv._native

    def native(func, *args):
        r = real(func, *args)
        assert r is not None or func not in names, func
        return r
    monkeypatch.setattr(kv, "_native", native)


def _inputs():
    g = torch.Generator(device="cuda").manual_seed(1)
    T, Hq, heads, D, page = 24, 8, 2, 128, 16
    x = torch.randn((T, Hq + 2 * heads, D), generator=g, device="cuda").bfloat16()
    cache = rfq.kv_cache(6, heads, page, D)
    for p in cache:
        p.zero_()
    return T, x[:, :Hq], x[:, Hq:Hq + heads], x[:, Hq + heads:], cache


def test_results_match(monkeypatch):
    _served(monkeypatch, ("block_assign", "block_release", "rope", "rope_backward", "kv_append",
                          "kv_gather", "kv_attention"))
    T, q, k, v, cache = _inputs()
    s = torch.cuda.current_stream()
    new = torch.tensor([5, 19], dtype=torch.int32, device="cuda")
    ctx = torch.zeros_like(new)
    free = torch.arange(6, dtype=torch.int32, device="cuda")
    count = torch.tensor([6], dtype=torch.int32, device="cuda")
    tables = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    args = (ctx, new, tables, free, count, 16, T)
    a = rfq.rfq_block_assign(*args)
    _same(a, rfq.rfq_block_assign(*args, stream=s))
    slots, positions, seq, starts, counts = a
    ended = torch.tensor([1, 0], dtype=torch.uint8, device="cuda")
    back = (seq, ended, tables, free.clone(), counts[:1].clone(), 16)
    _same(rfq.rfq_block_release(*back), rfq.rfq_block_release(*back, stream=s))
    pos3 = torch.stack((positions, positions // 2, positions % 7))
    cs, axes = rfq.rope_table(64, 128), rfq.rope_axes((16, 24, 24))
    for f in (rfq.rfq_rope, rfq.rfq_rope_backward):
        for inter in (False, True):
            _same(f(q, pos3, cs, axes, interleaved=inter),
                  f(q, pos3, cs, axes, interleaved=inter, stream=s))
        _same(f(q, positions, cs), f(q, positions, cs, stream=s))
        out = torch.empty_like(q)
        assert f(q, positions, cs, out=out) is out
        _same(out, f(q, positions, cs, stream=s))
    kw = dict(q=q, positions=pos3, cos_sin=cs, axes=axes)
    y = rfq.rfq_kv_append(k, v, slots, cache, **kw)
    held = [p.clone() for p in cache]
    _same(y, rfq.rfq_kv_append(k, v, slots, cache, stream=s, **kw))
    _same(tuple(held), tuple(cache))
    out = torch.empty_like(y)
    assert rfq.rfq_kv_append(k, v, slots, cache, q_out=out, **kw) is out
    _same(out, y)
    assert rfq.rfq_kv_append(k, v, slots, cache) is None
    for dt in (torch.bfloat16, torch.float32):
        _same(rfq.rfq_kv_gather(cache, slots, dt), rfq.rfq_kv_gather(cache, slots, dt, stream=s))
    at = (y, cache, tables, seq, starts, 19, 300)
    for kw in (dict(), dict(return_lse=True), dict(causal=False, window=4, scale=0.3)):
        _same(rfq.rfq_kv_attention(*at, **kw), rfq.rfq_kv_attention(*at, stream=s, **kw))
    ws = torch.empty(rfq.rfq_kv_attention_workspace_bytes(T, 8, 2, 128, 2, 19, 300),
                     dtype=torch.uint8, device="cuda")
    assert rfq.rfq_kv_attention(*at, out=out, workspace=ws) is out
    got, lse = rfq.rfq_kv_attention(*at, out=out, return_lse=True)
    assert got is out and lse.shape == (T, 8)
    _same(out, rfq.rfq_kv_attention(*at, stream=s))


def test_other_forms_go_through_python():
    T, q, k, v, cache = _inputs()
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    pos, cs = slots % 9, rfq.rope_table(9, 128)
    ref = rfq.rfq_rope(q, pos, cs)
    _same(rfq.rfq_rope(q.as_subclass(Sub), pos, cs).as_subclass(torch.Tensor), ref)
    _same(rfq.rfq_rope(q, pos, cs, [0] * 64), ref)               # a list of axes
    rfq.rfq_kv_append(k, v, slots, list(cache))
    with pytest.raises(ValueError, match="must be a device tensor"):
        rfq.rfq_rope(q.cpu(), pos, cs)
    with pytest.raises(ValueError):
        rfq.rfq_kv_gather(cache[:3], slots)
    with pytest.raises(ValueError, match="channels"):
        rfq.rfq_kv_attention(q[..., :0], cache, slots[None], slots[:1], slots[:2], 1, 1, scale=1.0)


def test_given_outputs_count_as_written():
    """A tensor saved for a backward pass and then given as an output is noticed there."""
    T, q, k, v, cache = _inputs()
    slots = torch.arange(T, dtype=torch.int32, device="cuda")
    pos, cs = slots % 9, rfq.rope_table(9, 128)
    tables = torch.arange(2, dtype=torch.int32, device="cuda")[None]
    lens, starts = torch.tensor([T], dtype=torch.int32, device="cuda"), slots[[0, -1]] + slots[:2]
    for stream in (None, torch.cuda.current_stream()):
        out = torch.empty_like(q)
        seen = out._version
        rfq.rfq_kv_append(k, v, slots, cache, q=q, positions=pos, cos_sin=cs, q_out=out,
                          stream=stream)
        assert out._version > seen
        seen = out._version
        rfq.rfq_kv_attention(q, cache, tables, lens, starts, T, T, out=out, stream=stream)
        assert out._version > seen
