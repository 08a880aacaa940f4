"""Host-side argument checks of the key/value cache calls: every refusal happens before
a device is touched, empty work is a no-op.  No call here reaches a launch."""
import ctypes

import pytest

from paper_2608_26581_amd import rfq as binding

OK, ENULL, ESHAPE, EDTYPE, EALIGN = range(5)
A, MIS = 0x10000, 0x10004                    # addresses never dereferenced


def _heads(data=A, ts=1024, hs=128):
    return ctypes.byref(binding.Heads(data, ts, hs))


def _spec(**kw):
    f = dict(positions=A, positions_stride=8, cos_sin=A, max_pos=100, axes=None, n_axes=1,
             rotary=128, interleaved=0)
    f.update(kw)
    return ctypes.byref(binding.RopeSpec(*f.values()))


def _cache(**kw):
    f = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, blocks=10, heads=2, page=16, D=128)
    f.update(kw)
    return ctypes.byref(binding.KvCacheArgs(*f.values()))


def _caller(func, args):
    def call(**kw):
        a = dict(args)
        a.update(kw)
        return getattr(binding.load(), func)(*a.values())
    return call


@pytest.mark.parametrize("func", ["rfq_rope", "rfq_rope_backward"])
def test_rope(func):
    call = _caller(func, dict(x=_heads(), dt=1, T=0, H=8, D=128, rope=_spec(), y=_heads(), s=None))
    assert call() == OK and call(T=4, H=0) == OK
    assert call(x=_heads(None), y=_heads(None), rope=_spec(positions=None, cos_sin=None)) == OK
    assert call(dt=2) == EDTYPE and call(dt=-1) == EDTYPE
    assert call(x=None) == ENULL and call(y=None) == ENULL and call(rope=None) == ENULL
    for kw in (dict(T=-1), dict(H=-1), dict(D=0), dict(D=120), dict(D=528), dict(T=1 << 40),
               dict(H=1 << 20), dict(x=_heads(ts=-8), T=4), dict(T=4, y=_heads(ts=0)),
               dict(T=4, y=_heads(hs=0)), dict(x=_heads(hs=1 << 50), T=4)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(rotary=0), dict(rotary=24), dict(rotary=144), dict(n_axes=0), dict(n_axes=9),
               dict(max_pos=-1), dict(axes=bytes([0] * 63 + [1])), dict(positions_stride=-1)):
        assert call(rope=_spec(**kw)) == ESHAPE, kw
    assert call(rope=_spec(axes=bytes([2] * 64), n_axes=3)) == OK
    assert call(T=4, x=_heads(None)) == ENULL and call(T=4, y=_heads(None)) == ENULL
    assert call(T=4, rope=_spec(positions=None)) == ENULL
    assert call(T=4, rope=_spec(cos_sin=None)) == ENULL
    assert call(T=4, x=_heads(A + 8)) == EALIGN and call(T=4, y=_heads(A + 8)) == EALIGN
    assert call(T=4, x=_heads(ts=1028)) == EALIGN and call(T=4, y=_heads(hs=132)) == EALIGN
    assert call(T=4, rope=_spec(positions=A + 2)) == EALIGN
    assert call(T=4, rope=_spec(cos_sin=A + 4)) == EALIGN


def test_append():
    call = _caller("rfq_kv_append", dict(k=_heads(), v=_heads(), dt=1, T=0, slots=A, cache=_cache(),
                                         q=_heads(), Hq=4, rope=_spec(), q_out=_heads(), s=None))
    assert call() == OK and call(q=None, q_out=None) == OK
    assert call(q=None, q_out=None, rope=None) == OK
    assert call(dt=3) == EDTYPE
    for kw in (dict(k=None), dict(v=None), dict(cache=None), dict(q=None), dict(q_out=None),
               dict(rope=None)):
        assert call(**kw) == ENULL, kw
    for kw in (dict(D=96), dict(D=32), dict(page=8), dict(page=48), dict(page=512), dict(heads=0),
               dict(heads=1 << 20), dict(blocks=-1), dict(blocks=1 << 28)):
        assert call(cache=_cache(**kw)) == ESHAPE, kw
    for kw in (dict(T=-1), dict(Hq=-1), dict(Hq=1 << 20), dict(T=1 << 30),
               dict(rope=_spec(rotary=144)), dict(k=_heads(ts=-8), T=2), dict(v=_heads(hs=-8), T=2),
               dict(q_out=_heads(ts=0), T=2)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(k=_heads(None)), dict(v=_heads(None)), dict(slots=None), dict(q=_heads(None)),
               dict(q_out=_heads(None)), dict(cache=_cache(k_codes=None)),
               dict(cache=_cache(v_scales=None)), dict(rope=_spec(positions=None))):
        assert call(T=3, **kw) == ENULL, kw
    for kw in (dict(k=_heads(MIS)), dict(v=_heads(ts=1028)), dict(q=_heads(hs=132)),
               dict(q_out=_heads(MIS)), dict(slots=A + 1), dict(cache=_cache(k_scales=MIS)),
               dict(cache=_cache(v_codes=MIS))):
        assert call(T=3, **kw) == EALIGN, kw


def test_gather():
    call = _caller("rfq_kv_gather", dict(cache=_cache(), slots=A, n=0, k=A, v=A, dt=1, s=None))
    assert call() == OK and call(slots=None, k=None, v=None) == OK
    assert call(dt=2) == EDTYPE and call(cache=None) == ENULL
    assert call(n=-1) == ESHAPE and call(n=1 << 40) == ESHAPE
    assert call(cache=_cache(D=100)) == ESHAPE
    for kw in (dict(slots=None), dict(k=None), dict(v=None), dict(cache=_cache(k_codes=None))):
        assert call(n=3, **kw) == ENULL, kw
    for kw in (dict(slots=A + 2), dict(k=MIS), dict(v=MIS), dict(cache=_cache(k_codes=MIS))):
        assert call(n=3, **kw) == EALIGN, kw


def test_attention():
    args = dict(q=_heads(), T=0, Hq=8, cache=_cache(), tables=A, width=4, lens=A, starts=A, B=2,
                max_query=1, max_seq=64, scale=0.1, causal=1, window=0, out=_heads(), lse=A, ws=A,
                ws_bytes=1024, s=None)
    call = _caller("rfq_kv_attention", args)
    assert call() == OK and call(T=2, B=0) == OK
    assert call(q=None) == ENULL and call(cache=None) == ENULL and call(out=None) == ENULL
    for kw in (dict(T=-1), dict(B=-1), dict(T=1 << 24), dict(B=1 << 24), dict(Hq=7), dict(Hq=0),
               dict(Hq=1 << 17), dict(width=-1), dict(max_query=-1), dict(max_seq=-1),
               dict(window=-1), dict(ws_bytes=-1), dict(T=2, q=_heads(ts=-8)),
               dict(T=2, out=_heads(hs=0)), dict(T=2, cache=_cache(blocks=0)),
               dict(T=(1 << 24) - 1, Hq=512)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(D=32), dict(page=17), dict(heads=3)):
        assert call(cache=_cache(**kw)) == ESHAPE, kw
    for kw in (dict(q=_heads(None)), dict(out=_heads(None)), dict(lens=None), dict(starts=None),
               dict(tables=None), dict(ws=None), dict(cache=_cache(v_codes=None))):
        assert call(T=2, **kw) == ENULL, kw
    for kw in (dict(q=_heads(MIS)), dict(out=_heads(ts=1020)), dict(lens=A + 1), dict(starts=A + 2),
               dict(tables=A + 3), dict(lse=A + 1), dict(ws=A + 8),
               dict(cache=_cache(k_codes=MIS))):
        assert call(T=2, **kw) == EALIGN, kw


def test_attention_workspace():
    f = binding.load().rfq_kv_attention_workspace_bytes
    assert f(4, 32, 8, 128, 4, 1, 100000) > 0
    assert f(4, 32, 8, 128, 4, 1, 16) == 0                    # nothing to split
    for bad in ((4, 32, 8, 96, 4, 1, 100000), (-1, 32, 8, 128, 4, 1, 9999), (4, 33, 8, 128, 4, 1, 9999),
                (4, 32, 8, 128, -4, 1, 9999), (4, 32, 8, 128, 4, -1, 9999), (4, 32, 8, 128, 4, 1, -9),
                (0, 32, 8, 128, 4, 1, 9999), (4, 32, 8, 128, 0, 1, 9999), (4, 32, 0, 128, 4, 1, 9999)):
        assert f(*bad) == 0, bad


def test_attention_workspace_of_extreme_hints():
    """No request has more queries than q has rows, whatever the hint says."""
    f = binding.load().rfq_kv_attention_workspace_bytes
    for sizes in ((64, 2 ** 24 - 1, 1, 64, 2 ** 23), (2 ** 23, 255, 255, 128, 2 ** 24 - 1),
                  (2 ** 23, 255, 1, 256, 5), (700, 28, 4, 128, 2)):
        for max_seq in (0, 4096, 2 ** 62):
            want = f(*sizes, sizes[0], max_seq)
            assert want >= 0
            assert f(*sizes, 2 ** 31 - 1, max_seq) == want, (sizes, max_seq)


def test_block_calls():
    call = _caller("rfq_block_assign", dict(
        ctx=A, new=A, B=-1, tables=A, width=4, free=A, n_free=9, count=A, page=16, tokens=4,
        slots=A, pos=A, seq=A, starts=A, counts=A, s=None))
    for kw in (dict(), dict(B=16385), dict(B=2, width=-1), dict(B=2, n_free=-1),
               dict(B=2, tokens=-1), dict(B=2, tokens=1 << 31), dict(B=2, page=20),
               dict(B=2, page=8), dict(B=2, n_free=1 << 31)):
        assert call(**kw) == ESHAPE, kw
    for k in ("ctx", "new", "tables", "free", "count", "slots", "pos", "seq", "starts", "counts"):
        assert call(B=2, **{k: None}) == ENULL, k
        assert call(B=2, **{k: A + 2}) == EALIGN, k
    call = _caller("rfq_block_release", dict(lens=A, ended=A, B=-1, tables=A, width=4, free=A,
                                             n_free=9, count=A, page=16, out=A, s=None))
    for kw in (dict(), dict(B=16385), dict(B=2, width=-1), dict(B=2, n_free=-1), dict(B=2, page=0)):
        assert call(**kw) == ESHAPE, kw
    for k in ("lens", "ended", "tables", "free", "count", "out"):
        assert call(B=2, **{k: None}) == ENULL, k
        if k != "ended":
            assert call(B=2, **{k: A + 2}) == EALIGN, k


def test_largest_sizes():
    """The sizes that the header names are taken (a missing pointer is what is found next),
    the next ones refused."""
    rope = _caller("rfq_rope", dict(x=_heads(None), dt=1, T=4, H=8, D=128, rope=_spec(),
                                    y=_heads(None), s=None))
    assert rope(T=(1 << 24) - 1) == ENULL and rope(T=1 << 24) == ESHAPE
    assert rope(H=65536) == ENULL and rope(H=65537) == ESHAPE
    append = _caller("rfq_kv_append", dict(
        k=_heads(None), v=_heads(None), dt=1, T=4, slots=A, cache=_cache(heads=8), q=_heads(None),
        Hq=32, rope=_spec(), q_out=_heads(None), s=None))
    assert append(T=(1 << 23) - 1) == ENULL and append(T=1 << 23) == ESHAPE
    assert append(Hq=65536) == ENULL and append(Hq=65537) == ESHAPE
    assert append(cache=_cache(heads=65536)) == ENULL and append(cache=_cache(heads=65537)) == ESHAPE
    gather = _caller("rfq_kv_gather", dict(cache=_cache(heads=8), slots=None, n=4, k=A, v=A, dt=1,
                                           s=None))
    assert gather(n=(1 << 24) - 1) == ENULL and gather(n=1 << 24) == ESHAPE
    attention = _caller("rfq_kv_attention", dict(
        q=_heads(None), T=4, Hq=8, cache=_cache(), tables=A, width=4, lens=A, starts=A, B=2,
        max_query=1, max_seq=64, scale=0.1, causal=1, window=0, out=_heads(), lse=A, ws=A,
        ws_bytes=1024, s=None))
    assert attention(T=(1 << 24) - 1) == ENULL and attention(T=1 << 24) == ESHAPE
    assert attention(B=(1 << 24) - 1) == ENULL and attention(B=1 << 24) == ESHAPE
    assert attention(Hq=65536) == ENULL and attention(Hq=65538) == ESHAPE


def test_rows_and_tiles_stay_within_32_bits():
    """A request may have all T * Hq rows of one cached head, in tiles of up to 128 rows
    whose ends are counted in 32 bits: 2^31 - 1 - 127 rows at most."""
    most = 2 ** 31 - 1 - 127
    f = binding.load().rfq_kv_attention_workspace_bytes
    attention = _caller("rfq_kv_attention", dict(
        q=_heads(None), T=4, Hq=8, cache=_cache(heads=1), tables=A, width=4, lens=A, starts=A, B=2,
        max_query=1, max_seq=64, scale=0.1, causal=1, window=0, out=_heads(), lse=A, ws=A,
        ws_bytes=1024, s=None))
    for Hq in (49981, 65536, 32768, 128, 129, 1000):
        T = min(most // Hq, 2 ** 24 - 1)
        assert attention(T=T, Hq=Hq) == ENULL, Hq
        if T < 2 ** 24 - 1:
            assert attention(T=T + 1, Hq=Hq) == ESHAPE and f(T + 1, Hq, 1, 64, 2, T, 4096) == 0, Hq
    assert 42966 * 49981 < 2 ** 31 and attention(T=42966, Hq=49981) == ESHAPE
