"""Host-side argument checks of the calls around a layer of experts: every refusal happens
before a device is touched, empty work is a no-op.  No call here reaches a launch."""
import pytest

from paper_2608_26581_amd import rfq as binding

OK, ENULL, ESHAPE, EDTYPE, EALIGN, EDEVICE = range(6)
A, MIS = 0x10000, 0x10004                    # addresses never dereferenced


def _caller(func, args):
    def call(**kw):
        a = dict(args)
        a.update(kw)
        return getattr(binding.load(), func)(*a.values())
    return call


def _all(call, status, *cases):
    for kw in cases:
        assert call(**kw) == status, kw


def test_route():
    call = _caller("rfq_route", dict(l=A, dt=1, T=0, E=64, k=8, renorm=1, w=A, x=A, s=None))
    assert call() == OK and call(l=None, w=None, x=None) == OK and call(dt=0) == OK
    _all(call, EDTYPE, dict(dt=2), dict(dt=-1))
    _all(call, ESHAPE, dict(T=-1), dict(E=0), dict(E=1025), dict(k=0), dict(k=-1), dict(k=17),
         dict(E=7), dict(T=1 << 28, k=8), dict(T=1 << 26, k=1), dict(T=1 << 62))
    _all(call, ENULL, *(dict(T=4, **{n: None}) for n in "lwx"))
    _all(call, EALIGN, dict(T=4, l=A + 1), dict(T=4, dt=0, l=A + 2), dict(T=4, w=A + 2),
         dict(T=4, x=A + 1))


def test_route_backward():
    call = _caller("rfq_route_backward", dict(d=A, l=A, dt=1, T=0, E=64, k=8, w=A, x=A, renorm=1,
                                              o=A, s=None))
    assert call() == OK and call(d=None, l=None, w=None, x=None, o=None) == OK
    _all(call, EDTYPE, dict(dt=7))
    _all(call, ESHAPE, dict(T=-1), dict(E=0), dict(E=2000), dict(k=0), dict(k=17), dict(E=7),
         dict(T=1 << 28))
    _all(call, ENULL, *(dict(T=4, **{n: None}) for n in "dlwxo"))
    _all(call, EALIGN, dict(T=4, d=A + 1), dict(T=4, l=A + 1), dict(T=4, w=A + 2),
         dict(T=4, x=A + 3), dict(T=4, o=A + 1), dict(T=4, dt=0, o=A + 2))


def test_sort():
    call = _caller("rfq_expert_sort", dict(x=A, T=4, k=2, first=0, E=8, o=A, r=A, sl=A, w=None,
                                           nb=0, s=None))
    _all(call, ESHAPE, dict(T=-1), dict(k=0), dict(k=17), dict(E=0), dict(E=1025), dict(nb=-1),
         dict(first=1 << 31), dict(first=-(1 << 31) - 1), dict(T=1 << 30))
    _all(call, ENULL, dict(x=None), dict(o=None), dict(r=None), dict(sl=None), dict(nb=16),
         dict(T=0, o=None))
    _all(call, EALIGN, dict(x=A + 2), dict(o=A + 1), dict(r=A + 2), dict(sl=A + 3),
         dict(w=MIS, nb=16))
    size = binding.load().rfq_expert_sort_workspace_bytes
    assert size(1024, 8, 256) == 0 < size(1025, 8, 256) and size(1 << 20, 8, 64) <= 128 * 64 * 4
    assert size(-1, 8, 256) == size(5000, 17, 256) == size(5000, 8, 0) == size(1 << 40, 8, 8) == 0


def test_gather():
    call = _caller("rfq_expert_gather", dict(x=A, dt=1, T=4, N=64, r=A, sl=A, k=2, P=0, o=A, s=None))
    assert call() == OK and call(N=0, P=3, x=None, r=None, sl=None, o=None) == OK
    _all(call, EDTYPE, dict(dt=2))
    _all(call, ESHAPE, dict(T=-1), dict(P=-1), dict(N=-1), dict(T=1 << 31), dict(P=1 << 31),
         dict(N=1 << 31), dict(T=1 << 26), dict(T=1 << 20, N=1 << 20), dict(P=(1 << 30) + 64),
         dict(k=0), dict(k=17))
    _all(call, ENULL, dict(P=3, x=None), dict(P=3, r=None), dict(P=3, sl=None), dict(P=3, o=None))
    _all(call, EALIGN, dict(P=3, x=MIS), dict(P=3, r=A + 2), dict(P=3, sl=A + 1), dict(P=3, o=MIS))


def test_combine():
    call = _caller("rfq_expert_combine", dict(z=A, dt=1, P=8, N=64, sl=A, w=A, T=0, k=2, o=A, s=None))
    assert call() == OK and call(N=0, T=3, z=None, sl=None, w=None, o=None) == OK
    _all(call, EDTYPE, dict(dt=2))
    _all(call, ESHAPE, dict(T=-1), dict(P=-1), dict(N=-1), dict(k=0), dict(k=17), dict(T=1 << 26),
         dict(P=1 << 31), dict(T=1 << 20, N=1 << 20))
    _all(call, ENULL, dict(T=3, z=None), dict(T=3, sl=None), dict(T=3, o=None))
    _all(call, EALIGN, dict(T=3, z=MIS), dict(T=3, sl=A + 2), dict(T=3, w=A + 1), dict(T=3, o=MIS))


def test_combine_backward():
    call = _caller("rfq_expert_combine_backward",
                   dict(d=A, z=A, dt=1, P=8, N=64, r=A, sl=A, w=A, T=4, k=2, dz=A, dw=A, s=None))
    assert call(dz=None, dw=None) == OK and call(T=0, P=0) == OK
    assert call(P=0, dw=None) == OK and call(T=0, dz=None) == OK and call(N=0, dw=None) == OK
    _all(call, EDTYPE, dict(dt=2))
    _all(call, ESHAPE, dict(T=-1), dict(P=-1), dict(N=-1), dict(k=0), dict(k=17), dict(T=1 << 24),
         dict(P=1 << 31), dict(P=(1 << 30) - 64))
    _all(call, ENULL, dict(d=None), dict(z=None), dict(sl=None), dict(r=None))
    _all(call, EALIGN, dict(d=MIS), dict(z=MIS), dict(r=A + 2), dict(sl=A + 2), dict(w=A + 1),
         dict(dz=MIS), dict(dw=A + 2))


@pytest.mark.parametrize("func", ["gather", "combine", "combine_backward"])
def test_rows_whose_pieces_pass_32_bits(func):
    args = {"gather": dict(x=A, dt=1, T=0, N=64, r=A, sl=A, k=2, P=0, o=A, s=None),
            "combine": dict(z=A, dt=1, P=8, N=64, sl=A, w=A, T=0, k=2, o=A, s=None),
            "combine_backward": dict(d=A, z=A, dt=1, P=0, N=64, r=A, sl=A, w=A, T=0, k=2, dz=A,
                                     dw=A, s=None)}[func]
    call = _caller("rfq_expert_" + func, args)
    most = (1 << 31) - 257                   # N + 256 below 2^31
    assert call(N=most) == OK and call(N=most, dt=0) == OK
    _all(call, ESHAPE, *(dict(N=n, dt=dt) for dt in (0, 1)
                         for n in (most + 1, most + 2, (1 << 31) - 8, (1 << 31) - 1)))


def test_product():
    call = _caller("rfq_gemm_experts",
                   dict(qc=A, qs=A, rc=A, rs=A, wc=A, ws=A, off=A, rows=A, M=4, P=0, E=2, N=64, K=64,
                        z=A, dt=1, s=None))
    none = dict(qc=None, qs=None, rc=None, rs=None, wc=None, ws=None, off=None, z=None)
    assert call() == OK and call(**none) == OK
    assert call(P=4, N=0, **none) == OK and call(P=4, E=0, **none) == OK
    assert call(rows=None, M=0, **none) == OK
    assert call(M=0) == OK and call(M=0, P=4, E=0) == OK
    _all(call, EDTYPE, dict(dt=2))
    _all(call, ESHAPE, dict(M=0, P=4), dict(M=-1), dict(P=-1), dict(E=-1), dict(N=-1), dict(K=0), dict(K=48),
         dict(E=1025), dict(rows=None, P=3), dict(M=1 << 31), dict(P=1 << 31), dict(N=1 << 31),
         dict(M=1 << 27), dict(N=1 << 27), dict(P=1 << 30, N=1 << 20), dict(K=1 << 32))
    _all(call, ENULL, *(dict(P=4, **{n: None}) for n in ("qc", "qs", "rc", "rs", "wc", "ws", "off", "z")))
    _all(call, EALIGN, *(dict(P=4, **{n: MIS}) for n in ("qc", "qs", "rc", "rs", "wc", "ws", "z")),
         dict(P=4, off=A + 2), dict(P=4, rows=A + 1))


@pytest.mark.parametrize("func,args", [
    ("rfq_route", (A, 1, 4, 64, 8, 1, A, A, None)),
    ("rfq_expert_sort", (A, 4, 2, 0, 8, A, A, A, None, 0, None)),
    ("rfq_expert_gather", (A, 1, 4, 64, A, A, 2, 3, A, None)),
    ("rfq_gemm_experts", (A, A, A, A, A, A, A, A, 4, 4, 2, 64, 64, A, 1, None)),
])
def test_a_call_without_a_device_is_refused(func, args):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    assert getattr(binding.load(), func)(*args) == EDEVICE
