"""No call around a layer of experts writes outside its outputs: guard bytes before and after
every output, through the C ABI, at sizes that end inside tiles, pieces and waves."""
import pytest
import torch

import experts_util as ref
import paper_2608_26581_amd as rfq
from paper_2608_26581_amd import rfq as binding

pytestmark = pytest.mark.gpu

GUARD, BYTE = 256, 0xA5


class Guarded:
    """`n` bytes at 16-byte alignment between guards."""

    def __init__(self, n):
        self.n = n
        self.all = torch.full((GUARD + n + GUARD,), BYTE, dtype=torch.uint8, device="cuda")
        self.ptr = self.all.data_ptr() + GUARD

    def check(self, what):
        torch.cuda.synchronize()
        assert (self.all[:GUARD] == BYTE).all() and (self.all[GUARD + self.n:] == BYTE).all(), what

    def as_(self, dtype):
        return self.all[GUARD:GUARD + self.n].view(dtype)


def call(name, *args):
    st = getattr(binding.load(), name)(*args, torch.cuda.current_stream().cuda_stream)
    assert st == 0, (name, st)


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (33, 60, 4), (129, 128, 8), (5, 1000, 16), (3000, 17, 3)])
def test_router_and_sort(T, E, k):
    l = torch.randn((T, E), device="cuda")
    for code, t in ((0, l), (1, l.bfloat16())):
        w, x, d = Guarded(4 * T * k), Guarded(4 * T * k), Guarded(t.element_size() * T * E)
        call("rfq_route", t.data_ptr(), code, T, E, k, code, w.ptr, x.ptr)
        call("rfq_route_backward", w.ptr, t.data_ptr(), code, T, E, k, w.ptr, x.ptr, code, d.ptr)
        for g, n in ((w, "weights"), (x, "experts"), (d, "dlogits")):
            g.check(n)
    experts = x.as_(torch.int32).clone()
    for nbytes in (0, binding.load().rfq_expert_sort_workspace_bytes(T, k, E)):
        off, rows, slots, work = Guarded(4 * E + 4), Guarded(4 * T * k), Guarded(4 * T * k), Guarded(nbytes)
        call("rfq_expert_sort", experts.data_ptr(), T, k, 0, E, off.ptr, rows.ptr, slots.ptr,
             work.ptr if nbytes else None, nbytes)
        for g, n in ((off, "offsets"), (rows, "rows"), (slots, "slots"), (work, "workspace")):
            g.check(n)


@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (7, 3, 5), (40, 2, 264), (13, 8, 1032), (9, 16, 100)])
@pytest.mark.parametrize("code", [0, 1])
def test_rows(T, k, N, code):
    dtype = (torch.float32, torch.bfloat16)[code]
    plan = ref.plan_tensors(ref.sort(ref.choices(T, 20, k, T), 13))
    _, rows, slots = plan
    P, size = T * k, dtype.itemsize
    x, z = torch.randn((T, N), device="cuda").to(dtype), torch.randn((P, N), device="cuda").to(dtype)
    w = torch.rand((T, k), device="cuda")
    xs, out, dz, dw = Guarded(P * N * size), Guarded(T * N * size), Guarded(P * N * size), Guarded(4 * P)
    call("rfq_expert_gather", x.data_ptr(), code, T, N, rows.data_ptr(), slots.data_ptr(), k, P, xs.ptr)
    call("rfq_expert_combine", z.data_ptr(), code, P, N, slots.data_ptr(), w.data_ptr(), T, k, out.ptr)
    call("rfq_expert_combine_backward", x.data_ptr(), z.data_ptr(), code, P, N, rows.data_ptr(),
         slots.data_ptr(), w.data_ptr(), T, k, dz.ptr, dw.ptr)
    for g, n in ((xs, "gather"), (out, "combine"), (dz, "dz"), (dw, "dweights")):
        g.check(n)


@pytest.mark.parametrize("lengths,N,K", [([1], 1, 32), ([3, 0, 2], 33, 128), ([17, 16, 40], 70, 96),
                                         ([130, 1, 300], 257, 512), ([2, 30], 5, 4224),
                                         ([700, 400], 8201, 64)])
@pytest.mark.parametrize("code", [0, 1])
def test_product(lengths, N, K, code):
    P, E = sum(lengths), len(lengths)
    a, w = ref.codes((P,), K, 1), ref.codes((E, N), K, 2, None)
    off = torch.tensor([0] + lengths).cumsum(0).int().cuda()
    z = Guarded(P * N * (4, 2)[code])
    call("rfq_gemm_experts", *(t.data_ptr() for t in (*a, *w, off)), None, P, P, E, N, K, z.ptr, code)
    z.check("product")
    got = z.as_((torch.float32, torch.bfloat16)[code]).view(P, N)
    want = rfq.rfq_gemm_experts(*a, *w, off, out_dtype=got.dtype)
    assert torch.equal(got, want)
