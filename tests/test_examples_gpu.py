"""The examples, at small sizes."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

FOLDER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


def _load(name):
    spec = importlib.util.spec_from_file_location(name, os.path.join(FOLDER, name + ".py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# Relative error: the weights' and the results' rounding to bf16, 2^-9 each at most,
# and fp32 sums.
@pytest.mark.parametrize("requests,prompt,sizes", [
    (3, 60, dict(hidden=256, heads=4, kv_heads=2, D=64, page=16, picture=5)),
    (20, 40, dict(hidden=512, heads=8, kv_heads=1, D=128, page=32, picture=3)),
    (2, 300, dict(hidden=256, heads=2, kv_heads=2, D=256, page=64, picture=4)),
])
def test_decode(requests, prompt, sizes):
    _, errors = _load("decode").main(requests, prompt, 6, **sizes)
    assert len(errors) == 3 and max(errors) <= 2 * 2.0 ** -9 + 2.0 ** -12


def test_rope_gradient():
    losses = _load("rope_gradient").main(side=8, steps=10)
    assert losses[-1] < 0.5 * losses[0]


def test_decode_refused_request_keeps_its_history():
    """A request that outgrows its table is refused in later steps, in replayed ones too:
    it keeps its tokens, the refusals are counted, and all blocks come back."""
    block = _load("decode").Block(3, 32, hidden=256, heads=4, kv_heads=2, D=64, page=16, picture=2)
    lens = torch.tensor([29, 30, 7], dtype=torch.int32)
    block.step(torch.randn((66, 256), device="cuda").bfloat16(), lens.cuda(), 30, 32)
    x = torch.randn((3, 256), device="cuda").bfloat16()
    one = torch.ones(3, dtype=torch.int32, device="cuda")
    block.step(x, one, 1, 32)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.step(x, one, 1, 32)
    refused = 0
    for i in range(2, 7):
        graph.replay()
        want = [min(29 + i, 32), min(30 + i, 32), 7 + i]
        refused += (29 + i > 32) + (30 + i > 32)
        assert block.lens.tolist() == want and int(block.refused) == refused
        held = sum(-(-n // 16) for n in want)
        assert int(block.count) == block.free.shape[0] - held
    block.end(torch.ones(3, dtype=torch.uint8, device="cuda"))
    assert int(block.count) == block.free.shape[0] == block.free.unique().numel()
