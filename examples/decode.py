"""A transformer's attention block that serves several requests from one 4-bit paged
key/value cache, with MXFP4 weights and RFQ activations:

    x, normalised -> q, k, v (RFQ product) -> blocks and slots of the step's tokens -> q and k
    rotated, k and v quantized into their slots -> attention over the cache -> output
    product (RFQ) -> x

First every request's prompt, ragged and all in one step; then decode steps of one
token a request, captured once in a graph and replayed, since lengths, blocks and
slots stay on the device; then half of the requests end, their blocks are given
back and new prompts take them.  Each prompt opens with a square picture, whose
tokens have a row and a column as positions (three position axes).

    python examples/decode.py [--requests 16] [--prompt 500] [--steps 64]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_26581_amd as rfq  # noqa: E402


class Block:
    """One attention block, its cache and the block tables of its requests."""

    def __init__(self, requests, max_tokens, hidden=4096, heads=32, kv_heads=8, D=128, page=32,
                 picture=12, device="cuda"):
        self.heads, self.kv_heads, self.D, self.page = heads, kv_heads, D, page
        self.picture = picture
        g = torch.Generator(device).manual_seed(0)

        def weight(n, k):
            w = torch.randn((n, k), generator=g, device=device) * k ** -0.5
            return rfq.rfq_quantize_weight(w)
        self.w_qkv = weight((heads + 2 * kv_heads) * D, hidden)
        self.w_out = weight(hidden, heads * D)
        self.width = -(-max_tokens // page)                 # blocks of a request, at most
        blocks = requests * self.width
        self.cache = rfq.kv_cache(blocks, kv_heads, page, D, device)
        self.cos_sin = rfq.rope_table(max_tokens + picture, D, device=device)
        self.axes = rfq.rope_axes((D // 8, 3 * D // 16, 3 * D // 16))

        def ints(shape, fill=0):
            return torch.full(shape, fill, dtype=torch.int32, device=device)
        self.tables = ints((requests, self.width), -1)
        self.free = torch.arange(blocks, dtype=torch.int32, device=device)
        self.count = ints((1,), blocks)
        self.lens, self.refused = ints((requests,)), ints((1,))

    def product(self, x, w):
        """RFQ product; few rows are quantized inside it (K a multiple of 512)."""
        if x.shape[0] <= 16 and x.shape[1] % 512 == 0:
            return rfq.rfq_gemm_stream(x, *w, out_dtype=torch.bfloat16)
        return rfq.rfq_gemm(*rfq.rfq_quantize_act(x), *w, out_dtype=torch.bfloat16, split=True)

    def positions(self, p):
        """[3][T]: time, row and column of a picture's tokens; text counts on all three."""
        n, side = self.picture ** 2, self.picture
        text = p - (n - side)
        inside = p < n
        return torch.stack((torch.where(inside, 0, text), torch.where(inside, p // side, text),
                            torch.where(inside, p % side, text)))

    def step(self, x, new_lens, max_query, max_seq):
        """x [T][hidden], the new tokens of all requests in their order -> its next value.
        Also leaves the step's rotated q, slots and lengths for check()."""
        T, Hq, Hk, D = x.shape[0], self.heads, self.kv_heads, self.D
        h = torch.nn.functional.rms_norm(x, x.shape[1:])
        qkv = self.product(h, self.w_qkv).view(T, Hq + 2 * Hk, D)
        slots, pos, seq, starts, counts = rfq.rfq_block_assign(
            self.lens, new_lens, self.tables, self.free, self.count, self.page, T)
        q = rfq.rfq_kv_append(qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:], slots, self.cache,
                              q=qkv[:, :Hq], positions=self.positions(pos), cos_sin=self.cos_sin,
                              axes=self.axes)
        o = rfq.rfq_kv_attention(q, self.cache, self.tables, seq, starts, max_query, max_seq)
        # A refused request has the length 0 in this step and keeps its tokens.
        torch.maximum(self.lens, seq, out=self.lens)
        self.count.copy_(counts[:1])
        self.refused.add_(counts[2:])
        self.last = (q, o, starts)
        return x + self.product(o.view(T, Hq * D), self.w_out)

    def end(self, ended):
        """Gives back the blocks of the requests with ended != 0 (uint8 [requests])."""
        self.count.copy_(rfq.rfq_block_release(self.lens, ended, self.tables, self.free,
                                               self.count, self.page))
        self.lens.mul_(1 - ended)

    def check(self):
        """The largest relative error of the last step's attention, request by request,
        against the formula in 64 bits on the cache's values."""
        q, o, starts = self.last
        assert int(self.refused) == 0, "requests were refused"
        starts, worst = starts.tolist(), 0.0
        for b, n in enumerate(self.lens.tolist()):
            i = torch.arange(n, dtype=torch.int32, device=q.device)
            slots = self.tables[b, (i // self.page).long()] * self.page + i % self.page
            group = self.heads // self.kv_heads
            k, v = (t.double().repeat_interleave(group, 1).cpu()
                    for t in rfq.rfq_kv_gather(self.cache, slots, torch.float32))
            rows = slice(starts[b], starts[b + 1])
            nq = rows.stop - rows.start
            if nq == 0:
                continue
            s = torch.einsum("thd,nhd->htn", q[rows].double().cpu(), k) * self.D ** -0.5
            see = torch.arange(n)[None] <= torch.arange(n - nq, n)[:, None]
            p = torch.softmax(s.masked_fill(~see, float("-inf")), -1)
            ref = torch.einsum("htn,nhd->thd", p, v)
            worst = max(worst, float((o[rows].double().cpu() - ref).norm() / ref.norm()))
        return worst


def main(requests=16, prompt=500, steps=64, **sizes):
    least = sizes.get("picture", 12) ** 2 + 1
    g = torch.Generator().manual_seed(1)
    prompts = torch.randint(least, max(least, prompt) + 1, (requests,), generator=g,
                            dtype=torch.int32)
    longest = max(least, prompt) + steps + 8
    block = Block(requests, longest, **sizes)
    hidden = block.w_out[0].shape[0]

    def run_prompts(lens):
        x = torch.randn((int(lens.sum()), hidden), device="cuda").bfloat16()
        y = block.step(x, lens.cuda(), int(lens.max()), longest)
        return y[(torch.cumsum(lens, 0) - 1).clamp(min=0).cuda()]

    x = run_prompts(prompts)
    errors = [block.check()]
    one = torch.ones(requests, dtype=torch.int32, device="cuda")
    # Decode: the same buffers every step, so one captured step serves them all.
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        x.copy_(block.step(x, one, 1, longest))
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.copy_(block.step(x, one, 1, longest))
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - start) / max(steps, 1) * 1e6
    errors.append(block.check())
    assert block.lens.cpu().tolist() == (prompts + 1 + steps).tolist()

    # Every second request ends; new prompts take its blocks while the others go on.
    ended = (torch.arange(requests, device="cuda") % 2 == 0).to(torch.uint8)
    block.end(ended)
    lens = torch.where(ended.cpu().bool(), prompts, torch.ones_like(prompts))
    run_prompts(lens)
    errors.append(block.check())
    held = -(-block.lens // block.page)
    assert int(block.count) + int(held.sum()) == block.free.shape[0]
    return us, errors


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    parser.add_argument("--requests", type=int, default=16)
    parser.add_argument("--prompt", type=int, default=500)
    parser.add_argument("--steps", type=int, default=64)
    us, errors = main(**vars(parser.parse_args()))
    print("decode step %.1f us; relative error of the attention %s" %
          (us, ", ".join("%.4f" % e for e in errors)))
