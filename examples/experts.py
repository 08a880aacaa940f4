"""A layer whose MLP is a set of experts, with MXFP4 weights and RFQ activations:

    x -> router -> experts and weights of each token -> tokens sorted by expert
      -> gate and up products (RFQ, each slot's expert) -> SwiGLU, quantized -> down product
      -> weighted sum of each token's results

A prompt, then decode steps captured once in a graph and replayed: how many tokens an expert
gets stays on the device.  The same layer in shares of the experts, whose sum is the layer.
And the router's gradient: the weights pass it on through the weighted sum.

    python examples/experts.py [--experts 128] [--choices 8] [--prompt 2000] [--steps 64]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_26581_amd as rfq  # noqa: E402


class Experts:
    """A share of a layer's experts: `held` of them from `first` on (None: all)."""

    def __init__(self, experts, choices, hidden, inner, first=0, held=None, device="cuda"):
        self.experts, self.k, self.first = experts, choices, first
        self.held = experts if held is None else held
        g = torch.Generator(device).manual_seed(0)
        self.router = torch.randn((experts, hidden), generator=g, device=device) * hidden ** -0.5

        def weight(n, k):
            codes, scales = [], []
            for e in range(experts):
                w = torch.randn((n, k), generator=g, device=device) * k ** -0.5
                if first <= e < first + self.held:
                    c, s = rfq.rfq_quantize_weight(w)
                    codes.append(c)
                    scales.append(s)
            return torch.stack(codes), torch.stack(scales)
        self.gate, self.up, self.down = weight(inner, hidden), weight(inner, hidden), weight(hidden, inner)

    def choose(self, x):
        """(weights, experts) of the tokens x [T][hidden]; differentiable in the router."""
        return rfq.rfq_route(x.float() @ self.router.T, self.k)

    def results(self, x, experts):
        """(z, plan): the experts' results [T k][hidden] in the slots of the plan."""
        plan = rfq.rfq_expert_sort(experts, self.held, first=self.first)
        q = rfq.rfq_quantize_act(x)
        # Slots past a share's last are not written: zeros, so that they quantize to zeros.
        g, u = (torch.zeros((plan.rows.shape[0], self.gate[0].shape[1]), dtype=x.dtype,
                            device=x.device) for _ in range(2))
        rfq.rfq_gemm_experts(*q, *self.gate, plan.offsets, rows=plan.rows, out=g)
        rfq.rfq_gemm_experts(*q, *self.up, plan.offsets, rows=plan.rows, out=u)
        h = rfq.rfq_swiglu_quantize_act(g, u)[:4]
        z = rfq.rfq_gemm_experts(*h, *self.down, plan.offsets, out_dtype=x.dtype)
        self.last = h, plan
        return z, plan

    def __call__(self, x):
        """x [T][hidden] bf16 -> [T][hidden]."""
        weights, experts = self.choose(x)
        z, plan = self.results(x, experts)
        return rfq.rfq_expert_combine(z, weights, plan)

    def check(self, x, out):
        """The relative error of `out`, the layer's last result, against the down product and
        the weighted sum in 64 bits."""
        (qc, qs, rc, rs), plan = self.last
        h = (rfq.rfq_dequant(qc, qs).double() + rfq.rfq_dequant(rc, rs).double())
        weights = self.choose(x)[0].double()
        z = torch.zeros((h.shape[0], x.shape[1]), dtype=torch.float64, device=x.device)
        ends = plan.offsets.tolist()
        for e in range(self.held):
            w = rfq.rfq_dequant(self.down[0][e], self.down[1][e]).double()
            z[ends[e]:ends[e + 1]] = h[ends[e]:ends[e + 1]] @ w.T.contiguous()
        s = plan.slots.long()
        rows = torch.where((s >= 0)[..., None], z[s.clamp(min=0)], 0.0)
        want = (weights[..., None] * rows).sum(1)
        return float((out.double() - want).norm() / want.norm())


def router_gradient(layer, x, dout):
    """The gradient of sum(dout * layer(x)) with respect to the router (the experts'
    results, which go through 4-bit products, count as given)."""
    layer.router.requires_grad_()
    weights, experts = layer.choose(x)
    z, plan = layer.results(x, experts)
    out = rfq.rfq_expert_combine(z, weights, plan)
    grad, = torch.autograd.grad(out, layer.router, dout)
    layer.router.requires_grad_(False)
    return grad, z, plan


def main(experts=128, choices=8, prompt=2000, steps=64, hidden=2048, inner=768, requests=16, shares=2):
    layer = Experts(experts, choices, hidden, inner)
    x = torch.randn((prompt, hidden), device="cuda").bfloat16()
    out = layer(x)
    errors = [layer.check(x, out)]

    # The shares' sum: each has its own rounding to bf16.
    held = experts // shares
    parts = [Experts(experts, choices, hidden, inner, first=i * held, held=held)(x).float()
             for i in range(shares)]
    apart = float((sum(parts) - out.float()).norm() / out.float().norm())

    x = x[:requests].contiguous()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer(x)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(x)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(steps):
        x.copy_(torch.nn.functional.rms_norm(x + out, x.shape[1:]))
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - start) / max(steps, 1) * 1e6
    errors.append(layer.check(x, out))
    return us, errors, apart


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    parser.add_argument("--experts", type=int, default=128)
    parser.add_argument("--choices", type=int, default=8)
    parser.add_argument("--prompt", type=int, default=2000)
    parser.add_argument("--steps", type=int, default=64)
    us, errors, apart = main(**vars(parser.parse_args()))
    print("decode step %.1f us; relative error of the layer's second half %s; of the sum of "
          "shares %.4f" % (us, ", ".join("%.4f" % e for e in errors), apart))
