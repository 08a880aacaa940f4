"""Rotary positions in training: a few steps through rfq_rope and its gradient
(rfq_rope_backward) that fit the projection of an image's queries to given scores.

    python examples/rope_gradient.py [--side 16] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_26581_amd as rfq  # noqa: E402


def main(side=16, steps=20, heads=4, D=64):
    torch.manual_seed(0)
    T = side * side
    i = torch.arange(T, dtype=torch.int32, device="cuda")
    positions = torch.stack((i // side, i % side))
    cos_sin, axes = rfq.rope_table(side, D), rfq.rope_axes((D // 4, D // 4))

    def project(w):
        return rfq.rfq_rope((x @ w.t()).view(T, heads, D), positions, cos_sin, axes)
    x = torch.randn(T, D, device="cuda")
    keys = torch.randn(T, heads, D, device="cuda")
    target = project(torch.randn(heads * D, D, device="cuda") * D ** -0.5)
    w = torch.zeros(heads * D, D, device="cuda", requires_grad=True)
    optimizer = torch.optim.SGD([w], lr=1.0)
    losses = []
    for _ in range(steps):
        error = ((project(w) - target) * keys).sum(-1)
        loss = error.square().mean() / (2 * D)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    parser.add_argument("--side", type=int, default=16)
    parser.add_argument("--steps", type=int, default=20)
    losses = main(**vars(parser.parse_args()))
    print("loss %.4f -> %.6f" % (losses[0], losses[-1]))
