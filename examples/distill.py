"""A student's head trained on the top logits of a teacher whose head runs in 8 bits.

    python examples/distill.py [--steps K] [--tokens N] [--hidden D] [--vocab V] [--top K] [--temperature T]

The teacher's head (random weights) is quantised once; for every batch of hidden states its logits are formed in 8 bits, the largest are kept with the
normaliser, and the student's head takes a step on them.  Needs an MI355X.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_25011_amd.distill import Int8Head, lsr_distill  # noqa: E402


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--hidden", type=int, default=768)
    ap.add_argument("--vocab", type=int, default=30522)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--temperature", type=float, default=2.0)
    a = ap.parse_args()
    dev = "cuda:0"
    gen = torch.Generator(device=dev).manual_seed(0)

    def normal(*shape, std=1.0):
        return torch.randn(shape, device=dev, generator=gen) * std

    teacher = Int8Head(normal(a.vocab, a.hidden, std=0.1), normal(a.vocab, std=0.5))
    W = normal(a.vocab, a.hidden, std=0.02).to(torch.bfloat16).requires_grad_(True)
    bias = torch.zeros(a.vocab, device=dev, requires_grad=True)
    opt = torch.optim.Adam([W, bias], lr=1e-2)
    H = normal(a.tokens, a.hidden).to(torch.bfloat16)
    mask = torch.rand(a.tokens, device=dev, generator=gen) < 0.85          # padding
    for step in range(a.steps):
        t0 = time.perf_counter()
        values, ids, lse = teacher.top_logits(H, a.top, a.temperature)
        loss, _ = lsr_distill(H, W, bias, ids, values, lse, mask, a.temperature)
        total = loss.sum() / mask.sum()
        opt.zero_grad()
        total.backward()
        opt.step()
        print(f"step {step}: loss {total.item():.4f}  {1e3 * (time.perf_counter() - t0):.2f} ms", flush=True)


if __name__ == "__main__":
    main()
