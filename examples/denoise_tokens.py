"""Trains a small residual block (TV pass along the tokens, two channel products, activations held in 8 bits) to find the
noise in piecewise-constant tokens, then runs one more sequence through it without gradients.

    python examples/denoise_tokens.py [--steps 200] [--tokens 512] [--channels 64] [--checkpoint 8bit|full]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2204_03643_amd.linear import TVMixer  # noqa: E402


def batch(n, tokens, channels, gen):
    """Clean tokens, constant over runs of 16 and more, and noisy ones."""
    runs = torch.randn(n, -(-tokens // 16), channels, generator=gen, device="cuda")
    keep = torch.rand(n, runs.shape[1], 1, generator=gen, device="cuda") < 0.5
    keep[:, 0] = False
    at = torch.where(keep, 0, torch.arange(runs.shape[1], device="cuda").view(1, -1, 1)).cummax(1).values
    clean = runs.gather(1, at.expand_as(runs)).repeat_interleave(16, 1)[:, :tokens]
    return clean, clean + 0.5 * torch.randn(clean.shape, generator=gen, device="cuda")


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--channels", type=int, default=64)
    p.add_argument("--checkpoint", choices=("8bit", "full"), default="8bit")
    a = p.parse_args()
    torch.manual_seed(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    block = TVMixer(a.channels, 4 * a.channels, checkpoint=a.checkpoint, init_lambda=1.0, device="cuda")
    opt = torch.optim.Adam(block.parameters(), lr=2e-3)
    for step in range(a.steps):
        clean, noisy = batch(16, a.tokens, a.channels, gen)
        loss = (noisy - block(noisy) - clean).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 50 == 0 or step == a.steps - 1:
            print("step %4d  loss %.4f  (noise alone %.4f)" % (step, loss.item(), (noisy - clean).square().mean().item()), flush=True)
    with torch.no_grad():
        clean, noisy = batch(1, a.tokens, a.channels, gen)
        print("one more sequence: %.4f" % (noisy - block(noisy) - clean).square().mean().item())


if __name__ == "__main__":
    main()
