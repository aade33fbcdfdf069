#!/usr/bin/env python3
"""A stack of feed-forward sublayers on one GPU, trained and then asked token by token.

Each sublayer is norm -> gated projections -> projection back -> norm, gate and residual sum; the norm behind one is joined with the norm before
the next (residual_norm).  The gates are ReLUs, so what the gated projections keep for backward, and their output, are zero in the same
places: with --stash a BitmapStash keeps all of it compressed.  The gradients are clipped to a common norm before each step.

    python examples/feed_forward.py --layers 4 --features 1024 --hidden 4096 --rows 4096 --steps 10 --stash
"""
import argparse
import contextlib
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2110_15362_amd import autograd, block  # noqa: E402


class FeedForwardStack(torch.nn.Module):
    """`layers` sublayers of `features`, `hidden` between their projections; one gate for each sequence, from its condition."""

    def __init__(self, layers, features, hidden, conditions, activation="relu", dtype=torch.bfloat16, device="cuda", seed=0):
        super().__init__()
        g = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return torch.nn.Parameter((torch.randn(*shape, generator=g) / math.sqrt(shape[-1])).to(device=device, dtype=dtype))

        def ones():
            return torch.nn.Parameter(torch.ones(features, device=device, dtype=dtype))
        self.activation, self.scale = activation, 1.0 / math.sqrt(2.0 * layers)
        self.first_norm = ones()
        self.w_gate = torch.nn.ParameterList([weight(hidden, features) for _ in range(layers)])
        self.w_up = torch.nn.ParameterList([weight(hidden, features) for _ in range(layers)])
        self.w_down = torch.nn.ParameterList([weight(features, hidden) for _ in range(layers)])
        self.post_norm = torch.nn.ParameterList([ones() for _ in range(layers)])
        self.pre_norm = torch.nn.ParameterList([ones() for _ in range(layers)])      # of the next sublayer; the last one's is the output norm
        self.w_condition = torch.nn.ParameterList([weight(features, conditions) for _ in range(layers)])

    def forward(self, x, condition):
        """x [sequences, tokens, features], condition [sequences, conditions] -> normed output of the same shape as x."""
        y = block.rms_norm(x, self.first_norm)
        for i in range(len(self.w_gate)):
            h = block.gated_linear(y, self.w_gate[i], self.w_up[i], self.activation)
            gate = torch.nn.functional.linear(condition, self.w_condition[i])
            x, y = block.residual_norm(x, torch.nn.functional.linear(h, self.w_down[i]), self.post_norm[i], gate, self.pre_norm[i], scale=self.scale)
        return y


def step(model, x, condition, target, stash, max_norm, rate):
    """One training step; returns the loss and the norm that the gradients had, both on the device."""
    for p in model.parameters():
        p.grad = None
    with stash if stash is not None else contextlib.nullcontext():
        loss = (model(x, condition) - target).float().square().mean()
    loss.backward()
    norm = block.clip_grad_norm_(model.parameters(), max_norm)
    with torch.no_grad():
        for p in model.parameters():
            p.sub_(p.grad, alpha=rate)
    return loss.detach(), norm


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--features", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--rows", type=int, default=4096, help="tokens of a step, over 8 sequences")
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--rate", type=float, default=0.5)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dtype", choices=("bf16", "f16", "f32"), default="bf16")
    ap.add_argument("--stash", action="store_true", help="keep what backward needs compressed")
    a = ap.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[a.dtype]
    g = torch.Generator(device="cuda").manual_seed(1)
    sequences = 8
    x, target = (torch.randn(sequences, a.rows // sequences, a.features, generator=g, device="cuda").to(dtype) for _ in range(2))
    condition = torch.randn(sequences, 32, generator=g, device="cuda").to(dtype)
    model = FeedForwardStack(a.layers, a.features, a.hidden, 32, dtype=dtype)
    stash = autograd.BitmapStash() if a.stash else None
    torch.cuda.reset_peak_memory_stats()
    before, losses = torch.cuda.memory_allocated(), []
    for i in range(a.steps):
        loss, norm = step(model, x, condition, target, stash, a.max_norm, a.rate)
        losses.append(float(loss))
        print("step %3d  loss %.5f  gradient norm %.4f" % (i, losses[-1], float(norm)), flush=True)
    print("peak memory of a step: %.1f MiB" % ((torch.cuda.max_memory_allocated() - before) / 2 ** 20))
    if stash is not None:
        s = stash.stats
        print("saved for backward: %d of %d tensors compressed, %.1f of %.1f MiB stored" % (
            s["compressed"], s["tensors"], s["stored_bytes"] / 2 ** 20, s["dense_bytes"] / 2 ** 20))
    with torch.no_grad():                     # one token at a time: the same calls on a row
        whole = model(x[:1], condition[:1])
        alone = model(x[:1, -1:], condition[:1])
    print("last token alone and in its sequence differ by %.4f at the most" % float((whole[:, -1:] - alone).abs().max()))
    return losses


if __name__ == "__main__":
    main()
