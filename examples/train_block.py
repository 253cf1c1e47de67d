#!/usr/bin/env python3
"""Two pre-norm MoE blocks trained for a few steps on packed sequences, as a
program uses the package: layer norm, router with a balance loss per sequence,
grouped SwiGLU experts, pre-activations kept in 8 bits, every gradient, and
plain SGD on float32 copies of the weights.

    python examples/train_block.py [--steps 20] [--act-bits 8|16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2601_14327_amd import BlockWeights, MoEBlockPlan  # noqa: E402

NAMES = ("gamma", "beta", "w_router", "w_gate_up", "w_down")


def make_weights(g, d, E, f, dev):
    def normal(*shape):
        return 0.03 * torch.randn(shape, generator=g, device=dev)

    return dict(gamma=torch.ones(d, device=dev), beta=torch.zeros(d, device=dev),
                w_router=normal(E, d), w_gate_up=normal(E, 2 * f, d), w_down=normal(E, d, f))


def working_copy(master):
    """What the kernels read: matrices in bf16, the norm's vectors in float32."""
    bf16 = torch.bfloat16
    return BlockWeights(*(master[n] if n in ("gamma", "beta") else master[n].to(bf16)
                          for n in NAMES))


def train(steps=20, T=1024, d=256, E=16, k=2, f=256, n_blocks=2, act_bits=8, coef=0.02, lr=0.3,
          seed=0, dev="cuda"):
    """Returns the losses (mean squared error and balance loss per step)."""
    g = torch.Generator(device=dev).manual_seed(seed)
    masters = [make_weights(g, d, E, f, dev) for _ in range(n_blocks)]
    offsets = torch.tensor([0, T // 2 - 7, T // 2 + 30, T], dtype=torch.int32, device=dev)
    blocks = []
    for _ in range(n_blocks):   # the blocks share what they do not keep
        blocks.append(MoEBlockPlan(T, d, E, k, f, n_seq=3, coef=coef, act_bits=act_bits,
                                   device=dev, scratch=blocks[0] if blocks else None))
    x = torch.randn((T, d), generator=g, device=dev).to(torch.bfloat16)
    turn = torch.randn((d, d), generator=g, device=dev) / d ** 0.5
    target = x.float() + torch.tanh(x.float() @ turn)
    history = []
    for _ in range(steps):
        weights = [working_copy(m) for m in masters]
        h, stream = x, None
        for block, w in zip(blocks, weights):
            h, stream = block.forward(h, w, stream, seq_offsets=offsets)
        err = h.float() + stream.float() - target
        grad = (2.0 / T * err).to(torch.bfloat16)      # of the squared error, meaned over tokens
        for block, w, m in zip(reversed(blocks), reversed(weights), reversed(masters)):
            grad = block.backward(grad, w)
            p = block.layer
            for name, dw in zip(NAMES, (block.dgamma, block.dbeta, p.dw_router, p.dw_gate_up,
                                        p.dw_down)):
                m[name].sub_(dw, alpha=lr)
        history.append((err.square().sum(1).mean(), sum(b.loss for b in blocks)[0]))
    return [(float(a), float(b)) for a, b in history]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--act-bits", type=int, default=8, choices=(8, 16))
    args = ap.parse_args()
    for i, (mse, balance) in enumerate(train(args.steps, act_bits=args.act_bits)):
        print(f"step {i:3d}  squared error {mse:9.4f}  balance loss {balance:.5f}")
