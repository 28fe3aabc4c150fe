"""Trains residual blocks (RMSNorm, gated feed-forward block, residual) whose backward pass reads 8-bit checkpoints only.

Forward, per block: the norm writes its output in bf16 for the block and in mx8 for the backward pass, and the stream in mx8; the block
writes both projections in mx8. Backward: the block's gradients from its checkpoints, the norm's from the 8-bit stream, added to the
stream's gradient. The weights' gradients are fp32 and summed over micro-batches.

    python examples/train_dense_blocks.py
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2609_34077_gb300 import mcft as M

D, W, T, BLOCKS, EPS = 256, 704, 300, 2, 1e-5
DESC = M.LayerDesc(D, 0, 0, W, 0, 0, M.MCFT_BF16)


class Block:
    """Weights, their gradients, and what a forward keeps."""

    def __init__(self, g):
        self.block = (torch.randn(3 * W * D, generator=g, device="cuda") / D ** 0.5).bfloat16()
        self.gamma = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).bfloat16()
        self.dblock = torch.zeros(3 * W * D, device="cuda")
        self.dgamma = torch.zeros(D, device="cuda")
        self.x8 = torch.empty(M.mcft_mx8_size(T, D), dtype=torch.uint8, device="cuda")
        self.ckpt = torch.empty(M.mcft_mx8_size(T, 2 * W), dtype=torch.uint8, device="cuda")

    def forward(self, x, y, ws):
        """x + y is the stream that enters; returns it and the block's output."""
        x, u, self.u8, self.rstd = M.mcft_residual_rmsnorm_mx8(DESC, x, y, self.gamma, EPS, x8=self.x8)
        return x, M.mcft_ffn_forward(DESC, u, self.block, ckpt=self.ckpt, workspace=ws)

    def backward(self, grad, ws):
        """The gradient of the stream that leaves -> that of the one that enters."""
        du, _ = M.mcft_ffn_grad(DESC, grad.bfloat16(), self.block, x8=self.u8, ckpt=self.ckpt, dblock=self.dblock,
                                accumulate=True, workspace=ws)
        grad, _ = M.mcft_rmsnorm_grad(DESC, self.gamma, self.rstd, du, dres=grad, x8=self.x8, dgamma=self.dgamma, accumulate=True)
        return grad


def main(steps=40, batches=2, verbose=True):
    g = torch.Generator(device="cuda").manual_seed(0)
    blocks, teacher = ([Block(g) for _ in range(BLOCKS)] for _ in range(2))
    ws = torch.empty(max(M.mcft_ffn_workspace_size(DESC, T), M.mcft_ffn_grad_workspace_size(DESC, T)), dtype=torch.uint8, device="cuda")

    def run(model, x):
        y = None
        for b in model:
            x, y = b.forward(x, y, ws)
        return x + y.float()

    inputs = [torch.randn(T, D, generator=g, device="cuda") for _ in range(batches)]
    targets = [run(teacher, x) for x in inputs]
    losses, first = [], None
    for step in range(steps):
        loss = 0.0
        for b in blocks:
            b.dblock.zero_(), b.dgamma.zero_()
        for x, target in zip(inputs, targets):
            diff = run(blocks, x) - target
            loss = loss + diff.square().mean() / batches
            grad = diff * (2.0 / diff.numel() / batches)
            for b in reversed(blocks):
                grad = b.backward(grad, ws)
        losses.append(loss)
        if first is None:  # what a test compares
            first = dict(inputs=inputs, targets=targets, blocks=[b.block.clone() for b in blocks], gammas=[b.gamma.clone() for b in blocks],
                         dblocks=[b.dblock.clone() for b in blocks], dgammas=[b.dgamma.clone() for b in blocks], dx=grad)
        for b in blocks:
            b.block -= (0.02 * b.dblock.sign() / D ** 0.5).bfloat16()
            b.gamma -= (0.002 * b.dgamma.sign()).bfloat16()
    M.mcft_device_error()
    losses = torch.stack(losses).tolist()
    kept = sum(t.numel() for t in (blocks[0].x8, blocks[0].u8, blocks[0].ckpt))
    if verbose:
        print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; a block keeps {kept} bytes for its backward pass, where its fp32 stream, "
              f"bf16 input and projections are {T * (4 * D + 2 * D + 4 * W)}")
    return dict(losses=losses, kept=kept, first=first)


if __name__ == "__main__":
    main()
