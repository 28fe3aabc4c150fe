"""Fine-tunes a masked, balanced router and then serves its layer from 4-bit expert blocks.

1. Training steps of the router: scored routing under a hard mask (a bias of -infinity) with a balance bias, the
   bf16 layer forward, the gates' gradient, the router's gradient, an update of the router and of the bias.
2. Serving: the experts packed to mx4 blocks, kept in host memory behind the expert cache, and decode steps that
   route, fetch what misses and run the layer on the 4-bit blocks.

    python examples/router_and_4bit_experts.py
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2609_34077_gb300 import mcft as M

D, E, K, W, T, SLOTS = 512, 32, 4, 256, 512, 12


def main(train_steps=60, decode_steps=8, verbose=True):
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()

    layer = M.LayerDesc(D, E, K, W, 0, M.MCFT_GATE_RENORM, M.MCFT_BF16)
    scored = M.ScoredDesc(D, E, K, 4, 3, 2, M.MCFT_SCORE_SIGMOID, M.MCFT_GATE_RENORM, M.MCFT_BF16, 1.0)
    experts = [normal(3 * W * D, std=0.05) for _ in range(E)]
    router = torch.randn(E, D, generator=g, device="cuda") * 0.05  # fp32 master copy
    bias = torch.zeros(E, device="cuda")
    masked = torch.randperm(E, generator=g, device="cuda")[: E // 4]
    bias[masked] = -float("inf")

    # a teacher's router gives the outputs to learn
    teacher = (torch.randn(E, D, generator=g, device="cuda") * 0.05).bfloat16()
    x = normal(T, D)
    idx, gate = M.mcft_route_scored(scored, x, teacher, bias)
    target = M.mcft_moe_forward(layer, x, idx, gate, experts).float()

    ws = torch.empty(M.mcft_moe_workspace_size(layer, T), dtype=torch.uint8, device="cuda")
    grad_ws = torch.empty(M.mcft_route_scored_grad_workspace_size(scored, T), dtype=torch.uint8, device="cuda")
    logits = torch.empty(T, E, device="cuda")
    load = torch.empty(E, dtype=torch.int32, device="cuda")
    losses, spread = [], []
    for _ in range(train_steps):
        w = router.bfloat16()
        idx, gate = M.mcft_route_scored(scored, x, w, bias, logits=logits, load=load)
        y = M.mcft_moe_forward(layer, x, idx, gate, experts, workspace=ws)
        diff = y.float() - target
        losses.append(diff.square().mean())
        dy = (diff * (2.0 / diff.numel())).bfloat16()
        dgate = M.mcft_gate_grad(layer, dy, ws)
        _, dw = M.mcft_route_scored_grad(scored, x, w, idx, gate, logits, dgate, workspace=grad_ws)
        router -= 2.0 * dw / dw.norm().clamp_min(1e-12) * 0.1
        free = bias > -float("inf")
        share = load.float() / load[free].float().mean()
        spread.append(share[free].max())
        bias = torch.where(free, bias - 0.003 * torch.sign(share - 1), bias)
    M.mcft_device_error()

    blocks = [M.mcft_mx4_pack_expert(layer, b) for b in experts]
    size = M.mcft_mx4_expert_size(layer)
    cache = M.mcft_cache_create(1, E, SLOTS, size, [b.cpu().pin_memory() for b in blocks], max_assign=K)
    copies = torch.cuda.Stream()
    w = router.bfloat16()
    errors = []
    for s in range(decode_steps):
        token = x[s: s + 1]
        idx, gate = M.mcft_route_scored(scored, token, w, bias)
        M.mcft_cache_step(cache, 0, idx)
        pointers = M.mcft_fetch_experts(cache, 0, copy_stream=copies)
        y = M.mcft_moe_forward_mx4(layer, token, idx, gate, pointers)
        full = M.mcft_moe_forward(layer, token, idx, gate, experts)
        errors.append((y.float() - full.float()).norm() / full.float().norm())
    M.mcft_device_error()
    hits, fetches, _ = M.mcft_cache_stats(cache)
    out = dict(first_loss=float(losses[0]), last_loss=float(losses[-1]), first_spread=float(spread[0]),
               last_spread=float(spread[-1]), masked_load=int(load[masked].sum()), hits=hits, fetches=fetches,
               mx4_bytes=size, bf16_bytes=experts[0].numel() * 2, mx4_error=float(torch.stack(errors).mean()))
    if verbose:
        print(f"loss {out['first_loss']:.4f} -> {out['last_loss']:.4f}; busiest expert {out['first_spread']:.2f} -> "
              f"{out['last_spread']:.2f} times the mean; masked experts chosen {out['masked_load']} times")
        print(f"{fetches} fetches of {size} bytes (bf16 blocks: {out['bf16_bytes']}), {hits} hits; "
              f"4-bit outputs {out['mx4_error']:.3f} from the bf16 ones")
    return out


if __name__ == "__main__":
    main()
