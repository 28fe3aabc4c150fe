"""The example of training from 8-bit checkpoints runs, and its first gradients are those of the fp64 chain: off by no more than
what three 8-bit factors of each term make (2^-4 / sqrt(3) of the mean square each, so 2^-4 of the norm), twice that below the
second block."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_train_dense_blocks():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_dense_blocks.py")
    spec = importlib.util.spec_from_file_location("example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(steps=3, verbose=False)
    f, n, d, w = r["first"], example.W * example.D, example.D, example.W
    assert len(r["losses"]) == 3 and all(v == v for v in r["losses"])
    assert r["kept"] * 1.9 < example.T * (6 * d + 4 * w)
    leaves = [t.double().cpu().requires_grad_() for t in (f["inputs"][-1], *f["blocks"], *f["gammas"])]
    loss = 0.0
    for i, target in enumerate(f["targets"]):
        s = leaves[0] if i == len(f["targets"]) - 1 else f["inputs"][i].double().cpu()
        for b, gm in zip(leaves[1:3], leaves[3:]):
            v = s * (s.square().mean(1, keepdim=True) + example.EPS).rsqrt() * gm
            s = s + (torch.nn.functional.silu(v @ b[:n].view(w, d).T) * (v @ b[n:2 * n].view(w, d).T)) @ b[2 * n:].view(d, w).T
        loss = loss + (s - target.double().cpu()).square().mean() / len(f["targets"])
    loss.backward()
    assert abs(r["losses"][0] - loss.item()) < 2.0 ** -7 * loss.item()
    for got, leaf, room in zip((f["dx"], *f["dblocks"], *f["dgammas"]), leaves, (2, 2, 1, 2, 1)):
        off = (got.double().cpu() - leaf.grad).norm() / leaf.grad.norm()
        assert off < room * 2.0 ** -4, off
