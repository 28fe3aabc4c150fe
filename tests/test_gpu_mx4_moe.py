"""The routed layer on mx4 expert blocks against the fp64 oracle.

Tolerance: the hidden activations are rounded to 4 bits after fp32 sums, so an element close to a tie may round
either way; the oracle says how far each output can move by that. On top: the last fp32 sums (2^-22 of the terms'
size, taken as 2^-18 of the row's largest output) and the rounding of y (2^-8 of it in bf16)."""
import numpy as np
import pytest
import torch

import oracle.mx4 as O
from paper_2609_34077_gb300 import mcft as M

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, d, E, K, w, S=0, dtype=torch.bfloat16, seed=0):
        self.desc = M.LayerDesc(d, E, K, w, S, M.MCFT_GATE_RENORM, M.MCFT_BF16 if dtype == torch.bfloat16 else M.MCFT_F32)
        self.dtype, self.seed = dtype, seed
        g = torch.Generator().manual_seed(seed)
        self.plain = [(torch.randn(3 * w * d, generator=g) * 0.05).to(dtype) for _ in range(E + S)]
        self.blocks = [M.mcft_mx4_pack_expert(self.desc, b.cuda()) for b in self.plain]
        self.triples = [(b[: w * d].view(w, d).double().numpy(), b[w * d: 2 * w * d].view(w, d).double().numpy(),
                         b[2 * w * d:].view(d, w).double().numpy()) for b in self.plain]

    def batch(self, T, drop=0.0):
        g = torch.Generator().manual_seed(self.seed + T)
        D = self.desc
        x = torch.randn(T, D.d, generator=g).to(self.dtype)
        idx = torch.stack([torch.randperm(D.E, generator=g)[: D.K] for _ in range(T)]).int()
        gate = torch.softmax(torch.randn(T, D.K, generator=g), 1)
        if drop:
            idx[torch.rand(T, D.K, generator=g) < drop] = -1
            idx[0] = -1
        return x, idx, gate

    def run(self, x, idx, gate, **kw):
        E = self.desc.E
        y = M.mcft_moe_forward_mx4(self.desc, x.cuda(), idx.cuda(), gate.cuda(), self.blocks[:E], self.blocks[E:], **kw)
        M.mcft_device_error()
        return y

    def check(self, y, x, idx, gate):
        E = self.desc.E
        ref, room = O.moe_layer(x.double().numpy(), idx.numpy(), gate.numpy(), self.triples[:E], self.triples[E:])
        big = np.abs(ref).max(1, keepdims=True)
        tol = room + big * (2.0 ** -18 + (2.0 ** -8 if self.dtype == torch.bfloat16 else 0.0)) + 1e-30
        err = np.abs(y.cpu().double().numpy() - ref)
        assert (err <= tol).all(), f"worst {np.max(err / tol):.3g} of the bound"


@pytest.mark.parametrize("T", [1, 2, 9, 64, 127, 128, 129, 200, 700])
@pytest.mark.parametrize("d,E,K,w,S", [(256, 8, 2, 512, 0), (192, 10, 3, 320, 2), (64, 1, 1, 64, 1)])
def test_layer(T, d, E, K, w, S):
    L = Layer(d, E, K, w, S)
    b = L.batch(T)
    L.check(L.run(*b), *b)


@pytest.mark.parametrize("T", [5, 300])
def test_fp32_layer(T):
    L = Layer(256, 8, 2, 384, 1, torch.float32)
    b = L.batch(T)
    L.check(L.run(*b), *b)


@pytest.mark.parametrize("T", [3, 40, 333])
def test_many_experts(T):
    L = Layer(128, 256, 16, 128, 8)
    b = L.batch(T, drop=0.2)
    L.check(L.run(*b), *b)


@pytest.mark.parametrize("T", [1, 50, 260])
@pytest.mark.parametrize("S", [0, 1])
def test_tokens_without_an_expert(T, S):
    L = Layer(192, 6, 2, 128, S)
    x, idx, gate = L.batch(T, drop=0.5)
    gate[idx < 0] = float("nan")  # not read
    y = L.run(x, idx, gate)
    L.check(y, x, idx, torch.where(idx < 0, torch.zeros_like(gate), gate))
    if S == 0:
        assert (y[0] == 0).all()


@pytest.mark.parametrize("T", [4, 150])
def test_an_expert_named_twice(T):
    L = Layer(128, 4, 3, 128)
    x, idx, gate = L.batch(T)
    idx[:, 2] = idx[:, 0]
    L.check(L.run(x, idx, gate), x, idx, gate)


@pytest.mark.parametrize("T", [7, 500])
def test_one_expert_takes_all(T):
    L = Layer(128, 64, 1, 192, 0)
    x, idx, gate = L.batch(T)
    idx[:] = 37
    L.check(L.run(x, idx, gate), x, idx, gate)


def test_the_same_bits_and_any_larger_workspace():
    L = Layer(256, 16, 4, 256, 1)
    ws = torch.full((M.mcft_mx4_workspace_size(L.desc, 600),), 0xFF, dtype=torch.uint8, device="cuda")  # NaN scales
    for T in (600, 3, 128, 129):
        b = L.batch(T)
        first = L.run(*b, workspace=ws)
        ws.random_(0, 256)
        assert torch.equal(first, L.run(*b, workspace=ws))
        L.check(first, *b)


def test_a_token_gives_the_same_bits_in_any_batch():
    L = Layer(256, 8, 2, 512, 1)
    x, idx, gate = L.batch(400)
    y = L.run(x, idx, gate)
    assert torch.equal(y[130:390], L.run(x[130:390], idx[130:390], gate[130:390]))


@pytest.mark.parametrize("T", [3, 200])
def test_bad_ids_and_missing_blocks_leave_y(T):
    L = Layer(128, 4, 2, 128)
    x, idx, gate = L.batch(T)
    y = torch.full((T, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    for bad in (4, -2, 2 ** 30):
        i = idx.clone()
        i[T - 1, 1] = bad
        M.mcft_moe_forward_mx4(L.desc, x.cuda(), i.cuda(), gate.cuda(), L.blocks, y=y)
        with pytest.raises(M.MCFTError):
            M.mcft_device_error()
        assert (y == 3).all()
    i = idx.clone()
    i[:] = 1
    M.mcft_moe_forward_mx4(L.desc, x.cuda(), i.cuda(), gate.cuda(), [L.blocks[0], None, None, None], y=y)
    with pytest.raises(M.MCFTError):
        M.mcft_device_error()
    assert (y == 3).all()
    i[:] = 0
    M.mcft_moe_forward_mx4(L.desc, x.cuda(), i.cuda(), gate.cuda(), [L.blocks[0], None, None, None], y=y)
    M.mcft_device_error()
    L.check(y, x, i, gate)


def test_refusals():
    L = Layer(128, 4, 2, 128)
    x, idx, gate = (t.cuda() for t in L.batch(8))
    with pytest.raises(M.MCFTError) as e:
        M.mcft_moe_forward_mx4(L.desc, x, idx, gate, L.blocks, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == M.MCFT_ERR_INVALID
    for D, status in ((M.LayerDesc(100, 4, 2, 128, 0, 0, 1), M.MCFT_ERR_INVALID),
                      (M.LayerDesc(128, 4, 5, 128, 0, 0, 1), M.MCFT_ERR_INVALID),
                      (M.LayerDesc(128, 257, 2, 128, 0, 0, 1), M.MCFT_ERR_UNSUPPORTED),
                      (M.LayerDesc(128, 64, 17, 128, 0, 0, 1), M.MCFT_ERR_UNSUPPORTED),
                      (M.LayerDesc(128, 4, 2, 128, 9, 0, 1), M.MCFT_ERR_UNSUPPORTED),
                      (M.LayerDesc(128, 4, 2, 128, 0, 0, 7), M.MCFT_ERR_INVALID)):
        with pytest.raises(M.MCFTError) as e:
            M.mcft_mx4_workspace_size(D, 8)
        assert e.value.status == status
    assert M.mcft_moe_forward_mx4(L.desc, x[:0], idx[:0], gate[:0], L.blocks).shape == (0, 128)


def test_blocks_through_the_expert_cache():
    """mx4 blocks are fetched by the cache like any others: same bits as with resident blocks."""
    L = Layer(256, 8, 2, 128)
    n = M.mcft_mx4_expert_size(L.desc)
    host = [b.cpu().pin_memory() for b in L.blocks]
    cache = M.mcft_cache_create(1, 8, 3, n, host, max_assign=8)
    copies = torch.cuda.Stream()
    for step in range(6):
        L.seed = step
        x, idx, gate = (t.cuda() for t in L.batch(2))
        M.mcft_cache_step(cache, 0, idx)
        ptrs = M.mcft_fetch_experts(cache, 0, copy_stream=copies)
        y = M.mcft_moe_forward_mx4(L.desc, x, idx, gate, ptrs)
        torch.cuda.synchronize()
        assert torch.equal(y, M.mcft_moe_forward_mx4(L.desc, x, idx, gate, L.blocks))
    M.mcft_device_error()
