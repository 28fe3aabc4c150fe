"""The Python binding allocates what a call needs from the memory of the stream that the call's kernels run on. On the CPU, with a
library, streams and an allocator that only write down what is asked of them."""
import contextlib

import pytest
import torch

from paper_2609_34077_gb300 import mcft as M


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle

    def __int__(self):
        return self.cuda_stream


@pytest.fixture
def seen(monkeypatch):
    """(stream of the allocation, bytes) of each torch.empty."""
    current, log = [None], []

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream.cuda_stream
        yield
        current[0] = before

    class Library:
        def __getattr__(self, name):
            return lambda *_: M.MCFT_OK

    real = torch.empty

    def empty(*shape, **kw):
        t = real(*shape, **kw)
        log.append((current[0], t.numel() * t.element_size()))
        return t

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: Stream(0))
    monkeypatch.setattr(M, "_raw_stream", lambda _: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(M, "lib", lambda: Library())
    return log


T, d, E, K, W = 3, 64, 4, 2, 64
LAYER = M.LayerDesc(d, E, K, W, 0, 0, M.MCFT_F32)
SCORED = M.ScoredDesc(d, E, K, 1, 1, 1, 0, 0, M.MCFT_F32, 1.0)
X, R = torch.zeros(T, d), torch.zeros(E, d)
IDX, GATE, Z = torch.zeros(T, K, dtype=torch.int32), torch.zeros(T, K), torch.zeros(T, E)
BYTES = torch.zeros(1 << 16, dtype=torch.uint8)
CALLS = dict(
    route=(2, lambda **s: M.mcft_route(LAYER, X, R, M.MCFT_ROUTE_TOPK, **s)),
    forward=(2, lambda **s: M.mcft_moe_forward(LAYER, X, IDX, GATE, [4096] * E, **s)),
    lora=(2, lambda **s: M.mcft_moe_forward_lora(LAYER, X, IDX, GATE, [4096] * E, **s)),
    scored=(2, lambda **s: M.mcft_route_scored(SCORED, X, R, **s)),
    grad=(3, lambda **s: M.mcft_route_scored_grad(SCORED, X, R, IDX, GATE, Z, GATE, **s)),
    quantize=(1, lambda **s: M.mcft_mx4_quantize(X, **s)),
    dequantize=(1, lambda **s: M.mcft_mx4_dequantize(BYTES, T, d, **s)),
    matmul=(1, lambda **s: M.mcft_mx4_matmul(BYTES, BYTES, T, E, d, **s)),
    pack=(1, lambda **s: M.mcft_mx4_pack_expert(LAYER, torch.zeros(3 * W * d), **s)),
    mx4=(2, lambda **s: M.mcft_moe_forward_mx4(LAYER, X, IDX, GATE, [4096] * E, **s)))


@pytest.mark.parametrize("name", sorted(CALLS))
def test_allocations(seen, name):
    n, call = CALLS[name]
    call()
    assert [at for at, _ in seen] == [None] * n  # (the current stream's)
    for stream, handle in ((Stream(7), 7), (7, 7), (0, 0)):
        seen.clear()
        call(stream=stream)
        assert [at for at, _ in seen] == [handle] * n
