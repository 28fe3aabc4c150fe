"""The dense gated feed-forward block, its checkpoint and its gradient against the fp64 oracle, elementwise within the bounds of
dense_model.py: from one token on, at the sizes where tiles, halves of tiles and split contractions end."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_34077_gb300 import mcft as M
from tests.dense_model import Case, f64, near
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
# (1 to 8, 16 and 32 tokens by the weights' size: the streaming kernels, with clusters where there are few rows)
SHAPES = [(1, 64, 64), (1, 2048, 1408), (8, 512, 2048), (9, 256, 64), (24, 64, 832), (32, 704, 1024), (33, 704, 1024), (9, 4096, 4096), (2, 192, 320), (4, 64, 4096), (5, 4096, 64), (16, 960, 704), (17, 128, 192), (64, 320, 128),
          (65, 64, 64), (65, 64, 4096), (127, 192, 448), (128, 256, 256), (129, 448, 192), (256, 512, 384), (257, 320, 704),
          (300, 1024, 1408), (1023, 960, 704), (3000, 64, 64), (2100, 512, 1408)]


def desc(c):
    return M.LayerDesc(c.d, 0, 0, c.w, 0, 0, M.MCFT_BF16 if c.dtype == BF16 else M.MCFT_F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d,w", SHAPES)
def test_forward_and_checkpoint(T, d, w, dtype):
    c = Case(T, d, w, dtype)
    D, e = desc(c), c.x.element_size()
    guards = [Guarded(T * d * e), Guarded(M.mcft_ffn_workspace_size(D, T)), Guarded(M.mcft_mx8_size(T, 2 * w)), Guarded(T * d * e)]
    y = M.mcft_ffn_forward(D, c.x, c.block, y=guards[0].view(dtype, (T, d)), workspace=guards[1].view())
    ckpt = guards[2].view()
    z = M.mcft_ffn_forward(D, c.x, c.block, y=guards[3].view(dtype, (T, d)), ckpt=ckpt, workspace=guards[1].view())
    M.mcft_device_error()
    for g in guards:
        g.check("forward")
    want, room = c.forward()
    near(y, want, room, "y")
    near(z, want, room, "y beside a checkpoint")
    g, u, eg, eu = c.projections(f64(c.x))
    gu, egu = np.concatenate((g, u), 1), np.concatenate((eg, eu), 1)
    got = M.mcft_mx8_dequantize(ckpt, T, 2 * w, F32)
    near(got, gu, egu + 0.5 * oracle.dense.mx8_step(np.abs(gu) + egu), "checkpoint")
    assert torch.equal(M.mcft_mx8_dequantize(M.mcft_mx8_quantize(got), T, 2 * w, F32), got)  # (its scales are the smallest)


@pytest.mark.parametrize("form", ["checkpoints", "x8", "x", "x and checkpoint"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d,w", SHAPES)
def test_gradient(T, d, w, dtype, form):
    c = Case(T, d, w, dtype, 1)
    D, e = desc(c), c.x.element_size()
    given = dict(x8=M.mcft_mx8_quantize(c.x)) if form in ("checkpoints", "x8") else dict(x=c.x)
    x = f64(M.mcft_mx8_dequantize(given["x8"], T, d, F32)) if "x8" in given else f64(c.x)
    if "checkpoint" in form:
        given["ckpt"] = torch.empty(M.mcft_mx8_size(T, 2 * w), dtype=torch.uint8, device="cuda")
        M.mcft_ffn_forward(D, c.x, c.block, ckpt=given["ckpt"])
        gu = f64(M.mcft_mx8_dequantize(given["ckpt"], T, 2 * w, F32))
        forward = (gu[:, :w], gu[:, w:])
    else:
        forward = c.projections(x)
    guards = [Guarded(T * d * e), Guarded(3 * w * d * e), Guarded(M.mcft_ffn_grad_workspace_size(D, T))]
    ws = guards[2].view()
    dx, db = M.mcft_ffn_grad(D, c.dy, c.block, **given, dx=guards[0].view(dtype, (T, d)), dblock=guards[1].view(dtype), workspace=ws)
    M.mcft_device_error()
    for g in guards:
        g.check("gradient")
    (wx, rx), (wb, rb) = c.gradient(x, *forward)
    near(dx, wx, rx, "dx")
    near(db, wb, rb, "dblock")
    # in fp32, and added to what is there: twice the gradient
    _, (_, rb32) = c.gradient(x, *forward, out_r=2.0 ** -22)
    _, full = M.mcft_ffn_grad(D, c.dy, c.block, **given, grad_dtype=F32, workspace=ws)
    near(full, wb, rb32, "fp32 dblock")
    M.mcft_ffn_grad(D, c.dy, c.block, **given, dblock=full, accumulate=True, workspace=ws)
    near(full, 2 * wb, 2 * rb32, "fp32 dblock, added to")
    M.mcft_ffn_grad(D, c.dy, c.block, **given, dblock=db, accumulate=True, workspace=ws)
    near(db, 2 * wb, 3 * rb, "dblock, added to")
    # one of the two alone
    for skip in (0, 1):
        outs = [torch.full((T, d), 3.0, dtype=dtype, device="cuda"), torch.full((3 * w * d,), 3.0, device="cuda")]
        p = [None if i == skip else t.data_ptr() for i, t in enumerate(outs)]
        v = {k: t.data_ptr() for k, t in given.items()}
        M._check(M.lib().mcft_ffn_grad(M.C.byref(D), c.dy.data_ptr(), T, c.block.data_ptr(), v.get("x"), v.get("x8"), v.get("ckpt"),
                                       p[0], p[1], M.MCFT_F32, 0, ws.data_ptr(), ws.numel(), M._stream(None)))
        M.mcft_device_error()
        if skip:
            near(outs[0], wx, rx, "dx alone")
        else:
            near(outs[1], wb, rb32, "dblock alone")
        assert bool((outs[skip] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [5, 300])
def test_input_gradient_from_the_checkpoint_alone(T, dtype):
    """dx wants neither x nor its mx8 matrix beside a checkpoint."""
    c = Case(T, 192, 320, dtype)
    D = desc(c)
    ckpt = torch.empty(M.mcft_mx8_size(T, 640), dtype=torch.uint8, device="cuda")
    M.mcft_ffn_forward(D, c.x, c.block, ckpt=ckpt)
    ws = torch.empty(M.mcft_ffn_grad_workspace_size(D, T), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(c.x)
    M._check(M.lib().mcft_ffn_grad(M.C.byref(D), c.dy.data_ptr(), T, c.block.data_ptr(), None, None, ckpt.data_ptr(), dx.data_ptr(),
                                   None, M.MCFT_F32, 0, ws.data_ptr(), ws.numel(), M._stream(None)))
    M.mcft_device_error()
    gu = f64(M.mcft_mx8_dequantize(ckpt, T, 640, F32))
    (want, room), _ = c.gradient(f64(c.x), gu[:, :320], gu[:, 320:])
    near(dx, want, room, "dx")


@pytest.mark.parametrize("T,d,w,dtype", [(19999, 64, 2048, BF16), (19999, 64, 1024, F32)])
def test_last_row_tiles_in_parts(T, d, w, dtype):
    """One round of tiles and a little more: the last ones' sums are split and joined."""
    c = Case(T, d, w, dtype)
    D = desc(c)
    guards = [Guarded(T * d * c.x.element_size()), Guarded(M.mcft_ffn_workspace_size(D, T))]
    y = M.mcft_ffn_forward(D, c.x, c.block, y=guards[0].view(dtype, (T, d)), workspace=guards[1].view())
    M.mcft_device_error()
    for g in guards:
        g.check("forward")
    near(y, *c.forward(), "y")
    again = M.mcft_ffn_forward(D, c.x, c.block)
    assert torch.equal(y, again)


@pytest.mark.parametrize("T,d,w", [(3, 128, 192), (200, 320, 448)])
def test_buffers_on_16_bytes(T, d, w):
    """Every tensor 16 bytes past a 32-byte boundary: the same bits."""
    c = Case(T, d, w, BF16)
    D = desc(c)

    def off(t):
        n = 16 // t.element_size()
        buf = torch.empty(t.numel() + 2 * n, dtype=t.dtype, device="cuda")
        v = buf[n:n + t.numel()].view(t.shape)
        v.copy_(t)
        assert v.data_ptr() % 32 == 16
        return v

    def step(x, dy, block, y, ckpt, x8, dx, db):
        M.mcft_ffn_forward(D, x, block, y=y, ckpt=ckpt)
        M.mcft_mx8_quantize(x, q=x8)
        M.mcft_ffn_grad(D, dy, block, x8=x8, ckpt=ckpt, dx=dx, dblock=db)
        return y, ckpt, x8, dx, db, M.mcft_ffn_forward(D, x, block, y=torch.empty_like(y))

    outs = [torch.zeros_like(c.x), torch.zeros(M.mcft_mx8_size(T, 2 * w), dtype=torch.uint8, device="cuda"),
            torch.zeros(M.mcft_mx8_size(T, d), dtype=torch.uint8, device="cuda"), torch.zeros_like(c.x), torch.zeros_like(c.block)]
    want = step(c.x, c.dy, c.block, *outs)
    got = step(off(c.x), off(c.dy), off(c.block), *[off(t) for t in outs])
    M.mcft_device_error()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_tokens(dtype):
    c = Case(0, 64, 128, dtype)
    D = desc(c)
    assert M.mcft_ffn_forward(D, c.x, c.block).shape == (0, 64)
    dx, db = M.mcft_ffn_grad(D, c.dy, c.block, x=c.x)
    assert dx.shape == (0, 64) and not db.any()
    db.fill_(2.0)
    M.mcft_ffn_grad(D, c.dy, c.block, x=c.x, dblock=db, accumulate=True)
    assert bool((db == 2.0).all())


@pytest.mark.parametrize("T", [9, 300])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_bad_token_stays_in_its_row(T, dtype):
    c = Case(T, 192, 320, dtype)
    D = desc(c)
    ckpt = torch.empty(M.mcft_mx8_size(T, 640), dtype=torch.uint8, device="cuda")
    y, dx = M.mcft_ffn_forward(D, c.x, c.block), None
    M.mcft_ffn_forward(D, c.x, c.block, ckpt=ckpt)
    dx, _ = M.mcft_ffn_grad(D, c.dy, c.block, x=c.x, ckpt=ckpt)
    x = c.x.clone()
    x[T // 2, 7], x[1, 3] = float("nan"), float("inf")
    rest = [t for t in range(T) if t not in (T // 2, 1)]
    assert torch.equal(M.mcft_ffn_forward(D, x, c.block)[rest], y[rest])
    bad = M.mcft_ffn_forward(D, x, c.block, ckpt=ckpt)
    assert bool(bad[T // 2].isnan().all())
    got, _ = M.mcft_ffn_grad(D, c.dy, c.block, x=x, ckpt=ckpt)
    assert torch.equal(got[rest], dx[rest]) and bool(got[T // 2].isnan().all())
    M.mcft_device_error()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_of_any_size(dtype):
    """Gates from -3e4 to 3e4: the logistic function's ends, where exp overflows or vanishes."""
    c = Case(130, 64, 64, dtype)
    c.x *= 2.0 ** torch.arange(130, device="cuda").remainder(15)[:, None].to(dtype)
    D = desc(c)
    ckpt = torch.empty(M.mcft_mx8_size(130, 128), dtype=torch.uint8, device="cuda")
    y = M.mcft_ffn_forward(D, c.x, c.block, ckpt=ckpt)
    near(y, *c.forward(), "y")
    dx, db = M.mcft_ffn_grad(D, c.dy, c.block, x=c.x, ckpt=ckpt)
    gu = f64(M.mcft_mx8_dequantize(ckpt, 130, 128, F32))
    (wx, rx), (wb, rb) = c.gradient(f64(c.x), gu[:, :64], gu[:, 64:])
    near(dx, wx, rx, "dx")
    near(db, wb, rb, "dblock")


@pytest.mark.parametrize("T,d,w,dtype", [(3, 256, 320, BF16), (700, 512, 704, BF16), (700, 256, 320, F32)])
def test_same_bits_on_streams_and_replayed(T, d, w, dtype):
    c, c2 = Case(T, d, w, dtype), Case(T, d, w, dtype, 99)
    D = desc(c)

    def step(c, ckpt, ws, stream=None):
        y = M.mcft_ffn_forward(D, c.x, c.block, ckpt=ckpt, workspace=ws, stream=stream)
        few = M.mcft_ffn_forward(D, c.x, c.block, workspace=ws, stream=stream)
        return (y, few, *M.mcft_ffn_grad(D, c.dy, c.block, x=c.x, ckpt=ckpt, workspace=ws, stream=stream),
                *M.mcft_ffn_grad(D, c.dy, c.block, x=c.x, workspace=ws, stream=stream))

    def room():  # (of a larger call: it serves smaller ones)
        n = max(M.mcft_ffn_workspace_size(D, T + 100), M.mcft_ffn_grad_workspace_size(D, T + 100))
        return (torch.empty(M.mcft_mx8_size(T, 2 * w), dtype=torch.uint8, device="cuda"),
                torch.full((n,), 255, dtype=torch.uint8, device="cuda"))

    want, want2 = step(c, *room()), step(c2, *room())
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    rooms = room(), room()
    torch.cuda.synchronize()
    got, got2 = [], []
    for _ in range(3):  # two programs at once
        with torch.cuda.stream(a):
            got = step(c, *rooms[0], stream=a)
        with torch.cuda.stream(b):
            got2 = step(c2, *rooms[1], stream=b.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and all(torch.equal(p, q) for p, q in zip(got2, want2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step(c, *rooms[0])
    c.x.copy_(c2.x), c.dy.copy_(c2.dy), c.block.copy_(c2.block)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(kept, want2))
    M.mcft_device_error()


def test_a_block_trained_from_its_checkpoints():
    """Two blocks of norm, feed-forward and residual with everything that the backward pass reads in 8 bits, against the fp64
    chain. A checkpoint's values are off by at most 2^-4 of themselves, evenly spread: 2^-4 / sqrt(3) in the mean square. A
    gradient's terms hold up to three of them (of x, g or u, and the stream), so it is off by sqrt(3) of that, 2^-4 of its norm;
    errors of the block above add theirs once more for the one below, and bf16's are far smaller."""
    T, d, w = 200, 256, 448
    g = torch.Generator().manual_seed(12)
    D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_BF16)
    blocks = [(torch.randn(3 * w * d, generator=g) / d ** 0.5).bfloat16().cuda() for _ in range(2)]
    gammas = [(1 + 0.1 * torch.randn(d, generator=g)).bfloat16().cuda() for _ in range(2)]
    x0, dout = torch.randn(T, d, generator=g).cuda(), torch.randn(T, d, generator=g).cuda()
    u8s, x8s, ckpts, rstds = ([], [], [], [])
    stream, y = x0, None
    for block, gamma in zip(blocks, gammas):
        x8 = torch.empty(M.mcft_mx8_size(T, d), dtype=torch.uint8, device="cuda")
        ck = torch.empty(M.mcft_mx8_size(T, 2 * w), dtype=torch.uint8, device="cuda")
        stream, u, u8, r = M.mcft_residual_rmsnorm_mx8(D, stream, y, gamma, x8=x8)
        y = M.mcft_ffn_forward(D, u, block, ckpt=ck)
        u8s.append(u8), x8s.append(x8), ckpts.append(ck), rstds.append(r)
    out = stream + y.float()
    grad, dblocks, dgammas = dout, [None, None], [None, None]
    for i in (1, 0):
        du, dblocks[i] = M.mcft_ffn_grad(D, grad.bfloat16(), blocks[i], x8=u8s[i], ckpt=ckpts[i], grad_dtype=F32)
        grad, dgammas[i] = M.mcft_rmsnorm_grad(D, gammas[i], rstds[i], du, dres=grad, x8=x8s[i])
    M.mcft_device_error()
    # the chain in fp64
    leaves = [t.double().cpu().requires_grad_() for t in (x0, *blocks, *gammas)]
    s, n = leaves[0], w * d
    for b, gm in zip(leaves[1:3], leaves[3:]):
        v = s * (s.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gm
        s = s + (torch.nn.functional.silu(v @ b[:n].view(w, d).T) * (v @ b[n:2 * n].view(w, d).T)) @ b[2 * n:].view(d, w).T
    (s * dout.double().cpu()).sum().backward()
    rel = lambda a, b: ((a.double().cpu() - b).norm() / b.norm()).item()  # noqa: E731
    assert rel(out, s.detach()) < 2.0 ** -7
    for got, leaf, room in zip((grad, *dblocks, *dgammas), leaves, (2, 2, 1, 2, 1)):
        assert rel(got, leaf.grad) < room * 2.0 ** -4


def test_offsets_past_32_bits():
    """70000 tokens by 2 x 30784: the checkpoint, dg and du pass 2^32 elements. The last tokens' rows are those of a call on them
    alone up to the order of sums (both within their bounds of the oracle); dW sums over all tokens, of which only the last four
    have a gradient."""
    T, d, w, n = 70_000, 64, 30784, 4
    c = Case(n, d, w, BF16)
    D = desc(c)
    x = torch.randn(T, d, device="cuda").to(BF16)
    dy = torch.zeros(T, d, dtype=BF16, device="cuda")
    x[-n:], dy[-n:] = c.x, c.dy
    ckpt = torch.empty(M.mcft_mx8_size(T, 2 * w), dtype=torch.uint8, device="cuda")
    y = M.mcft_ffn_forward(D, x, c.block, ckpt=ckpt)
    near(y[-n:], *c.forward(), "y")
    gu = M.mcft_mx8_dequantize(ckpt, T, 2 * w, BF16)[-n:]
    g, u, eg, eu = c.projections(f64(c.x))
    want, room = np.concatenate((g, u), 1), np.concatenate((eg, eu), 1)
    near(gu, want, room + 0.5 * oracle.dense.mx8_step(np.abs(want) + room), "checkpoint")
    dx, db = M.mcft_ffn_grad(D, dy, c.block, x=x, ckpt=ckpt)
    gu = f64(gu)
    (wx, rx), (wb, rb) = c.gradient(f64(c.x), gu[:, :w], gu[:, w:])
    near(dx[-n:], wx, rx, "dx")
    near(db, wb, rb, "dblock")
    assert not dx[:-n].any()
    M.mcft_device_error()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [4, 70])
def test_weights_past_32_bits(T, dtype):
    """W1, W3 and W2 of 65600 x 32768: 2^31 elements each and more. All are zero but the last 64 units', whose block by itself
    gives the same values up to the order of sums (both within their bounds of the oracle)."""
    d, w, n = 32768, 65600, 64
    c = Case(T, d, n, dtype)
    D = M.LayerDesc(d, 0, 0, w, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)
    block = torch.zeros(3 * w * d, dtype=dtype, device="cuda")
    parts = lambda b, w: (b[:w * d].view(w, d), b[w * d: 2 * w * d].view(w, d), b[2 * w * d:].view(d, w))  # noqa: E731
    for big, small in zip(parts(block, w)[:2], parts(c.block, n)[:2]):
        big[-n:] = small
    parts(block, w)[2][:, -n:] = parts(c.block, n)[2]
    near(M.mcft_ffn_forward(D, c.x, block), *c.forward(), "y")
    dx, db = M.mcft_ffn_grad(D, c.dy, block, x=c.x)
    M.mcft_device_error()
    del block
    (wx, rx), (wb, rb) = c.gradient(f64(c.x), *c.projections(f64(c.x)))
    near(dx, wx, rx, "dx")
    g1, g3, g2 = parts(db, w)
    last = torch.cat((g1[-n:].flatten(), g3[-n:].flatten(), g2[:, -n:].flatten()))
    near(last, wb, rb, "dblock")
    assert not g1[:-n].any() and not g3[:-n].any() and not g2[:, :-n].any()


def test_tensors_of_the_host_are_refused():
    c = Case(5, 128, 192, BF16)
    D = desc(c)
    gamma = torch.ones(128, dtype=BF16, device="cuda")
    calls = [lambda: M.mcft_mx8_quantize(c.x.cpu()), lambda: M.mcft_mx8_dequantize(M.mcft_mx8_quantize(c.x).cpu(), 5, 128),
             lambda: M.mcft_ffn_forward(D, c.x, c.block.cpu()), lambda: M.mcft_ffn_grad(D, c.dy, c.block, x=c.x.cpu()),
             lambda: M.mcft_residual_rmsnorm_mx8(D, c.x.float(), None, gamma.cpu()),
             lambda: M.mcft_rmsnorm_grad(D, gamma, torch.ones(5), c.dy, x=c.x.float())]
    for i, call in enumerate(calls):
        with pytest.raises(M.MCFTError) as e:
            call()
        assert e.value.status == M.MCFT_ERR_INVALID, i
