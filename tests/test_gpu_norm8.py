"""RMSNorm with the residual's addition and mx8 outputs, and its gradient, against the fp64 oracle.

Tolerances. v = x + y is one fp32 addition: 2^-24 of it. r: the library sums squares to more than fp32, so r is within 2^-23 of
itself, and u = gamma v r within 3 roundings more: 2^-22; in bf16 half a step, 2^-8 of u, comes on top. u8 may differ from the
oracle's by one step where u lies within 2^-22 of the middle between two codes (or of a power-of-two scale's border), and is
equal elsewhere. The gradient's sums run over d (or T) terms, whose fp32 errors are at most n 2^-24 of the sum of magnitudes; their
random walk is far below 2^-18, which the bounds take for all n here (d <= 32768, T <= 4200) beside 2^-22 for the products."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_34077_gb300 import mcft as M
from tests.test_gpu_canary import Guarded

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
WIDTHS = [64, 128, 192, 320, 2048, 2112, 4096, 4160, 8192, 8256, 16384, 16448, 32768]


def desc_of(d, dtype):
    return M.LayerDesc(d, 0, 0, 0, 0, 0, M.MCFT_BF16 if dtype == BF16 else M.MCFT_F32)


def make(T, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g) * torch.exp2(torch.randint(-6, 7, (T, 1), generator=g).float())
    x[:, ::37] *= 7
    return (x, torch.randn(T, d, generator=g).to(dtype), (1 + 0.2 * torch.randn(d, generator=g)).to(dtype),
            torch.randn(T, d, generator=g).to(dtype), torch.randn(T, d, generator=g))


def f64(t):
    return t.double().cpu().numpy()


def near(got, want, room):
    off = np.abs(got - want) - room
    assert (off <= 0).all(), f"{off.max()} over the bound"


def near_codes(q, T, d, exact, rel):
    """mx8 values equal to the oracle's but where `exact` is within rel of itself of another rounding."""
    got = f64(M.mcft_mx8_dequantize(q, T, d, F32))
    want = oracle.dense.mx8(exact)[0]
    lo, hi = oracle.dense.mx8(exact * (1 - rel))[0], oracle.dense.mx8(exact * (1 + rel))[0]
    assert ((got == want) | (got == lo) | (got == hi)).all()
    assert (got != want).mean() < 1e-3


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(T, d) for d in WIDTHS for T in (1, 7)] + [(300, 64), (1000, 320), (65, 4096), (3, 32768)])
def test_forward(T, d, dtype):
    x, y, gamma, _, _ = (t.cuda() for t in make(T, d, dtype, T + d))
    D = desc_of(d, dtype)
    guards = [Guarded(n) for n in (T * d * 4, T * d * x.new_empty(0, dtype=dtype).element_size(), M.mcft_mx8_size(T, d), M.mcft_mx8_size(T, d), T * 4)]
    out, u, u8, x8, rstd = (guards[0].view(F32, (T, d)), guards[1].view(dtype, (T, d)), guards[2].view(), guards[3].view(),
                            guards[4].view(F32, (T,)))
    M.mcft_residual_rmsnorm_mx8(D, x, y, gamma, 1e-5, out=out, u=u, u8=u8, x8=x8, rstd=rstd)
    M.mcft_device_error()
    for g in guards:
        g.check("norm")
    v, uu, r = oracle.dense.norm(f64(x), f64(y), f64(gamma), float(np.float32(1e-5)))
    near(f64(out), v, 2.0 ** -24 * np.abs(v))
    v, uu, r = oracle.dense.norm(f64(out), None, f64(gamma), float(np.float32(1e-5)))  # (of what the kernel has added up)
    near(f64(rstd), r, 2.0 ** -23 * r)
    near(f64(u), uu, (2.0 ** -22 + (2.0 ** -8 if dtype == BF16 else 0)) * np.abs(uu))
    near_codes(u8, T, d, uu, 2.0 ** -22)
    assert torch.equal(x8, M.mcft_mx8_quantize(out))
    # every output by itself, without a residual, and in place
    for k, t in dict(out=out, u=u, u8=u8, x8=x8, rstd=rstd).items():
        only = torch.empty_like(t)
        p = {n: None for n in ("out", "u", "u8", "x8", "rstd")}
        p[k] = only.data_ptr()
        M._check(M.lib().mcft_residual_rmsnorm_mx8(M.C.byref(D), x.data_ptr(), y.data_ptr(), T, gamma.data_ptr(), M.C.c_float(1e-5),
                                                   p["out"], p["u"], p["u8"], p["x8"], p["rstd"], M._stream(None)))
        assert torch.equal(only, t), k
    again = M.mcft_residual_rmsnorm_mx8(D, out, None, gamma, 1e-5)
    assert all(torch.equal(a, b) for a, b in zip(again, (out, u, u8, rstd)))
    stream = x.clone()
    got = M.mcft_residual_rmsnorm_mx8(D, stream, y, gamma, 1e-5, out=stream)
    assert got[0] is stream and torch.equal(stream, out) and torch.equal(got[1], u)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(4201, 1024), (900, 4096), (70, 32768)])
def test_rows_that_are_asked_for_ahead(T, d, dtype):
    """More rows than are asked for at a time, in both directions."""
    test_forward(T, d, dtype)
    test_gradient(T, d, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(T, d) for d in WIDTHS for T in (1, 6)] + [(4200, 64), (1000, 320), (700, 4096), (200, 16384)])
def test_gradient(T, d, dtype):
    x, _, gamma, du, dres = (t.cuda() for t in make(T, d, dtype, 2 * T + d))
    D = desc_of(d, dtype)
    rstd = torch.from_numpy(oracle.dense.norm(f64(x), None, f64(gamma), 1e-5)[2]).float().cuda()
    x8 = M.mcft_mx8_quantize(x)
    for form in ("x", "x8"):
        v = f64(x) if form == "x" else f64(M.mcft_mx8_dequantize(x8, T, d, F32))
        given = dict(x=x) if form == "x" else dict(x8=x8)
        n = v * f64(rstd)[:, None]
        dx, dg = oracle.dense.norm_grad(v, f64(rstd), f64(gamma), f64(du), f64(dres))
        g = np.abs(f64(gamma) * f64(du))
        room = np.abs(dx) * 2.0 ** -23 + f64(rstd)[:, None] * (g + np.abs(n) * (g * np.abs(n)).mean(1, keepdims=True)) * 2.0 ** -18
        room_g = (np.abs(f64(du)) * np.abs(n)).sum(0) * 2.0 ** -18
        guards = [Guarded(T * d * 4), Guarded(d * 4), Guarded(M.mcft_rmsnorm_grad_workspace_size(D, T))]
        got = M.mcft_rmsnorm_grad(D, gamma, rstd, du, dres, **given, dx=guards[0].view(F32, (T, d)), dgamma=guards[1].view(F32, (d,)),
                                  workspace=guards[2].view())
        M.mcft_device_error()
        for q in guards:
            q.check("norm gradient")
        near(f64(got[0]), dx, room)
        near(f64(got[1]), dg, room_g)
        # without a residual gradient; in place over it; added to
        alone = M.mcft_rmsnorm_grad(D, gamma, rstd, du, **given)
        near(f64(alone[0]), dx - f64(dres), room)
        assert torch.equal(alone[1], got[1])
        stream = dres.clone()
        M.mcft_rmsnorm_grad(D, gamma, rstd, du, stream, **given, dx=stream, dgamma=alone[1], accumulate=True)
        assert torch.equal(stream, got[0])
        near(f64(alone[1]), 2 * dg, 3 * room_g)
        # one of the two alone
        for skip in (0, 1):
            outs = [torch.full_like(t, 3.0) for t in got]
            p = [None if i == skip else t.data_ptr() for i, t in enumerate(outs)]
            ws = torch.empty(M.mcft_rmsnorm_grad_workspace_size(D, T), dtype=torch.uint8, device="cuda")
            M._check(M.lib().mcft_rmsnorm_grad(M.C.byref(D), given["x"].data_ptr() if form == "x" else None,
                                               x8.data_ptr() if form == "x8" else None, rstd.data_ptr(), gamma.data_ptr(),
                                               du.data_ptr(), T, dres.data_ptr(), p[0], p[1], 0, ws.data_ptr() if p[1] else None,
                                               ws.numel() if p[1] else 0, M._stream(None)))
            assert torch.equal(outs[1 - skip], got[1 - skip]) and bool((outs[skip] == 3.0).all())


def test_gradient_is_the_slope():
    """Differences of the fp32 forward: u moves by h du/dx, h large against the fp32 steps of u (2^-24) and small enough for
    the second derivative: (h^2 + 2^-22 / h) of the values' size, at h = 2^-7 under 2^-13."""
    T, d = 2, 64
    x, _, gamma, du, _ = (t.cuda() for t in make(T, d, F32, 3))
    x = x / x.square().mean(1, keepdim=True).sqrt()
    D = desc_of(d, F32)
    _, _, _, rstd = M.mcft_residual_rmsnorm_mx8(D, x, None, gamma)
    dx, dgamma = M.mcft_rmsnorm_grad(D, gamma, rstd, du, x=x)
    loss = lambda v, w: (M.mcft_residual_rmsnorm_mx8(D, v, None, w)[1].double() * du.double()).sum().item()  # noqa: E731
    h = 2.0 ** -7
    room = 2.0 ** -13 * (du.abs() * gamma.abs()).sum().item()
    for j in range(0, d, 7):
        e = torch.zeros_like(x)
        e[1, j] = h
        assert abs((loss(x + e, gamma) - loss(x - e, gamma)) / (2 * h) - dx[1, j].item()) < room
        assert abs((loss(x, gamma + e[1]) - loss(x, gamma - e[1])) / (2 * h) - dgamma[j].item()) < room


def test_no_tokens():
    D = desc_of(128, BF16)
    gamma, empty = torch.ones(128, dtype=BF16, device="cuda"), torch.empty(0, 128, device="cuda")
    out, u, u8, rstd = M.mcft_residual_rmsnorm_mx8(D, empty, None, gamma)
    assert out.shape == u.shape == (0, 128) and u8.numel() == 0 and rstd.shape == (0,)
    _, dg = M.mcft_rmsnorm_grad(D, gamma, rstd, u, x=empty)
    assert not dg.any()
    dg.fill_(2.0)
    M.mcft_rmsnorm_grad(D, gamma, rstd, u, x=empty, dgamma=dg, accumulate=True)
    assert bool((dg == 2.0).all())


@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_of_extremes(eps):
    """Rows of zeros (r = 1 / sqrt(eps); with eps 0 the quotient 0 / 0), of huge values whose squares overflow (r = 0), of tiny ones,
    and with a NaN or an infinity, each of which stays in its row."""
    d = 256
    x = torch.randn(6, d)
    x[0], x[1], x[2] = 0.0, x[1] * 1e30, x[2] * 1e-25
    x[3, 5], x[4, 9] = float("nan"), float("inf")
    D, gamma = desc_of(d, F32), torch.ones(d).cuda()
    _, u, u8, rstd = M.mcft_residual_rmsnorm_mx8(D, x.cuda(), None, gamma, eps)
    u, r = u.cpu(), rstd.cpu()
    assert bool(u[3].isnan().all()) and bool(u[4, 9].isnan()) and r[4] == 0 and bool(u[5].isfinite().all())
    assert r[1] == 0 and not u[1].any()
    if eps:
        assert not u[0].any() and abs(r[0] - eps ** -0.5) <= 2.0 ** -22 * r[0]
    else:
        assert r[0] == float("inf") and bool(u[0].isnan().all())
    back = M.mcft_mx8_dequantize(u8, 6, d, F32).cpu()
    assert bool(back[3].isnan().all()) and bool(back[4].view(-1, 32)[0].isnan().all()) and not back[1].any()
    assert bool(back[5].isfinite().all())


@pytest.mark.parametrize("T,d", [(5, 192), (700, 4096)])
def test_same_bits_on_a_stream_and_replayed(T, d):
    x, y, gamma, du, dres = (t.cuda() for t in make(T, d, BF16, 8))
    D = desc_of(d, BF16)
    x8 = torch.empty(M.mcft_mx8_size(T, d), dtype=torch.uint8, device="cuda")
    ws = torch.empty(M.mcft_rmsnorm_grad_workspace_size(D, 4096), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        out, u, u8, r = M.mcft_residual_rmsnorm_mx8(D, x, y, gamma, x8=x8, stream=stream)
        dx, dg = M.mcft_rmsnorm_grad(D, gamma, r, du, dres, x8=x8, workspace=ws, stream=stream)
        return out, u, u8, r, dx, dg, x8.clone()

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for t in kept:
        t.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, want))
    M.mcft_device_error()


def test_offsets_past_32_bits():
    T, d = 132_000, 32768  # 4.3e9 values
    D = desc_of(d, BF16)
    x = torch.zeros(T, d, device="cuda")
    last, _, gamma, du, _ = (t.cuda() for t in make(2, d, BF16, 5))
    x[-2:] = last
    u8 = torch.empty(M.mcft_mx8_size(T, d), dtype=torch.uint8, device="cuda")
    M._check(M.lib().mcft_residual_rmsnorm_mx8(M.C.byref(D), x.data_ptr(), None, T, gamma.data_ptr(), M.C.c_float(1e-5), None, None,
                                               u8.data_ptr(), None, None, M._stream(None)))
    _, _, want, rstd = M.mcft_residual_rmsnorm_mx8(D, last, None, gamma)
    n = T * d
    assert torch.equal(u8[n - 2 * d: n], want[:2 * d]) and torch.equal(u8[n + n // 32 - d // 16:], want[2 * d:])
    del u8
    grad, dg = M.mcft_rmsnorm_grad(D, gamma, rstd, du, x=last)
    big = torch.zeros(T, d, dtype=BF16, device="cuda")
    big[-2:] = du
    r = torch.ones(T, device="cuda")
    r[-2:] = rstd
    M.mcft_rmsnorm_grad(D, gamma, r, big, x=x, dx=x)
    assert torch.equal(x[-2:], grad) and not x[:100].any()
    M.mcft_device_error()
