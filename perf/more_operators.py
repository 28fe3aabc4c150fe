"""Timing and comparison cases of the dense gated feed-forward block, its 8-bit (mx8) activation checkpoints and
the RMSNorm that feeds it, forward and backward.

Five operators, each in a plain form (elementary torch operations, 32-bit arithmetic) and through the library's own
calls:

* ``norm``: the residual added to the fp32 stream, RMSNorm of the sum, and the norm's output and the stream in
  microscaled 8-bit floating point (e4m3 values, one power-of-two scale for each 32 along a row);
* ``normgrad``: the gradient of that norm, added to the stream's gradient, and the scales' gradient;
* ``ffn``: y = W2 (silu(W1 x) * (W3 x)) for every token, W1, W3 and W2 one packed block;
* ``train``: the same forward and its gradients, dx and the block's, either from the 8-bit checkpoints of x and of
  both projections or (without checkpoints) from x itself;
* ``quant``: rows to that 8-bit format and back to the values they stand for.

Sizes are those of the layer shapes in ``paper_2609_34077_gb300/inputs.py`` and generic ones around them.
"""
import math

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
LARGEST = 448.0  # of e4m3


def listed():
    return [
        # one decoded token ahead of a layer of the DeepSeek-V2-Lite shape: launch latency
        dict(name="norm token", op="norm", T=1, d=2048, dtype="bf16", residual=True, stream8=False),
        # a fine-tuning batch at the Mixtral shape's width, both checkpoints written
        dict(name="norm batch", op="norm", T=8192, d=4096, dtype="bf16", residual=True, stream8=True),
        # its gradient from the 8-bit stream
        dict(name="normgrad batch", op="normgrad", T=8192, d=4096, dtype="bf16", stream8=True),
        # an odd token count in 32 bits, from the stream itself
        dict(name="normgrad odd f32", op="normgrad", T=1999, d=2048, dtype="f32", stream8=False),
        # one decoded token through a shared expert of the DeepSeek-V2-Lite shape
        dict(name="ffn token", op="ffn", T=1, d=2048, w=1408, dtype="bf16"),
        # a decode batch through a dense block of the Mixtral expert's shape: the weights are read once
        dict(name="ffn batch", op="ffn", T=16, d=4096, w=14336, dtype="bf16"),
        # a prompt through the same block
        dict(name="ffn prompt", op="ffn", T=4096, d=4096, w=14336, dtype="bf16"),
        # a small fine-tuning step, odd sizes, without checkpoints
        dict(name="train odd", op="train", T=1023, d=960, w=704, dtype="bf16", ckpt=False),
        # a fine-tuning step of a shared expert of the DeepSeek-V2-Lite shape from its checkpoints
        dict(name="train shared", op="train", T=4096, d=2048, w=1408, dtype="bf16", ckpt=True),
        # a fine-tuning step of the large block from its checkpoints
        dict(name="train batch", op="train", T=4096, d=4096, w=14336, dtype="bf16", ckpt=True),
        # a step in 32 bits
        dict(name="train f32", op="train", T=512, d=1024, w=1408, dtype="f32", ckpt=False),
        # what a layer's checkpoint of both projections is, there and back
        dict(name="quant checkpoint", op="quant", R=4096, C=28672, dtype="bf16"),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(("norm", "normgrad", "ffn", "ffn", "train", "train", "train", "quant"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if op in ("norm", "normgrad"):
        T = _log(rng, 1, 32768)
        c = dict(op=op, T=T, d=_log(rng, 64, max(128, min(16384, 33_000_000 // T)), 64), dtype=dtype, stream8=rng.random() < 0.5)
        return dict(c, residual=rng.random() < 0.7) if op == "norm" else c
    if op == "quant":
        R = _log(rng, 1, 32768)
        return dict(op="quant", R=R, C=_log(rng, 16, max(64, min(32768, 110_000_000 // R)), rng.choice((1, 32))), dtype=dtype)
    while True:
        T, d, w = _log(rng, 1, 8192), _log(rng, 64, 4096, 64), _log(rng, 64, 14336, 64)
        c = dict(op=op, T=T, d=d, w=w, dtype=dtype)
        if op == "train":  # (in 32 bits a rounding to 8 bits of a sum's last place is a difference of its own)
            c["ckpt"] = dtype == "bf16" and rng.random() < 0.6
        if T * d * w <= (4e9 if dtype == "f32" else 2.4e11 if op == "ffn" else 1.8e11):
            return c


def work(case):
    c = case
    if c["op"] == "quant":
        return {"bytes": 2 * c["R"] * c["C"] * (4 if c["dtype"] == "f32" else 2), "flops": 0}
    eb = 4 if c["dtype"] == "f32" else 2
    T, d = c["T"], c["d"]
    mx = 1 + 1 / 32
    if c["op"] == "norm":
        return {"bytes": T * d * (4 + 4 + (eb if c["residual"] else 0) + eb + mx + (mx if c["stream8"] else 0)) + T * 4 + d * eb,
                "flops": 0}
    if c["op"] == "normgrad":
        return {"bytes": T * d * ((mx if c["stream8"] else 4) + eb + 4 + 4) + T * 4 + d * (eb + 4), "flops": 0}
    w = c["w"]
    by, fl = 3 * w * d * eb + 2 * T * d * eb, 6 * T * d * w
    if c["op"] == "train":  # dy read, dx written, the weights' gradients written; three more products of each size
        by += 2 * T * d * eb + 3 * w * d * eb
        fl += 12 * T * d * w
        if c["ckpt"]:
            by += 2 * T * (2 * w + d) * mx
    return {"bytes": by, "flops": fl}


# ---- inputs ----


def _normal(g, *shape, std=1.0, dtype=BF16):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=F32) * std).to(dtype)


def _inputs(case, seed):
    """The tensors of a case by name, in the types in which a program holds them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = F32 if case["dtype"] == "f32" else BF16
    if case["op"] == "quant":
        x = _normal(g, case["R"], case["C"], dtype=dt)
        x[::7] *= 2.0 ** -9  # rows of other magnitudes
        x[:, ::64] *= 8  # outlying columns, as activations have them
        return dict(x=x)
    T, d = case["T"], case["d"]
    if case["op"] in ("norm", "normgrad"):
        s = dict(x=_normal(g, T, d, std=1.5, dtype=F32), gamma=1 + _normal(g, d, std=0.1, dtype=F32))
        s["x"][:, ::97] *= 6  # a few wide units, as residual streams have them
        s["gamma"] = s["gamma"].to(dt)
        if case["op"] == "norm":
            s["y"] = _normal(g, T, d, dtype=dt) if case["residual"] else None
        else:
            s["du"], s["dres"] = _normal(g, T, d, std=0.1, dtype=dt), _normal(g, T, d, std=0.1, dtype=F32)
            s["rstd"] = (s["x"].double().square().mean(1) + EPS).rsqrt().float()  # as the forward left it
        return s
    w = case["w"]
    s = dict(x=_normal(g, T, d, dtype=dt), block=_normal(g, 3 * w * d, std=1.28 / math.sqrt(d), dtype=dt))
    if case["op"] == "train":
        s["dy"] = _normal(g, T, d, std=0.1, dtype=dt)
    return s


EPS = 1e-5


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if not own and case["op"] == "normgrad" and case["stream8"]:
        s["x"] = _mx8(s["x"])
    if own:
        from paper_2609_34077_gb300 import mcft as M
        if case["op"] == "quant":
            return s
        s["desc"] = desc = M.LayerDesc(case["d"], 1, 1, case.get("w", 64), 0, M.MCFT_GATE_RENORM,
                                       M.MCFT_F32 if case["dtype"] == "f32" else M.MCFT_BF16)
        T, n = case["T"], 0
        if case["op"] == "normgrad":
            n = M.mcft_rmsnorm_grad_workspace_size(desc, T)
            if case["stream8"]:  # what the forward wrote
                s["x8"], s["x"] = M.mcft_mx8_quantize(s["x"]), None
        elif case["op"] in ("ffn", "train"):
            n = M.mcft_ffn_workspace_size(desc, T)
            if case["op"] == "train":
                n = max(n, M.mcft_ffn_grad_workspace_size(desc, T))
        s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms ----


def _power(e):
    """2^e in 32 bits from its bits, exact (e from -126 to 127)."""
    return ((e + 127) << 23).view(F32)


def _mx8(x):
    """The values, in 32 bits, that x [R, C] reads back as from the 8-bit format: blocks of 32 along a row under the
    smallest power of two with max|x| <= 448 of it, each value rounded to four significant bits (even ties), or
    to a multiple of 2^-9 where it is below 2^-6. (Inputs are far from the ends of the exponents' range.)"""
    R, C = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -C % 32)).view(R, -1, 32)
    m, e = torch.frexp(v.abs().amax(2, keepdim=True))  # m in [0.5, 1)
    s = torch.where(m > 0, e - 9 + (m > LARGEST / 512), -126).clamp(min=-126)
    a = v * _power(-s)
    step = _power(torch.frexp(a).exponent.clamp(min=-5) - 4)  # a power of two: quotient and product are exact
    return (torch.round(a / step) * step * _power(s)).flatten(1)[:, :C].contiguous()


def _plain_norm(c, x, y, gamma):
    out = x if y is None else x + y.float()
    r = 1 / torch.sqrt(out.square().mean(1) + EPS)
    u = out * r[:, None] * gamma.float()
    got = {"out": out, "u": u.to(gamma.dtype), "u8": _mx8(u).to(BF16), "rstd": r}
    if c["stream8"]:
        got["x8"] = _mx8(out).to(BF16)
    return got


def _plain_normgrad(x, gamma, rstd, du, dres):
    xh = x * rstd[:, None]
    g = du.float() * gamma.float()
    return {"dx": dres + rstd[:, None] * (g - xh * (g * xh).mean(1, keepdim=True)), "dgamma": (du.float() * xh).sum(0)}


def _plain_ffn(c, s):
    d, w = c["d"], c["w"]
    x, block = s["x"].float(), s["block"].float()
    w1, w3, w2 = block[: w * d].view(w, d), block[w * d: 2 * w * d].view(w, d), block[2 * w * d:].view(d, w)
    g, u = x @ w1.T, x @ w3.T
    y = ((g * torch.sigmoid(g) * u) @ w2.T).to(s["x"].dtype)
    if c["op"] == "ffn":
        return y
    if c["ckpt"]:
        x, g, u = _mx8(x), _mx8(g), _mx8(u)
    sig = torch.sigmoid(g)
    dy = s["dy"].float()
    dh = dy @ w2
    dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
    dblock = torch.cat(((dg.T @ x).flatten(), (du.T @ x).flatten(), (dy.T @ (g * sig * u)).flatten()))
    return {"y": y, "dx": (dg @ w1 + du @ w3).to(y.dtype), "dblock": dblock.to(y.dtype)}


def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    if c["op"] == "norm":
        return _plain_norm(c, s["x"], s["y"], s["gamma"])
    if c["op"] == "normgrad":
        return _plain_normgrad(s["x"], s["gamma"], s["rstd"], s["du"], s["dres"])
    if c["op"] == "quant":
        return _mx8(s["x"]).to(s["x"].dtype)
    return _plain_ffn(c, s)


# ---- the library's calls ----


def _own(s, c):
    from paper_2609_34077_gb300 import mcft as M
    if c["op"] == "quant":
        return M.mcft_mx8_dequantize(M.mcft_mx8_quantize(s["x"]), c["R"], c["C"], s["x"].dtype)
    if c["op"] == "norm":
        T, d = c["T"], c["d"]
        x8 = torch.empty(M.mcft_mx8_size(T, d), dtype=torch.uint8, device="cuda") if c["stream8"] else None
        out, u, u8, rstd = M.mcft_residual_rmsnorm_mx8(s["desc"], s["x"], s["y"], s["gamma"], eps=EPS, x8=x8)
        got = {"out": out, "u": u, "u8": M.mcft_mx8_dequantize(u8, T, d, BF16), "rstd": rstd}
        if c["stream8"]:
            got["x8"] = M.mcft_mx8_dequantize(x8, T, d, BF16)
        return got
    if c["op"] == "normgrad":
        dx, dgamma = M.mcft_rmsnorm_grad(s["desc"], s["gamma"], s["rstd"], s["du"], dres=s["dres"], x=s["x"],
                                         x8=s.get("x8"), workspace=s["ws"])
        return {"dx": dx, "dgamma": dgamma}
    if c["op"] == "ffn":
        return M.mcft_ffn_forward(s["desc"], s["x"], s["block"], workspace=s["ws"])
    if not c["ckpt"]:
        y = M.mcft_ffn_forward(s["desc"], s["x"], s["block"], workspace=s["ws"])
        dx, dblock = M.mcft_ffn_grad(s["desc"], s["dy"], s["block"], x=s["x"], workspace=s["ws"])
    else:
        ckpt = torch.empty(M.mcft_mx8_size(c["T"], 2 * c["w"]), dtype=torch.uint8, device="cuda")
        y = M.mcft_ffn_forward(s["desc"], s["x"], s["block"], ckpt=ckpt, workspace=s["ws"])
        dx, dblock = M.mcft_ffn_grad(s["desc"], s["dy"], s["block"], x8=M.mcft_mx8_quantize(s["x"]), ckpt=ckpt,
                                     workspace=s["ws"])
    return {"y": y, "dx": dx, "dblock": dblock}


# ---- the definitions in 64 bits ----


def _fake64(x):
    """x [R, C] in 64 bits, each 32 along a row rounded to the e4m3 grid under their power-of-two scale."""
    R, C = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -C % 32)).reshape(R, -1, 32)
    big = v.abs().amax(2, keepdim=True)
    power = lambda n: ((n + 1023) << 52).view(torch.float64)  # noqa: E731 (exact, where exp2 need not be)
    s = torch.ceil(torch.log2(torch.where(big > 0, big, 1.0) / LARGEST)).long()
    s = torch.where(power(s - 1) * LARGEST >= big, s - 1, torch.where(power(s) * LARGEST < big, s + 1, s))  # where log2 rounded
    s = torch.where(big > 0, s, -127).clamp(-127, 127)
    a = v.abs() / power(s)
    near = torch.floor(torch.log2(a.clamp_min(2.0 ** -6))).long()
    near = torch.where(power(near) > a.clamp_min(2.0 ** -6), near - 1, torch.where(power(near + 1) <= a, near + 1, near))
    grid = power(near - 3)
    low = torch.floor(a / grid)
    rest = a / grid - low
    q = low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1))).double()
    return (torch.sign(v) * q * grid * power(s)).reshape(R, -1)[:, :C]


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["op"] == "quant":
        return _fake64(s["x"])
    if c["op"] == "norm":
        out = s["x"].double() + (0 if s["y"] is None else s["y"].double())
        rms = torch.sqrt((out * out).sum(1) / c["d"] + EPS)
        u = s["gamma"].double() * (out / rms[:, None])
        got = {"out": out, "u": u, "u8": _fake64(u), "rstd": 1 / rms}
        if c["stream8"]:
            got["x8"] = _fake64(out.float())  # the stream is held in 32 bits
        return got
    if c["op"] == "normgrad":
        x = _fake64(s["x"]) if c["stream8"] else s["x"].double()
        r, gam, du = s["rstd"].double()[:, None], s["gamma"].double(), s["du"].double()
        dot = (x * gam * du).sum(1, keepdim=True)
        return {"dx": s["dres"].double() + gam * du * r - x * dot * r ** 3 / c["d"], "dgamma": torch.einsum("td,td->d", du, x * r)}
    d, w = c["d"], c["w"]
    x = s["x"].double()
    w13, w2 = s["block"][: 2 * w * d].view(2 * w, d).double(), s["block"][2 * w * d:].view(d, w).double()
    gu = x @ w13.T
    silu = lambda v: v / (1 + torch.exp(-v))  # noqa: E731
    y = (silu(gu[:, :w]) * gu[:, w:]) @ w2.T
    if c["op"] == "ffn":
        return y
    if c["ckpt"]:
        x, gu = _fake64(x), _fake64(gu)
    g, u = gu[:, :w], gu[:, w:]
    dy = s["dy"].double()
    dh = dy @ w2
    slope = (1 + torch.exp(-g) * (1 + g)) / (1 + torch.exp(-g)) ** 2  # of silu
    dgu = torch.cat((dh * u * slope, dh * silu(g)), 1)
    dblock = torch.cat(((dgu.T @ x).flatten(), (dy.T @ (silu(g) * u)).flatten()))
    return {"y": y, "dx": dgu @ w13, "dblock": dblock}
