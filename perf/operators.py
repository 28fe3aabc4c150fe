"""Timing and comparison cases of the scored routing and the 4-bit (mx4) operators.

Five operators, each in a plain form (elementary torch operations, 32-bit arithmetic) and through the
library's own calls:

* ``route``: router product, softmax or sigmoid scores, a balance bias, expert groups, Top-K, gates and the
  experts' loads; with ``train`` also the gradients of the router and of its input;
* ``quant``: rows to microscaled 4-bit floating point (e2m1 values, one power-of-two scale for each 32
  along a row) and back to the values they stand for;
* ``matmul``: the product A B^T of two such matrices;
* ``experts``: the routed layer forward with 4-bit expert blocks (input and hidden activations quantised
  to the same format).

Sizes are those of the layer shapes in ``paper_2609_34077_gb300/inputs.py`` and generic ones around them.
"""
import math

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
MID_DOWN = (0.25, 1.25, 2.5, 5.0)  # midpoints of the e2m1 grid whose tie goes down, and up
MID_UP = (0.75, 1.75, 3.5)
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _route(name, T, d, E, K, *, score="softmax", groups=1, keep_groups=1, group_top=1, renorm=True, scale=1.0,
           bias=False, masked=0, train=False, dtype="bf16"):
    named = {} if name is None else {"name": name}
    return dict(named, op="route", T=T, d=d, E=E, K=K, score=score, groups=groups, keep_groups=keep_groups,
                group_top=group_top, renorm=renorm, scale=scale, bias=bias, masked=masked, train=train, dtype=dtype)


def listed():
    return [
        # one decoded token through the 64-expert router of the DeepSeek-V2-Lite shape: launch latency
        _route("route token", 1, 2048, 64, 6, renorm=False),
        # a prompt through a grouped 256-expert router with a balance bias
        _route("route prompt groups", 4096, 4096, 256, 8, score="sigmoid", groups=8, keep_groups=4, group_top=2,
               scale=2.5, bias=True),
        # a fine-tuning step under a hard mask (16 of 64 experts eligible), odd token count; the softmax
        # gradient reaches every expert
        _route("route train masked", 1999, 2048, 64, 6, renorm=False, masked=48, train=True),
        # a fine-tuning step of the large grouped router
        _route("route train groups", 8192, 4096, 256, 8, score="sigmoid", groups=8, keep_groups=4, group_top=2,
               scale=2.5, bias=True, train=True),
        # activations of one decode batch, rows of the Mixtral shape
        dict(name="quant activations", op="quant", R=16, C=4096, dtype="bf16"),
        # the gate and up weights of one Mixtral expert
        dict(name="quant expert", op="quant", R=28672, C=4096, dtype="bf16"),
        # one token through a dense down projection of the Mixtral shape: the weights are read once
        dict(name="matmul token", op="matmul", M=1, N=4096, K=14336, out="bf16"),
        # ragged sizes, 32-bit result
        dict(name="matmul ragged", op="matmul", M=333, N=1000, K=1440, out="f32"),
        # a prompt through a dense up projection of the Mixtral shape
        dict(name="matmul prompt", op="matmul", M=4096, N=14336, K=4096, out="bf16"),
        # one decoded token through a DeepSeek-V2-Lite-shaped layer
        dict(name="experts token", op="experts", T=1, d=2048, w=1408, E=64, K=6, S=2, drop=0.0),
        # a decode batch through a Mixtral-shaped layer
        dict(name="experts batch", op="experts", T=16, d=4096, w=14336, E=8, K=2, S=0, drop=0.0),
        # a prompt through a DeepSeek-V2-Lite-shaped layer
        dict(name="experts prompt", op="experts", T=4096, d=2048, w=1408, E=64, K=6, S=2, drop=0.0),
    ]


def _log(rng, lo, hi, step=1):
    v = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))
    return v + step if v == 3072 else v


def draw(rng):
    op = rng.choice(("route", "route", "quant", "matmul", "experts", "experts"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * _log(rng, 8 if groups == 1 else 4, 256 // groups)
        K = rng.randint(1, min(8, max(1, E // 4)))
        keep = rng.randint(max(1, math.ceil(K * groups / E)), groups)
        train, T, d = rng.random() < 0.5, _log(rng, 1, 8192), _log(rng, 256, 4096, 64)
        if dtype == "f32":
            T = min(T, 2048)
        masked = rng.randint(0, E // 2) if groups == 1 and rng.random() < 0.3 else 0
        return _route(None, T, d, E, K, score=rng.choice(("softmax", "sigmoid")), groups=groups, keep_groups=keep,
                      group_top=rng.randint(1, 2), renorm=rng.random() < 0.5, scale=rng.choice((1.0, 2.5)),
                      bias=rng.random() < 0.6, masked=masked, train=train, dtype=dtype)
    if op == "quant":
        R = _log(rng, 1, 32768)
        return dict(op="quant", R=R, C=_log(rng, 32, max(64, min(16384, 110_000_000 // R)), rng.choice((1, 32))), dtype=dtype)
    if op == "matmul":
        while True:
            c = dict(op="matmul", M=_log(rng, 1, 8192), N=_log(rng, 64, 16384), K=_log(rng, 64, 16384, 32),
                     out=rng.choice(("bf16", "bf16", "f32")))
            if 2 * c["M"] * c["N"] * c["K"] <= 4.8e11:
                return c
    while True:
        E = _log(rng, 2, 256)
        c = dict(op="experts", T=_log(rng, 1, 8192), d=_log(rng, 256, 4096, 64), w=_log(rng, 128, 8192, 64), E=E,
                 K=rng.randint(1, min(8, E)), S=rng.choice((0, 0, 1, 2)), drop=rng.choice((0.0, 0.0, 0.1)))
        if 3 * E * c["d"] * c["w"] <= 1.2e9 and 6 * c["T"] * (c["K"] + c["S"]) * c["d"] * c["w"] <= 5.6e11:
            return c


def _mx4_bytes(rows, cols):
    return rows * cols * (0.5 + 1 / 32)


def work(case):
    c = case
    if c["op"] == "route":
        eb = 4 if c["dtype"] == "f32" else 2
        T, d, E, K = c["T"], c["d"], c["E"], c["K"]
        by, fl = (T + E) * d * eb + T * K * 8 + E * 4, 2 * T * d * E
        if c["train"]:  # the input read again, its gradient and the router's written; both products
            by += 2 * T * d * eb + E * d * (eb + 4) + T * K * 4
            fl += 4 * T * d * (E if c["score"] == "softmax" and not c["renorm"] else K)
        return {"bytes": by, "flops": fl}
    if c["op"] == "quant":
        return {"bytes": 2 * c["R"] * c["C"] * (4 if c["dtype"] == "f32" else 2), "flops": 0}
    if c["op"] == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": _mx4_bytes(M + N, K) + M * N * (4 if c["out"] == "f32" else 2), "flops": 2 * M * N * K}
    T, d, w, E, K, S = (c[k] for k in ("T", "d", "w", "E", "K", "S"))
    live = E * (1 - (1 - K / E) ** T) if K < E else E
    return {"bytes": _mx4_bytes((live + S) * 3 * w, d) + 2 * T * d * 2 + T * K * 8, "flops": 6 * T * (K * (1 - c["drop"]) + S) * d * w}


# ---- inputs ----


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=BF16):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=F32) * std).to(dtype)


def _scores64(case, x, w, bias):
    """Scores, choice values and their group-filtered form in 64 bits."""
    z = x.double() @ w.double().T
    s = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, 1)
    c = s if bias is None else s + bias.double()
    if case["groups"] > 1:
        G = case["groups"]
        by = c.view(-1, G, c.shape[1] // G)
        gs = by.sort(2, descending=True).values[..., : case["group_top"]].sum(2)
        keep = torch.zeros_like(gs).scatter_(1, gs.sort(dim=1, descending=True, stable=True).indices[:, : case["keep_groups"]], 1.0)
        return z, s, torch.where(keep[..., None] > 0, by, -math.inf).flatten(1), gs
    return z, s, c, None


def _clear(case, x, w, bias):
    """Tokens whose decisions do not hang on the last bits of a score: every pair of neighbours among the
    K + 1 best choices, and the last group kept and the first left out, are apart."""
    _, s, c, gs = _scores64(case, x, w, bias)
    K = case["K"]
    top = c.sort(1, descending=True).values[:, : K + 1]
    unit = s.sort(1, descending=True).values[:, min(K, s.shape[1] - 1)][:, None] + (0.01 if bias is not None else 0.0)
    far = ((top[:, :-1] - top[:, 1:]) > 1e-4 * unit) | (top[:, 1:] == -math.inf)
    ok = far.all(1)
    if gs is not None and case["keep_groups"] < case["groups"]:
        gt = gs.sort(1, descending=True).values
        k = case["keep_groups"]
        ok &= (gt[:, k - 1] - gt[:, k]) > 1e-4 * unit[:, 0]
    return ok


def _route_inputs(case, seed):
    g = _gen(seed)
    T, d, E = case["T"], case["d"], case["E"]
    dtype = F32 if case["dtype"] == "f32" else BF16
    w = _normal(g, E, d, std=1.28 / math.sqrt(d), dtype=dtype)
    bias = None
    if case["bias"] or case["masked"]:
        spread = 0.05 if case["score"] == "sigmoid" else 0.2 / E
        bias = torch.randn(E, generator=g, device="cuda") * (spread if case["bias"] else 0.0)
        if case["masked"]:
            bias[torch.randperm(E, generator=g, device="cuda")[: case["masked"]]] = -math.inf
    # a few more tokens than asked for, those with a near tie last: near ties are left out
    x = _normal(g, T + T // 4 + 32, d, dtype=dtype)
    ok = _clear(case, x, w, bias)
    x = x[torch.argsort(ok.logical_not().to(torch.int8), stable=True)[:T]].contiguous()
    dgate = torch.randn(T, case["K"], generator=g, device="cuda") if case["train"] else None
    return x, w, bias, dgate


def _mx4(x):
    """x [R, C] -> (codes [R, C32 / 2] of two 4-bit values each, scale exponents + 127 [R, C32 / 32]), C
    padded with zeros to a multiple of 32."""
    R, C = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -C % 32)).view(R, -1, 32)
    e = torch.frexp(v.abs().amax(2, keepdim=True)).exponent - 3
    e = torch.where(v.abs().amax(2, keepdim=True) > 0, e, -127).clamp(-127, 127)
    a = v.abs() * ((127 - e) << 23).view(F32)  # 2^-e, from its bits: exact
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.clamp(torch.round(a / step) * step, max=6.0)
    code = torch.where(q < 2, q * 2, torch.where(q < 4, q + 2, q / 2 + 4)).to(torch.uint8)
    code = torch.where(v < 0, code + 8, code).view(R, -1, 2)
    return code[..., 0] + 16 * code[..., 1], (e[..., 0] + 127).to(torch.uint8)


def _values(codes, scales, C):
    """The values that codes and scales stand for, in 32 bits: [..., C]."""
    lut = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    unit = torch.where(scales > 0, scales.int() << 23, 1 << 22).view(F32)  # 2^(scale - 127), from its bits
    v = lut[both].unflatten(-1, (-1, 32)) * unit[..., None]
    return v.flatten(-2)[..., :C]


def _quant_input(case, seed):
    x = _normal(_gen(seed), case["R"], case["C"], dtype=F32 if case["dtype"] == "f32" else BF16)
    x[::7] *= 2.0 ** -9  # rows of other magnitudes
    x[:, ::64] *= 8  # outlying columns, as activations have them
    return x


def _matmul_inputs(case, seed):
    g = _gen(seed)
    return _normal(g, case["M"], case["K"]), _normal(g, case["N"], case["K"], std=0.02)


def _expert_inputs(case, seed):
    """Input, routing, and the generator that _expert_weights goes on with."""
    g = _gen(seed)
    T, E, K = case["T"], case["E"], case["K"]
    x = _normal(g, T, case["d"])
    fav = torch.randn(T, E, generator=g, device="cuda") + 0.7 * torch.randn(E, generator=g, device="cuda")
    idx = fav.topk(K, 1).indices.int()
    gate = torch.softmax(torch.randn(T, K, generator=g, device="cuda"), 1)
    if case["drop"]:  # entries, and whole rows, without an expert
        idx[torch.rand(T, K, generator=g, device="cuda") < case["drop"]] = -1
        idx[torch.rand(T, generator=g, device="cuda") < case["drop"] / 2] = -1
    return x, idx.contiguous(), gate.contiguous(), g


def _expert_weights(case, g):
    """One expert after another: its packed block [W1 | W3 | W2]."""
    for _ in range(case["E"] + case["S"]):
        yield _normal(g, 3 * case["w"] * case["d"], std=0.02)


def prepare(case, seed):
    s = dict(case=case)
    if case["op"] == "route":
        s["x"], s["w"], s["bias"], s["dgate"] = _route_inputs(case, seed)
    elif case["op"] == "quant":
        s["x"] = _quant_input(case, seed)
    elif case["op"] == "matmul":
        a, b = _matmul_inputs(case, seed)
        if own:
            from paper_2609_34077_gb300 import mcft as M
            s["a"], s["b"] = M.mcft_mx4_quantize(a), M.mcft_mx4_quantize(b)
        else:
            s["a"], s["b"] = _mx4(a), _mx4(b)
    else:
        s["x"], s["idx"], s["gate"], g = _expert_inputs(case, seed)
        d, w = case["d"], case["w"]
        if own:  # the blocks are laid out once, as a program that serves the layer does
            from paper_2609_34077_gb300 import mcft as M
            s["desc"] = M.LayerDesc(d, case["E"], case["K"], w, case["S"], M.MCFT_GATE_RENORM, M.MCFT_BF16)
            blocks = [M.mcft_mx4_pack_expert(s["desc"], b) for b in _expert_weights(case, g)]
            s["experts"], s["shared"] = blocks[: case["E"]], blocks[case["E"]:]
            s["ws"] = torch.empty(M.mcft_mx4_workspace_size(s["desc"], case["T"]), dtype=torch.uint8, device="cuda")
        else:
            up, down = [], []
            for b in _expert_weights(case, g):
                up.append(_mx4(b[: 2 * w * d].view(2 * w, d)))
                down.append(_mx4(b[2 * w * d:].view(d, w)))
            s["up"], s["down"] = ([torch.stack(t) for t in zip(*m)] for m in (up, down))
    return s


# ---- plain forms ----


def _route_scores(case, x, w, bias):
    z = x.float() @ w.float().T
    s = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, 1)
    return s, s if bias is None else s + bias


def _plain_route(case, x, w, bias, dgate):
    E, K, G = case["E"], case["K"], case["groups"]
    s, c = _route_scores(case, x, w, bias)
    if G > 1:
        by = c.view(-1, G, E // G)
        gs = by.sort(2, descending=True).values[..., : case["group_top"]].sum(2)
        kept = gs.sort(dim=1, descending=True, stable=True).indices[:, : case["keep_groups"]]
        keep = torch.zeros_like(gs, dtype=torch.bool).scatter_(1, kept, True)
        c = by.masked_fill(~keep[..., None], -math.inf).flatten(1)
    top = c.sort(dim=1, descending=True, stable=True)
    at = top.indices[:, :K]
    valid = top.values[:, :K] > -math.inf
    sa = torch.where(valid, s.gather(1, at), 0.0)
    total = sa.sum(1, keepdim=True) if case["renorm"] else torch.ones_like(sa[:, :1])
    gate = torch.where(total > 0, sa / total, 0.0) * case["scale"]
    idx = torch.where(valid, at, -1).int()
    load = torch.bincount(at[valid], minlength=E).int()
    if not case["train"]:
        return {"idx": idx, "gate": gate, "load": load}
    dg = torch.where(valid, dgate, 0.0)
    if case["renorm"]:
        dg = torch.where(total > 0, (dg - (gate * dg).sum(1, keepdim=True) / case["scale"]) / total, 0.0)
    ds = torch.zeros_like(s).scatter_(1, at, torch.where(valid, dg * case["scale"], 0.0))
    if case["score"] == "sigmoid":
        dz = ds * s * (1 - s)
    else:
        dz = s * (ds - (s * ds).sum(1, keepdim=True))
    return {"idx": idx, "gate": gate, "load": load, "dx": (dz @ w.float()).to(x.dtype), "dw": dz.T @ x.float()}


def _plain_experts(s):
    c, x, idx, gate = s["case"], s["x"], s["idx"], s["gate"]
    T, d, w, E, K, S = (c[k] for k in ("T", "d", "w", "E", "K", "S"))
    w13, w2 = _values(*s["up"], d), _values(*s["down"], w)  # [E + S, 2 w, d], [E + S, d, w]
    xq = _values(*_mx4(x), d)

    def ffn(xe, m13, m2):  # [n, rows, d] -> [n, rows, d]
        gu = xe @ m13.mT
        h = gu[..., :w] * torch.sigmoid(gu[..., :w]) * gu[..., w:]
        hq = _values(*_mx4(h.flatten(0, 1)), w).view_as(h)
        return hq @ m2.mT

    flat = idx.flatten().long()
    flat = torch.where(flat < 0, E, flat)  # entries without an expert go last
    order = flat.argsort(stable=True)
    counts = torch.bincount(flat, minlength=E + 1)
    place = torch.arange(T * K, device=x.device) - (counts.cumsum(0) - counts)[flat[order]]
    cap = max(1, int(counts[:E].max()))
    live = flat[order] < E
    e, p, a = flat[order][live], place[live], order[live]
    rows = torch.zeros(E, cap, d, device=x.device)
    rows[e, p] = xq[a // K]
    o = torch.zeros(T * K, d, device=x.device)
    o[a] = ffn(rows, w13[:E], w2[:E])[e, p]
    y = (o.view(T, K, d) * gate[..., None]).sum(1)
    if S:
        y = y + ffn(xq.expand(S, T, d), w13[E:], w2[E:]).sum(0)
    return y.to(x.dtype)


def run(s):
    c = s["case"]
    if own:
        return _own(s, c)
    if c["op"] == "route":
        return _plain_route(c, s["x"], s["w"], s["bias"], s["dgate"])
    if c["op"] == "quant":
        return _values(*_mx4(s["x"]), c["C"]).to(s["x"].dtype)
    if c["op"] == "matmul":
        y = _values(*s["a"], c["K"]) @ _values(*s["b"], c["K"]).T
        return y.to(F32 if c["out"] == "f32" else BF16)
    return _plain_experts(s)


# ---- the library's calls ----


def _own(s, c):
    from paper_2609_34077_gb300 import mcft as M
    if c["op"] == "route":
        desc = M.ScoredDesc(c["d"], c["E"], c["K"], c["groups"], c["keep_groups"], c["group_top"],
                            M.MCFT_SCORE_SIGMOID if c["score"] == "sigmoid" else M.MCFT_SCORE_SOFTMAX,
                            M.MCFT_GATE_RENORM if c["renorm"] else M.MCFT_GATE_PLAIN,
                            M.MCFT_F32 if c["dtype"] == "f32" else M.MCFT_BF16, c["scale"])
        x, w = s["x"], s["w"]
        logits = torch.empty(c["T"], c["E"], device=x.device) if c["train"] else None
        load = torch.empty(c["E"], dtype=torch.int32, device=x.device)
        idx, gate = M.mcft_route_scored(desc, x, w, s["bias"], logits=logits, load=load)
        out = {"idx": idx, "gate": gate, "load": load}
        if c["train"]:
            out["dx"], out["dw"] = M.mcft_route_scored_grad(desc, x, w, idx, gate, logits, s["dgate"])
        return out
    if c["op"] == "quant":
        return M.mcft_mx4_dequantize(M.mcft_mx4_quantize(s["x"]), c["R"], c["C"], s["x"].dtype)
    if c["op"] == "matmul":
        return M.mcft_mx4_matmul(s["a"], s["b"], c["M"], c["N"], c["K"], F32 if c["out"] == "f32" else BF16)
    return M.mcft_moe_forward_mx4(s["desc"], s["x"], s["idx"], s["gate"], s["experts"], s["shared"], workspace=s["ws"])


# ---- the definitions in 64 bits ----


def _fake64(x):
    """x [R, C] in 64 bits, each 32 along a row rounded to the e2m1 grid under their power-of-two scale."""
    R, C = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -C % 32)).reshape(R, -1, 32)
    big = v.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(big > 0, big, 1.0))).long()
    power = lambda n: ((n + 1023) << 52).view(torch.float64)  # noqa: E731 (exact, where exp2 need not be)
    e = torch.where(power(e) > big, e - 1, torch.where(power(e + 1) <= big, e + 1, e))  # where log2 rounded
    unit = power(torch.clamp(torch.where(big > 0, e, -127) - 2, -127, 127))
    a = v.abs() / unit
    n = sum((a > m).long() for m in MID_DOWN) + sum((a >= m).long() for m in MID_UP)
    q = torch.tensor(GRID, dtype=torch.float64, device=x.device)[n]
    return (torch.sign(v) * q * unit).reshape(R, -1)[:, :C]


def _exact_route(case, seed):
    x, w, bias, dgate = _route_inputs(case, seed)
    z, s, c, _ = _scores64(case, x, w, bias)
    T, E, K = case["T"], case["E"], case["K"]
    order = torch.argsort(c, dim=1, descending=True, stable=True)[:, :K]
    on = torch.gather(c, 1, order) > -math.inf
    member = torch.zeros(T, E, dtype=torch.float64, device=x.device).scatter_(1, order, on.double())
    p = s * member
    full = p / p.sum(1, keepdim=True).clamp_min(1e-300) if case["renorm"] else p
    gate = torch.gather(full, 1, order) * case["scale"]
    out = {"idx": torch.where(on, order, -1).int(), "gate": gate, "load": member.sum(0).int()}
    if case["train"]:
        up = torch.zeros(T, E, dtype=torch.float64, device=x.device).scatter_(1, order, dgate.double()) * member * case["scale"]
        slope = (1 - s) if case["score"] == "sigmoid" else None
        if case["renorm"]:  # through log p: d log p_e / dz is (1 - s_e) for the sigmoid, and 1 - shift for softmax
            dlog = full * (up - (up * full).sum(1, keepdim=True))
            dz = dlog * slope if slope is not None else dlog
        else:
            dlog = up * s
            dz = dlog * slope if slope is not None else dlog - s * dlog.sum(1, keepdim=True)
        out["dx"], out["dw"] = dz @ w.double(), dz.T @ x.double()
    return out


def exact(case, seed):
    if case["op"] == "route":
        return _exact_route(case, seed)
    if case["op"] == "quant":
        return _fake64(_quant_input(case, seed))
    if case["op"] == "matmul":
        a, b = _matmul_inputs(case, seed)
        return _fake64(a) @ _fake64(b).T
    x, idx, gate, g = _expert_inputs(case, seed)
    d, w, E = case["d"], case["w"], case["E"]
    xq = _fake64(x)
    y = torch.zeros(case["T"], d, dtype=torch.float64, device=x.device)
    for e, b in enumerate(_expert_weights(case, g)):
        w13, w2 = _fake64(b[: 2 * w * d].view(2 * w, d)), _fake64(b[2 * w * d:].view(d, w))
        if e < E:
            t, k = torch.nonzero(idx == e, as_tuple=True)
            share = gate[t, k].double()[:, None]
        else:
            t, share = torch.arange(case["T"], device=x.device), 1.0
        if not len(t):
            continue
        u = xq[t] @ w13.T
        h = u[:, :w] / (1 + torch.exp(-u[:, :w])) * u[:, w:]
        y.index_add_(0, t, share * (_fake64(h) @ w2.T))
    return y
