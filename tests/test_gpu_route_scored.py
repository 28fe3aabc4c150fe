"""Scored routing and its gradient against the fp64 oracle.

Choices are compared on tokens whose decisions lie more than 1e-4 of the scores' size apart (an fp32 logit of a few
thousand terms is good to about 1e-5); all others are left out before the call. Gates: |g - g_ref| <= 1e-5 of the
token's largest gate, plus 1e-5 |g_ref|: twice what 1e-5 in a logit moves a score by.
Gradients: dz has a relative error of a few 1e-6 from the gates and scores, its largest part 1e-5; a sum of n
products by fp32 adds less: 2e-5 of the sum of the terms' magnitudes, and 2^-8 of the value where it rounds to
bf16."""
import numpy as np
import pytest
import torch

import oracle.scored as O
from paper_2609_34077_gb300 import mcft as M

pytestmark = pytest.mark.gpu


def desc_of(d, E, K, dtype, score="softmax", n_group=1, topk_group=1, group_top=1, renorm=True, scale=1.0):
    return M.ScoredDesc(d, E, K, n_group, topk_group, group_top,
                        M.MCFT_SCORE_SIGMOID if score == "sigmoid" else M.MCFT_SCORE_SOFTMAX,
                        M.MCFT_GATE_RENORM if renorm else M.MCFT_GATE_PLAIN,
                        M.MCFT_BF16 if dtype == torch.bfloat16 else M.MCFT_F32, scale)


def case(seed, T, d, E, K, dtype, bias=None, **kw):
    """x [T, d] of clear decisions, w, the oracle's routing of them."""
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(E, d, generator=g) * 1.28 / d ** 0.5).to(dtype)
    x = torch.randn(2 * T + 64, d, generator=g).to(dtype)
    b = None if bias is None else bias.numpy()
    clear = O.route(x.double().numpy(), w.double().numpy(), K, bias=b, **kw)["clear"]
    x = x[torch.from_numpy(clear)][:T].contiguous()
    assert len(x) == T
    return x, w, O.route(x.double().numpy(), w.double().numpy(), K, bias=b, **kw)


def run(desc, x, w, bias=None):
    T = x.shape[0]
    logits = torch.full((T, desc.E), 7.0, device="cuda")
    load = torch.full((desc.E,), -5, dtype=torch.int32, device="cuda")
    idx, gate = M.mcft_route_scored(desc, x.cuda(), w.cuda(), None if bias is None else bias.cuda(), logits=logits, load=load)
    M.mcft_device_error()
    return idx, gate, logits, load


def check(idx, gate, logits, load, ref):
    np.testing.assert_array_equal(idx.cpu().numpy(), ref["idx"])
    g = ref["gate"]
    assert (np.abs(gate.cpu().double().numpy() - g) <= 1e-5 * (np.abs(g) + g.max(1, keepdims=True))).all()
    np.testing.assert_allclose(logits.cpu().double().numpy(), ref["z"], atol=2e-5 * max(1.0, np.abs(ref["z"]).max()))
    np.testing.assert_array_equal(load.cpu().numpy(), ref["load"])


RULES = [
    dict(E=64, K=6, renorm=False),
    dict(E=8, K=2),
    dict(E=256, K=8, score="sigmoid", n_group=8, topk_group=4, group_top=2, scale=2.5),
    dict(E=160, K=6, n_group=8, topk_group=3, group_top=1, renorm=False, scale=16.0),
    dict(E=96, K=16, score="sigmoid", n_group=32, topk_group=9, group_top=2),
    dict(E=1, K=1, score="sigmoid"),
    dict(E=33, K=5, score="sigmoid", n_group=3, topk_group=2, renorm=False),
]


def with_bias(rule, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(rule["E"], generator=g) * (0.05 if rule.get("score") == "sigmoid" else 0.2 / rule["E"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 3, 5, 64, 65, 130, 1000])
@pytest.mark.parametrize("rule", range(len(RULES)))
def test_routing(rule, T, dtype):
    r = RULES[rule]
    bias = with_bias(r, T) if rule % 2 == 0 else None
    d = 64 * (1 + (rule + T) % 5) if T > 100 else 64 * (1 + (rule * 7 + T) % 40)
    kw = {k: v for k, v in r.items() if k not in ("E", "K")}
    x, w, ref = case(T, T, d, r["E"], r["K"], dtype, bias, **kw)
    check(*run(desc_of(d, r["E"], r["K"], dtype, **kw), x, w, bias), ref)


@pytest.mark.parametrize("T", [4, 100, 600])
@pytest.mark.parametrize("keep", [0, 1, 3, 9])
def test_masked_experts(T, keep):
    """A bias of -infinity: fewer eligible experts than K leave the last places empty, none leave the row empty."""
    bias = torch.full((64,), -float("inf"))
    bias[torch.randperm(64, generator=torch.Generator().manual_seed(keep))[:keep]] = 0.0
    for kw in (dict(renorm=False), dict(score="sigmoid", n_group=8, topk_group=3, group_top=2)):
        x, w, ref = case(T, T, 256, 64, 6, torch.bfloat16, bias, **kw)
        idx, gate, logits, load = run(desc_of(256, 64, 6, torch.bfloat16, **kw), x, w, bias)
        check(idx, gate, logits, load, ref)
        if keep == 0:
            assert (idx == -1).all() and (gate == 0).all() and (load == 0).all()


@pytest.mark.parametrize("T", [2, 70, 300])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_go_to_the_lower_index(T, dtype):
    g = torch.Generator().manual_seed(0)
    w = torch.randn(1, 128, generator=g).repeat(48, 1).to(dtype)
    x = torch.randn(T, 128, generator=g).to(dtype)
    idx, _, _, load = run(desc_of(128, 48, 4, dtype), x, w)
    assert (idx.cpu() == torch.arange(4)).all() and load.tolist() == [T] * 4 + [0] * 44
    idx, *_ = run(desc_of(128, 48, 4, dtype, score="sigmoid", n_group=6, topk_group=2, group_top=2), x, w)
    assert (idx.cpu() == torch.arange(4)).all()
    bias = torch.zeros(48)
    bias[40:] = 0.5
    idx, *_ = run(desc_of(128, 48, 4, dtype, score="sigmoid", n_group=6, topk_group=2, group_top=1), x, w, bias)
    assert (idx.cpu() == torch.arange(40, 44)).all()


@pytest.mark.parametrize("T", [3, 80, 400])
def test_extreme_and_nan_logits(T):
    w = torch.zeros(16, 64)
    w[:, 0] = torch.arange(16) * 30.0 - 200
    x = torch.zeros(T, 64)
    x[:, 0] = 1.0
    for score in ("sigmoid", "softmax"):
        kw = dict(score=score, renorm=False)
        ref = O.route(x.numpy(), w.numpy(), 3, **kw)
        idx, gate, *_ = run(desc_of(64, 16, 3, torch.float32, **kw), x, w)
        if score == "softmax":  # (sigmoids of 100 and more are all 1: ties in fp32)
            np.testing.assert_array_equal(idx.cpu().numpy(), ref["idx"])
        assert torch.isfinite(gate).all() and (gate <= 1).all()
    x[1, 0] = float("nan")
    idx, gate = M.mcft_route_scored(desc_of(64, 16, 3, torch.float32, score="sigmoid"), x.cuda(), w.cuda())
    with pytest.raises(M.MCFTError):
        M.mcft_device_error()
    assert (idx[1] == -1).all() and (gate[1] == 0).all() and (idx[0] >= 0).all()


def check_gradient(dx, dw, x, w, ref, dg, dtype, score, renorm, scale, base=None):
    xd, wd = x.double().numpy(), w.double().numpy()
    rx, rw = O.gradient(xd, wd, ref["idx"], dg, score, renorm, scale)
    # the terms' magnitudes, with dz's own parts taken apart
    s, on = ref["s"], ref["idx"] >= 0
    size = np.zeros_like(s)
    spread = np.abs(dg) + (np.abs(dg * on).max(1, keepdims=True) if renorm else 0.0)
    np.put_along_axis(size, np.maximum(ref["idx"], 0).astype(np.int64), np.where(on, ref["gate"] * spread, 0.0), 1)
    if score == "softmax" and not renorm:
        size = size + s * size.sum(1, keepdims=True)
    tx, tw = 2e-5 * size @ np.abs(wd), 2e-5 * size.T @ np.abs(xd)
    if dtype == torch.bfloat16:
        tx = tx + 2.0 ** -8 * np.abs(rx)
    if base is not None:
        rw = rw + base
        tw = tw + 1e-6 * np.abs(rw)
    for got, want, tol, name in ((dx, rx, tx, "dx"), (dw, rw, tw, "dw")):
        err = np.abs(got.cpu().double().numpy() - want)
        assert (err <= tol + 1e-30).all(), f"{name}: worst {np.max(err / (tol + 1e-30)):.3g} of the bound"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 5, 66, 129, 1000])
@pytest.mark.parametrize("rule", [0, 1, 2, 4, 5, 6])
def test_gradient(rule, T, dtype):
    r = RULES[rule]
    d = 64 * (1 + (rule + T) % 5)
    kw = {k: v for k, v in r.items() if k not in ("E", "K")}
    x, w, ref = case(T + 1, T, d, r["E"], r["K"], dtype, None, **kw)
    D = desc_of(d, r["E"], r["K"], dtype, **kw)
    idx, gate, logits, _ = run(D, x, w)
    dg = torch.randn(T, r["K"], generator=torch.Generator().manual_seed(9))
    args = D, x.cuda(), w.cuda(), idx, gate, logits, dg.cuda()
    dx, dw = M.mcft_route_scored_grad(*args)
    M.mcft_device_error()
    rest = (x, w, ref, dg.double().numpy(), dtype, r.get("score", "softmax"), r.get("renorm", True), r.get("scale", 1.0))
    check_gradient(dx, dw, *rest)
    again = M.mcft_route_scored_grad(*args)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    base = torch.randn(r["E"], d, generator=torch.Generator().manual_seed(8))
    acc = base.cuda()
    M.mcft_route_scored_grad(*args, dw=acc, accumulate=True)
    check_gradient(dx, acc, *rest, base=base.double().numpy())


@pytest.mark.parametrize("T", [6, 200])
def test_gradient_of_tokens_without_an_expert(T):
    bias = torch.full((32,), -float("inf"))
    bias[[3, 7]] = 0.0
    for kw in (dict(renorm=False), dict(score="sigmoid", scale=1.5), dict()):
        x, w, ref = case(T, T, 128, 32, 4, torch.bfloat16, bias, **kw)
        D = desc_of(128, 32, 4, torch.bfloat16, **kw)
        idx, gate, logits, _ = run(D, x, w, bias)
        dg = torch.randn(T, 4, generator=torch.Generator().manual_seed(9))
        rest = (x, w, ref, dg.double().numpy(), torch.bfloat16, kw.get("score", "softmax"), kw.get("renorm", True), kw.get("scale", 1.0))
        gate[:, 2:], dg[:, 2:] = float("nan"), float("nan")  # not read
        dx, dw = M.mcft_route_scored_grad(D, x.cuda(), w.cuda(), idx, gate, logits, dg.cuda())
        ref["gate"][:, 2:] = 0
        rest[3][:, 2:] = 0
        check_gradient(dx, dw, *rest)
        idx[:] = -1
        dx, dw = M.mcft_route_scored_grad(D, x.cuda(), w.cuda(), idx, gate, logits, dg.cuda())
        assert (dx == 0).all() and (dw == 0).all()


def test_one_gradient_alone_and_no_tokens():
    x, w, ref = case(1, 90, 128, 16, 2, torch.bfloat16)
    D = desc_of(128, 16, 2, torch.bfloat16)
    idx, gate, logits, _ = run(D, x, w)
    dg = torch.randn(90, 2).cuda()
    dx, dw = M.mcft_route_scored_grad(D, x.cuda(), w.cuda(), idx, gate, logits, dg)
    ws = torch.empty(M.mcft_route_scored_grad_workspace_size(D, 90), dtype=torch.uint8, device="cuda")
    L, p = M.lib(), M._ptr
    for keep_x in (True, False):
        ox, ow = torch.zeros_like(dx), torch.zeros_like(dw)
        M._check(L.mcft_route_scored_grad(M.C.byref(D), p(x.cuda()), 90, p(w.cuda()), p(idx), p(gate), p(logits), p(dg),
                                          p(ox) if keep_x else None, None if keep_x else p(ow), 0, p(ws), ws.numel(),
                                          M._stream(None)))
        assert torch.equal(ox, dx) if keep_x else torch.equal(ow, dw)
    none = M.mcft_route_scored_grad(D, x[:0].cuda(), w.cuda(), idx[:0], gate[:0], logits[:0], dg[:0])
    assert none[0].shape == (0, 128) and (none[1] == 0).all()
    assert M.mcft_route_scored(D, x[:0].cuda(), w.cuda())[0].shape == (0, 2)


def test_refusals():
    x, w = torch.zeros(4, 128, device="cuda"), torch.zeros(300, 128, device="cuda")
    good = dict(d=128, E=64, K=4, n_group=8, topk_group=2, group_top=1, score=0, gate=0, dtype=0, scale=1.0)
    bad = [(dict(d=100), 1), (dict(E=0), 1), (dict(E=264), 5), (dict(K=65), 1), (dict(K=17), 5), (dict(n_group=7), 1),
           (dict(n_group=64), 5), (dict(topk_group=9), 1), (dict(group_top=9), 1), (dict(group_top=3), 5), (dict(score=2), 1),
           (dict(gate=2), 1), (dict(dtype=2), 1), (dict(scale=0.0), 1), (dict(scale=float("inf")), 1),
           (dict(scale=float("nan")), 1)]
    for change, status in bad:
        D = M.ScoredDesc(**{**good, **change})
        for call in (lambda: M.mcft_route_scored(D, x, w), lambda: M.mcft_route_scored_grad_workspace_size(D, 4)):
            with pytest.raises(M.MCFTError) as e:
                call()
            assert e.value.status == status, change
    D = M.ScoredDesc(**good)
    idx, gate = M.mcft_route_scored(D, x, w)
    z = torch.zeros(4, 64, device="cuda")
    with pytest.raises(M.MCFTError):
        M.mcft_route_scored_grad(D, x, w, idx, gate, z, gate, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(M.MCFTError):
        M.mcft_route_scored(D, x.flatten()[1:].narrow(0, 0, 384).view(3, 128), w)
    idx[0, 0] = 64
    M.mcft_route_scored_grad(D, x, w, idx, gate, z, gate)
    with pytest.raises(M.MCFTError):
        M.mcft_device_error()
