"""The gradient of causal attention over packed prompts on the GPU against the formula in 64 bits, and against differences.
Needs an MI355X: ``-m gpu``.

Tolerances, element by element.  P and dS are rounded to bf16 (2^-8 each), `out` (which delta is made of) and the results too; scores and dP are
fp32 sums of 128 exact products.  With e = 2^-8, moved = 2^-17 of the largest scale * sum |q k| (the change of a weight, relatively) and |.|
taken inside the sums:
  dV = sum P dout                      off by (e + moved) sum P |dout| + e |dV|
  dS = P (dP - delta)                  off by (e + moved) |dS| + P (2^-17 sum |dout v| + e sum |dout out|)
  dQ, dK = scale sum dS (k, q)         off by scale sum (off dS) |k, q| + e |dQ, dK|
Probabilities below 2^-126, the smallest normal number of 32 bits and of bf16, count as zero: with at most 2^13 terms of at most 2^13
each here, off by 2^-100 at the most."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_prompt import D, DEV, definition, make, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    ws = torch.empty(512 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(ws)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)


@pytest.fixture(params=[None, "4x100000", "8x1", "4x3"])
def shape_of_launch(request, monkeypatch):
    if request.param:
        monkeypatch.setenv("COMMFUSE_CAUSAL", request.param)


def gradient(q, k, v, dout, at, scale):
    """({dq, dk, dv} in 64 bits, {their limits}); rows of no sequence NaN"""
    T, h = q.shape[:2]
    g, e = h // k.shape[1], 2.0 ** -8
    q, k, v, dout = (x.double() for x in (q, k, v, dout))
    res = {n: torch.full_like(x, math.nan) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    off = {n: torch.full_like(x, math.nan) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    for a, b in zip(at[:-1].tolist(), at[1:].tolist()):
        for n in ("dk", "dv"):
            res[n][a:b] = off[n][a:b] = 0
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device=DEV).triu(1)
        for i in range(h):
            qq, kk, vv, gg = q[a:b, i], k[a:b, i // g], v[a:b, i // g], dout[a:b, i]
            p = torch.softmax((qq @ kk.t() * scale).masked_fill(hidden, -math.inf), 1)
            out = p @ vv
            ds = p * (gg @ vv.t() - (gg * out).sum(1)[:, None])
            moved = 2.0 ** -17 * (qq.abs() @ kk.abs().t() * scale).masked_fill(hidden, 0).amax(1)[:, None] if b > a else 0
            ods = (e + moved) * ds.abs() + p * (2.0 ** -17 * (gg.abs() @ vv.abs().t()) + e * (gg * out).abs().sum(1)[:, None])
            res["dq"][a:b, i] = scale * ds @ kk
            off["dq"][a:b, i] = scale * ods @ kk.abs() + e * res["dq"][a:b, i].abs()
            res["dk"][a:b, i // g] += scale * ds.t() @ qq
            res["dv"][a:b, i // g] += p.t() @ gg
            off["dk"][a:b, i // g] += scale * ods.t() @ qq.abs()
            off["dv"][a:b, i // g] += ((e + moved) * p).t() @ gg.abs()
    for n in ("dk", "dv"):
        off[n] += e * res[n].abs()
    return res, off


def forward_and_gradient(x, dout, h, kv, at, scale):
    T, s = x.shape[0], x.stride()[:2]
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    out = torch.full((T, h, D), -7.0, dtype=torch.bfloat16, device=DEV)
    lse, delta = torch.full((h, T), -7.0, device=DEV), torch.full((h, T), -7.0, device=DEV)
    desc = cf.prompt_desc(T, at.numel() - 1, h, kv, scale, q=s, k=s, v=s)
    cf.attn_prompt(desc, q, k, v, at, out, lse)
    dx = torch.full_like(x, -7.0)
    got = dict(dq=dx[:, :h], dk=dx[:, h:h + kv], dv=dx[:, h + kv:])
    cf.attn_prompt_grad(desc, q, k, v, out, lse, dout, at, delta, got["dq"], got["dk"], got["dv"])
    torch.cuda.synchronize()
    return got


def check(got, ref):
    res, off = ref
    for n in ("dq", "dk", "dv"):
        some = ~torch.isnan(res[n])
        bad = ~((got[n].double() - res[n]).abs() <= off[n] + 2.0 ** -100) & some
        assert not bool(bad.any()), (n, int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got[n].double() - res[n]).abs() / off[n])[some].max()))
        assert bool((got[n][~some] == -7).all()), n


def problem(seed, lens, h, kv, before=0, behind=0, sigma=1.0):
    T = before + sum(lens) + behind
    x = make(seed, T, h, kv, sigma)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    return x, torch.randn(T, h, D, generator=g, device=DEV).to(torch.bfloat16), starts(lens, before)


CASES = [  # heads, key heads, lengths
    (1, 1, [2]), (8, 1, [3, 1, 5]), (4, 4, [64]), (4, 2, [65, 1]), (8, 1, [127, 129, 3]), (2, 2, [300]), (5, 1, [17, 0, 33, 0, 0, 260]),
    (6, 2, [1] * 70 + [200] + [2] * 40), (16, 2, [311, 213]), (1, 1, [1025, 7]), (3, 3, [340, 64, 128, 5]), (32, 1, [40, 100]), (12, 4, [400]),
    (8, 8, [0, 5, 0]), (100, 1, [70])]


@pytest.mark.parametrize("case", CASES)
def test_gradient(case, shape_of_launch):
    h, kv, lens = case
    x, dout, at = problem(len(lens) * 100 + lens[0], lens, h, kv)
    ref = gradient(x[:, :h], x[:, h:h + kv], x[:, h + kv:], dout, at, 1 / math.sqrt(D))
    got = forward_and_gradient(x, dout, h, kv, at, 1 / math.sqrt(D))
    check(got, ref)
    again = forward_and_gradient(x, dout, h, kv, at, 1 / math.sqrt(D))
    assert all(torch.equal(got[n], again[n]) for n in got)


def test_sequences_of_one_token():
    """P = 1: dV is dout; dP and delta are the same sum, so dQ and dK are nothing but its rounding: 2^-17 of sum |dout v| times |k|."""
    x, dout, at = problem(3, [1] * 150, 4, 2)
    got = forward_and_gradient(x, dout, 4, 2, at, 0.3)
    check(got, gradient(x[:, :4], x[:, 4:6], x[:, 6:], dout, at, 0.3))


def test_rows_of_no_sequence_are_left_as_they_were(shape_of_launch):
    h, kv, lens = 4, 2, [70, 0, 130]
    x, dout, at = problem(3, lens, h, kv, 37, 96)
    for t in (x, dout):
        t[:37], t[237:] = math.nan, math.inf
    check(forward_and_gradient(x, dout, h, kv, at, 0.1), gradient(x[:, :h], x[:, h:h + kv], x[:, h + kv:], dout, at, 0.1))


def test_peaked_scores(shape_of_launch):
    x, dout, at = problem(5, [190, 200], 2, 1, sigma=4.0)
    check(forward_and_gradient(x, dout, 2, 1, at, 0.3), gradient(x[:, :2], x[:, 2:3], x[:, 3:], dout, at, 0.3))


@pytest.mark.parametrize("what", ["kv", "q", "dout"])
def test_what_the_mask_hides_has_no_influence(what, shape_of_launch):
    """One token of the middle sequence is not finite: the other sequences' gradients are as without; of its own, dQ of the rows that do not
    see its K and V, and dK, dV of the keys that its row does not see."""
    h, kv, lens, t = 4, 2, [150, 81, 160], 180
    x, dout, at = problem(21, lens, h, kv)
    ref = gradient(x[:, :h], x[:, h:h + kv], x[:, h + kv:], dout, at, 0.09)
    if what == "kv":
        x[t, h:] = math.nan
    elif what == "q":
        x[t, :h] = math.inf
    else:
        dout[t] = -math.inf
    got = forward_and_gradient(x, dout, h, kv, at, 0.09)
    touched = dict(kv=dict(dq=slice(t, 231), dk=slice(150, 231), dv=slice(150, 231)), q=dict(dq=slice(t, t + 1), dk=slice(150, t + 1), dv=slice(150, t + 1)))
    for n, r in touched.get(what, touched["q"]).items():
        assert not bool(torch.isfinite(got[n][r].float()).all())
        for part in ref:
            part[n][r] = math.nan
        got[n][r] = -7
    check(got, ref)


def test_gradient_against_differences():
    """Along a direction, the loss sum(out * dout) in 64 bits changes as the gradient says.  A central difference over 2 eps along a unit-size
    direction is off by eps^2 times a third derivative of the loss (taken as 10 |loss change|); the gradient's elements are off by their limits."""
    h, kv, lens, scale = 4, 2, [60, 90], 0.09
    x, dout, at = problem(31, lens, h, kv)
    got = forward_and_gradient(x, dout, h, kv, at, scale)
    _, off = gradient(x[:, :h], x[:, h:h + kv], x[:, h + kv:], dout, at, scale)
    eps = 1e-4
    for n, r in (("dq", slice(0, h)), ("dk", slice(h, h + kv)), ("dv", slice(h + kv, h + 2 * kv))):
        step = torch.randn(x[:, r].shape, dtype=torch.float64, device=DEV)
        loss = []
        for sign in (1, -1):
            y = x.double().clone()
            y[:, r] += sign * eps * step
            loss.append(float((definition(y[:, :h], y[:, h:h + kv], y[:, h + kv:], at, scale)[0] * dout.double()).sum()))
        change = (loss[0] - loss[1]) / (2 * eps)
        # independent errors, each within its limit: ten times their root mean square is out of reach
        slack = 10 * float((off[n] * step).square().sum().sqrt()) + 1e-5 * abs(change) + 1e-6
        assert abs(change - float((got[n].double() * step).sum())) <= slack


def test_heads_outermost_and_offsets_beyond_32_bits():
    T, stride = 4200, 1 << 19
    x, dout, at = problem(41, [4000, 200], 1, 1)
    big = [torch.zeros((T - 1) * stride + 3 * D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    view, dview = (b.as_strided((T, 3, D), (stride, D, 1)) for b in big)
    view.copy_(x)
    want = forward_and_gradient(x, dout, 1, 1, at, 0.09)
    out, lse, delta = torch.empty(T, 1, D, dtype=torch.bfloat16, device=DEV), torch.empty(1, T, device=DEV), torch.empty(1, T, device=DEV)
    s = view.stride()[:2]
    desc = cf.prompt_desc(T, 2, 1, 1, 0.09, q=s, k=s, v=s)
    q, k, v = view[:, :1], view[:, 1:2], view[:, 2:]
    cf.attn_prompt(desc, q, k, v, at, out, lse)
    cf.attn_prompt_grad(desc, q, k, v, out, lse, dout, at, delta, dview[:, :1], dview[:, 1:2], dview[:, 2:])
    torch.cuda.synchronize()
    for n, r in (("dq", 0), ("dk", 1), ("dv", 2)):
        assert torch.equal(dview[:, r:r + 1], want[n])
    del big, view, dview
    h, kv, lens = 4, 2, [100, 57]
    T = sum(lens)
    x, dout, at = problem(42, lens, h, kv)
    want = forward_and_gradient(x, dout, h, kv, at, 0.09)
    q, k, v, g = (t.transpose(0, 1).contiguous() for t in (x[:, :h], x[:, h:h + kv], x[:, h + kv:], dout))
    out, lse, delta = torch.empty_like(q), torch.empty(h, T, device=DEV), torch.empty(h, T, device=DEV)
    res = [torch.empty_like(t) for t in (q, k, v)]
    o = (D, T * D)
    desc = cf.prompt_desc(T, 2, h, kv, 0.09, q=o, k=o, v=o, o=o)
    cf.attn_prompt(desc, q, k, v, at, out, lse)
    cf.attn_prompt_grad(desc, q, k, v, out, lse, g, at, delta, *res)
    torch.cuda.synchronize()
    assert all(torch.equal(r.transpose(0, 1), want[n]) for r, n in zip(res, ("dq", "dk", "dv")))


def test_graph_replays_with_other_sequences():
    h, kv, T = 4, 2, 600
    x, dout, at = problem(51, [600, 0, 0], h, kv)
    q, k, v, s = x[:, :h], x[:, h:h + kv], x[:, h + kv:], x.stride()[:2]
    out, lse, delta, dx = torch.zeros_like(dout), torch.zeros(h, T, device=DEV), torch.zeros(h, T, device=DEV), torch.zeros_like(x)
    desc = cf.prompt_desc(T, 3, h, kv, 0.09, q=s, k=s, v=s)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cf.attn_prompt(desc, q, k, v, at, out, lse, side)
        cf.attn_prompt_grad(desc, q, k, v, out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:], side)
    for i, lens in enumerate(([600, 0, 0], [1, 599, 0], [200, 200, 200], [0, 0, 600])):
        at.copy_(starts(lens))
        x.copy_(make(60 + i, T, h, kv))
        graph.replay()
        torch.cuda.synchronize()
        eager = forward_and_gradient(x, dout, h, kv, at, 0.09)
        assert torch.equal(dx, torch.cat([eager["dq"], eager["dk"], eager["dv"]], 1))
