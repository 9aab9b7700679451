"""Attention with a sliding window and first tokens that stay visible, over packed prompts, and its gradient, on the GPU against the definition in 64
bits.  The tolerances are those of causal attention (the tests of which say why): they are sums over what is visible, and the mask
changes only what that is.  Needs an MI355X: ``-m gpu``."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_grad import check as check_grad
from tests.test_gpu_attn_prompt import D, DEV, check, make, starts

pytestmark = pytest.mark.gpu
WORKSPACE = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    global WORKSPACE
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    WORKSPACE = torch.empty(512 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(WORKSPACE)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)
    WORKSPACE = None


@pytest.fixture(params=[None, "4x100000", "8x1", "4x3"])
def shape_of_launch(request, monkeypatch):
    """Waves of a workgroup, and key tiles of a split."""
    if request.param:
        monkeypatch.setenv("COMMFUSE_CAUSAL", request.param)


def _hidden(n, window, sinks):
    i, j = torch.arange(n, device=DEV)[:, None], torch.arange(n, device=DEV)[None, :]
    return (j > i) | ((j <= i - window) & (j >= sinks))


def definition(x, h, kv, at, scale, window, sinks, dout=None):
    """(out, lse, weighted mean of |v|, largest scale * sum |q k| of a visible key), and with dout ({dq, dk, dv}, {their limits}), in 64 bits; rows of
    no sequence are NaN."""
    T, g, e = x.shape[0], h // kv, 2.0 ** -8
    q, k, v = (t.double() for t in (x[:, :h], x[:, h:h + kv], x[:, h + kv:]))
    out, lse, mean, size = (torch.full(s, math.nan, dtype=torch.float64, device=DEV) for s in ((T, h, D), (h, T), (T, h, D), (h, T)))
    res, off = ({n: torch.full_like(t, math.nan) for n, t in (("dq", q), ("dk", k), ("dv", v))} for _ in range(2))
    for a, b in zip(at[:-1].tolist(), at[1:].tolist()):
        hidden = _hidden(b - a, window, sinks)
        for n in ("dk", "dv"):
            res[n][a:b] = off[n][a:b] = 0
        for i in range(h):
            qq, kk, vv = q[a:b, i], k[a:b, i // g], v[a:b, i // g]
            s = (qq @ kk.t() * scale).masked_fill(hidden, -math.inf)
            p = torch.softmax(s, 1)
            lse[i, a:b], out[a:b, i], mean[a:b, i] = torch.logsumexp(s, 1), p @ vv, p @ vv.abs()
            size[i, a:b] = (qq.abs() @ kk.abs().t() * scale).masked_fill(hidden, 0).amax(1) if b > a else 0
            if dout is not None:
                gg, o = dout[a:b, i].double(), p @ vv
                ds = p * (gg @ vv.t() - (gg * o).sum(1)[:, None])
                moved = 2.0 ** -17 * size[i, a:b, None]
                ods = (e + moved) * ds.abs() + p * (2.0 ** -17 * (gg.abs() @ vv.abs().t()) + e * (gg * o).abs().sum(1)[:, None])
                res["dq"][a:b, i] = scale * ds @ kk
                off["dq"][a:b, i] = scale * ods @ kk.abs() + e * res["dq"][a:b, i].abs()
                res["dk"][a:b, i // g] += scale * ds.t() @ qq
                res["dv"][a:b, i // g] += p.t() @ gg
                off["dk"][a:b, i // g] += scale * ods.t() @ qq.abs()
                off["dv"][a:b, i // g] += ((e + moved) * p).t() @ gg.abs()
    for n in ("dk", "dv"):
        off[n] += e * res[n].abs()
    return (out, lse, mean, size) if dout is None else ((out, lse, mean, size), (res, off))


def run(x, h, kv, at, scale, window, sinks, dout=None, with_lse=True):
    """(out, lse), and with dout {dq, dk, dv}"""
    T, s = x.shape[0], x.stride()[:2]
    q, k, v, w = x[:, :h], x[:, h:h + kv], x[:, h + kv:], cf.window(window, sinks)
    out = torch.full((T, h, D), -7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((h, T), -7.0, device=DEV) if with_lse else None
    desc = cf.prompt_desc(T, at.numel() - 1, h, kv, scale, q=s, k=s, v=s)
    cf.attn_prompt_window(desc, w, q, k, v, at, out, lse)
    if dout is None:
        torch.cuda.synchronize()
        return out, lse
    dx, delta = torch.full_like(x, -7.0), torch.empty(h, T, device=DEV)
    cf.attn_prompt_window_grad(desc, w, q, k, v, out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:])
    torch.cuda.synchronize()
    return (out, lse), dict(dq=dx[:, :h], dk=dx[:, h:h + kv], dv=dx[:, h + kv:])


def problem(seed, lens, h, kv, before=0, behind=0, sigma=1.0):
    T = before + sum(lens) + behind
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    return make(seed, T, h, kv, sigma), torch.randn(T, h, D, generator=g, device=DEV).to(torch.bfloat16), starts(lens, before)


CASES = [  # heads, key heads, lengths, window, sinks
    (1, 1, [3], 1, 0), (1, 1, [2], 1, 1), (8, 1, [3, 1, 5], 2, 0), (8, 1, [3, 1, 9], 2, 1), (4, 4, [64], 17, 3), (4, 2, [65, 1], 64, 0), (8, 1, [127, 129, 3], 64, 2),
    (2, 2, [300], 63, 65), (5, 1, [17, 0, 33, 0, 0, 260], 40, 4), (6, 2, [1] * 70 + [200] + [2] * 40, 33, 5), (16, 2, [511, 513], 100, 0), (1, 1, [1025, 7], 129, 1),
    (3, 3, [640, 64, 128, 5], 200, 130), (32, 1, [40, 300], 16, 4), (12, 4, [700], 256, 64), (8, 8, [0, 5, 0], 3, 1), (2, 1, [1500], 1, 0), (2, 1, [1500], 64, 64),
    (1, 1, [900], 100, 700), (4, 1, [333, 777, 21], 300, 7), (100, 1, [70], 30, 2)]


@pytest.mark.parametrize("case", CASES)
def test_output_lse_and_gradient(case, shape_of_launch):
    h, kv, lens, window, sinks = case
    x, dout, at = problem(len(lens) * 100 + lens[0], lens, h, kv)
    ref, gref = definition(x, h, kv, at, 1 / math.sqrt(D), window, sinks, dout)
    (out, lse), got = run(x, h, kv, at, 1 / math.sqrt(D), window, sinks, dout)
    check(out, lse, ref)
    check_grad(got, gref)
    check(run(x, h, kv, at, 1 / math.sqrt(D), window, sinks, with_lse=False)[0], None, ref)
    (out2, lse2), again = run(x, h, kv, at, 1 / math.sqrt(D), window, sinks, dout)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("case", [(8, 1, [2000, 90], 500, 4), (4, 4, [1, 3000], 1024, 0), (2, 1, [4097], 700, 16), (1, 1, [6000], 64, 1), (16, 2, [2500], 100, 200),
                                  (4, 4, [1000] * 3, 128, 4)])
def test_longer_prompts_without_overrides(case):
    h, kv, lens, window, sinks = case
    x, dout, at = problem(7, lens, h, kv, sigma=1.5)
    ref, gref = definition(x, h, kv, at, 0.05, window, sinks, dout)
    desc = cf.prompt_desc(sum(lens), len(lens), h, kv, 0.05)
    assert cf.attn_prompt_window_workspace_bytes(desc, cf.window(window, sinks)) <= WORKSPACE.numel()
    for ws in (WORKSPACE, None, WORKSPACE[:3 << 20]):                         # without a workspace nothing is split, with a small one less
        cf.set_workspace(ws)
        try:
            (out, lse), got = run(x, h, kv, at, 0.05, window, sinks, dout)
        finally:
            cf.set_workspace(WORKSPACE)
        check(out, lse, ref)
        check_grad(got, gref)


def test_a_window_that_hides_nothing_is_causal_attention():
    h, kv, lens = 8, 2, [300, 1, 420]
    x, dout, at = problem(4, lens, h, kv)
    T, s = x.shape[0], x.stride()[:2]
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    desc = cf.prompt_desc(T, 3, h, kv, 0.09, q=s, k=s, v=s)
    out, lse, delta, dx = torch.zeros_like(dout), torch.zeros(h, T, device=DEV), torch.zeros(h, T, device=DEV), torch.zeros_like(x)
    cf.attn_prompt(desc, q, k, v, at, out, lse)
    cf.attn_prompt_grad(desc, q, k, v, out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:])
    ref, gref = definition(x, h, kv, at, 0.09, T, 0, dout)
    for window, sinks in ((T, 0), (2 ** 31 - 1, 2 ** 31 - 1), (700, 21), (1, T)):
        (o, l), got = run(x, h, kv, at, 0.09, window, sinks, dout)
        assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(dx, torch.cat([got["dq"], got["dk"], got["dv"]], 1))
    for window, sinks in ((420, 0), (600, 50), (1, 700), (719, 1)):          # nothing is hidden of these sequences, but of a longer one
        (o, l), got = run(x, h, kv, at, 0.09, window, sinks, dout)
        check(o, l, ref)
        check_grad(got, gref)


def test_rows_of_no_sequence_are_left_as_they_were(shape_of_launch):
    h, kv, lens = 4, 2, [70, 0, 230]
    x, dout, at = problem(3, lens, h, kv, 37, 96)
    for t in (x, dout):
        t[:37], t[337:] = math.nan, math.inf
    ref, gref = definition(x, h, kv, at, 0.1, 50, 3, dout)
    (out, lse), got = run(x, h, kv, at, 0.1, 50, 3, dout)
    check(out, lse, ref)
    check_grad(got, gref)
    for r in (slice(0, 37), slice(337, 433)):
        assert bool((out[r] == -7).all()) and bool((lse[:, r] == -7).all())


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("t", [150, 155, 190, 280, 420])
def test_what_the_window_hides_has_no_influence(t, value, shape_of_launch):
    """One token's K and V are not finite: a sink, one behind the sinks, one in the middle, one of another sequence.  The rows that do not see it are as
    without; so are the gradients of what those rows alone reach."""
    h, kv, lens, window, sinks = 4, 2, [150, 381, 60], 70, 4
    x, dout, at = problem(21, lens, h, kv)
    x[t, h:] = 0
    ref, gref = definition(x, h, kv, at, 0.09, window, sinks, dout)
    x[t, h:] = value
    (out, lse), got = run(x, h, kv, at, 0.09, window, sinks, dout)
    rows = torch.zeros(591, dtype=torch.bool, device=DEV)
    rows[150:531] = ~_hidden(381, window, sinks)[:, t - 150]
    reached = torch.zeros_like(rows)                                         # keys that such a row sees
    reached[150:531] = (~_hidden(381, window, sinks))[rows[150:531]].any(0)
    assert not bool(torch.isfinite(out[rows].float()).all())
    for part in ref:
        (part if part.ndim == 3 else part.t())[rows] = math.nan
    out[rows], lse[:, rows] = -7, -7
    check(out, lse, ref)
    for n, touched in (("dq", rows), ("dk", reached), ("dv", reached)):
        for part in gref:
            part[n][touched] = math.nan
        got[n][touched] = -7
    check_grad(got, gref)


@pytest.mark.parametrize("what", ["q", "dout", "v_feature"])
def test_one_row_that_is_not_finite(what, shape_of_launch):
    """Q or dout of one token, or one feature of V of one: the gradients of keys that the token does not see are as without."""
    h, kv, lens, window, sinks, t = 4, 1, [150, 381, 60], 64, 2, 300
    x, dout, at = problem(22, lens, h, kv)
    if what == "v_feature":
        x[t, h + kv:, 7] = 0
    ref, gref = definition(x, h, kv, at, 0.09, window, sinks, dout)
    if what == "q":
        x[t, :h] = math.inf
    elif what == "dout":
        dout[t] = -math.inf
    else:
        x[t, h + kv:, 7] = math.nan
    (out, lse), got = run(x, h, kv, at, 0.09, window, sinks, dout)
    hidden = _hidden(381, window, sinks)
    rows, reached = torch.zeros(591, dtype=torch.bool, device=DEV), torch.zeros(591, dtype=torch.bool, device=DEV)
    if what == "v_feature":
        rows[150:531] = ~hidden[:, t - 150]
    else:
        rows[t] = True
    reached[150:531] = (~hidden)[rows[150:531]].any(0)
    if what != "dout":
        for part in ref:
            (part if part.ndim == 3 else part.t())[rows] = math.nan
        out[rows], lse[:, rows] = -7, -7
    check(out, lse, ref)
    for n, touched in (("dq", rows), ("dk", reached), ("dv", reached)):
        if what == "v_feature" and n == "dv":                                # (dV = P^T dout is not made of V)
            continue
        assert not bool(torch.isfinite(got[n][touched].float()).all())
        for part in gref:
            part[n][touched] = math.nan
        got[n][touched] = -7
    check_grad(got, gref)


@pytest.mark.parametrize("case", [(4, 4, [700, 500], 128, 4), (8, 1, [900], 256, 16), (2, 1, [64, 300, 33], 40, 0)])
def test_dq_is_rounded_once(case, shape_of_launch):
    """dS enters dQ with more than bf16 holds, so that dQ's error has two parts.  Its own rounding: an element x = m 2^e, 1 <= m < 2, is off by up to
    2^(e-8), evenly spread, of root mean square 2^(e-8) / sqrt(3) <= 2^-8 |x| / sqrt(3).  And that of `out` in delta = sum of g o: a row's delta is off by
    the root mean square 2^-8 / sqrt(3) |g o|_2, and its dQ by scale times that times P K.  Sums of squares over 4e4 elements and more (150 rows of delta
    and more) stay within 15 % of what is expected of them; what is left out, fp32 sums and second roundings (2^-16), is far below."""
    h, kv, lens, window, sinks = case
    x, dout, at = problem(31, lens, h, kv)
    scale, g = 1 / math.sqrt(D), h // kv
    _, (res, _) = definition(x, h, kv, at, scale, window, sinks, dout)
    _, got = run(x, h, kv, at, scale, window, sinks, dout)
    expected = (2.0 ** -16 / 3) * float((res["dq"] ** 2).sum())
    for a, b in zip(at[:-1].tolist(), at[1:].tolist()):
        for i in range(h):
            q, k, v, go = x[a:b, i].double(), x[a:b, h + i // g].double(), x[a:b, h + kv + i // g].double(), dout[a:b, i].double()
            p = torch.softmax((q @ k.t() * scale).masked_fill(_hidden(b - a, window, sinks), -math.inf), 1)
            expected += (2.0 ** -16 / 3) * scale ** 2 * float((((go * (p @ v)) ** 2).sum(1) * ((p @ k) ** 2).sum(1)).sum())
    assert float(((got["dq"].double() - res["dq"]) ** 2).sum()) <= 1.15 * expected


def test_gradient_against_differences():
    """Along a direction, the loss sum(out * dout) in 64 bits changes as the gradient says (slack as in the test of causal attention)."""
    h, kv, lens, scale, window, sinks = 4, 2, [60, 190], 0.09, 37, 3
    x, dout, at = problem(31, lens, h, kv)
    _, (_, off) = definition(x, h, kv, at, scale, window, sinks, dout)
    _, got = run(x, h, kv, at, scale, window, sinks, dout)
    eps = 1e-4
    for n, r in (("dq", slice(0, h)), ("dk", slice(h, h + kv)), ("dv", slice(h + kv, h + 2 * kv))):
        step = torch.randn(x[:, r].shape, dtype=torch.float64, device=DEV)
        loss = []
        for sign in (1, -1):
            y = x.double().clone()
            y[:, r] += sign * eps * step
            loss.append(float((definition(y, h, kv, at, scale, window, sinks)[0] * dout.double()).sum()))
        change = (loss[0] - loss[1]) / (2 * eps)
        slack = 10 * float((off[n] * step).square().sum().sqrt()) + 1e-5 * abs(change) + 1e-6
        assert abs(change - float((got[n].double() * step).sum())) <= slack


def test_graph_replays_with_other_sequences():
    h, kv, T, w = 4, 2, 600, cf.window(90, 3)
    x, dout, at = problem(51, [600, 0, 0], h, kv)
    q, k, v, s = x[:, :h], x[:, h:h + kv], x[:, h + kv:], x.stride()[:2]
    out, lse, delta, dx = torch.zeros_like(dout), torch.zeros(h, T, device=DEV), torch.zeros(h, T, device=DEV), torch.zeros_like(x)
    desc = cf.prompt_desc(T, 3, h, kv, 0.09, q=s, k=s, v=s)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cf.attn_prompt_window(desc, w, q, k, v, at, out, lse, side)
        cf.attn_prompt_window_grad(desc, w, q, k, v, out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:], side)
    for i, lens in enumerate(([600, 0, 0], [1, 599, 0], [200, 200, 200], [0, 0, 600])):
        at.copy_(starts(lens))
        x.copy_(make(60 + i, T, h, kv))
        graph.replay()
        torch.cuda.synchronize()
        eager = run(x, h, kv, at, 0.09, 90, 3, dout)[1]
        assert torch.equal(dx, torch.cat([eager["dq"], eager["dk"], eager["dv"]], 1))


def test_heads_outermost_and_offsets_beyond_32_bits():
    T, stride, lens = 4200, 1 << 19, [4000, 200]
    x, dout, at = problem(41, lens, 1, 1)
    (want, wlse), wgrad = run(x, 1, 1, at, 0.09, 600, 5, dout)
    big = [torch.zeros((T - 1) * stride + 3 * D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    view, dview = (b.as_strided((T, 3, D), (stride, D, 1)) for b in big)
    view.copy_(x)
    out, lse, delta = torch.empty(T, 1, D, dtype=torch.bfloat16, device=DEV), torch.empty(1, T, device=DEV), torch.empty(1, T, device=DEV)
    s, w = view.stride()[:2], cf.window(600, 5)
    desc = cf.prompt_desc(T, 2, 1, 1, 0.09, q=s, k=s, v=s)
    q, k, v = view[:, :1], view[:, 1:2], view[:, 2:]
    cf.attn_prompt_window(desc, w, q, k, v, at, out, lse)
    cf.attn_prompt_window_grad(desc, w, q, k, v, out, lse, dout, at, delta, dview[:, :1], dview[:, 1:2], dview[:, 2:])
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wlse)
    assert all(torch.equal(dview[:, r:r + 1], wgrad[n]) for n, r in (("dq", 0), ("dk", 1), ("dv", 2)))


@pytest.mark.parametrize("room", [512 << 20, 40 << 20, 8 << 20, 300 << 10])
def test_first_keys_of_a_long_sequence_among_many_blocks(room):
    """Keys enough to fill the chip, of which only a sequence's first are seen to its end: their walks alone are cut, as far as the workspace reaches."""
    h, kv, lens, window, sinks = 16, 16, [8000, 210], 100, 3
    x, dout, at = problem(61, lens, h, kv)
    desc = cf.prompt_desc(sum(lens), 2, h, kv, 0.09)
    assert 0 < cf.attn_prompt_window_workspace_bytes(desc, cf.window(window, sinks)) <= WORKSPACE.numel()
    cf.set_workspace(WORKSPACE[:room])
    try:
        (out, lse), got = run(x, h, kv, at, 0.09, window, sinks, dout)
    finally:
        cf.set_workspace(WORKSPACE)
    for u in (0, 7, 15):                                                     # (head by head: the definition's scores are large)
        part = torch.cat([x[:, u:u + 1], x[:, h + u:h + u + 1], x[:, h + kv + u:h + kv + u + 1]], 1).contiguous()
        ref, gref = definition(part, 1, 1, at, 0.09, window, sinks, dout[:, u:u + 1])
        check(out[:, u:u + 1], lse[u:u + 1], ref)
        check_grad({n: t[:, u:u + 1] for n, t in got.items()}, gref)


@pytest.mark.parametrize("h, kv", [(8, 1), (16, 16)])
def test_a_long_sequence_among_many_short_ones(h, kv):
    """More than 64 sequences, some of them empty or of one token, and a long one whose first keys are seen by all of it."""
    lens, window, sinks = [1, 0, 3, 70] * 20 + [4000] + [40, 1, 0] * 15, 64, 2
    x, dout, at = problem(62, lens, h, kv)
    (out, lse), got = run(x, h, kv, at, 0.09, window, sinks, dout)
    g = h // kv
    for u in (0, kv - 1):
        part = torch.cat([x[:, u * g:(u + 1) * g], x[:, h + u:h + u + 1], x[:, h + kv + u:h + kv + u + 1]], 1).contiguous()
        ref, gref = definition(part, g, 1, at, 0.09, window, sinks, dout[:, u * g:(u + 1) * g])
        check(out[:, u * g:(u + 1) * g], lse[u * g:(u + 1) * g], ref)
        check_grad(dict(dq=got["dq"][:, u * g:(u + 1) * g], dk=got["dk"][:, u:u + 1], dv=got["dv"][:, u:u + 1]), gref)


@pytest.mark.parametrize("seed", range(4))
def test_starts_of_nonsense_touch_nothing_outside(seed, shape_of_launch):
    """Whatever the table holds, only rows of the results change, and the calls end."""
    h, kv, T, n = 4, 2, 500, (3, 3, 80, 1)[seed]
    x, dout, _ = problem(70 + seed, [T], h, kv)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    top = 2 ** 31 - 1
    lo, hi = ((-top, top), (-600, 1200), (-top, top), (-top, top))[seed]
    at = torch.randint(lo, hi, (n + 1,), generator=g, device=DEV, dtype=torch.int32)
    q, k, v, s = x[:, :h], x[:, h:h + kv], x[:, h + kv:], x.stride()[:2]
    desc, w = cf.prompt_desc(T, n, h, kv, 0.09, q=s, k=s, v=s), cf.window(40, 3)
    out = torch.full((T + 2, h, D), 3.0, dtype=torch.bfloat16, device=DEV)
    dx = torch.full((T + 2, h + 2 * kv, D), 3.0, dtype=torch.bfloat16, device=DEV)
    lse, delta = torch.zeros(h, T, device=DEV), torch.zeros(h, T, device=DEV)
    cf.attn_prompt_window(desc, w, q, k, v, at, out[1:-1], lse)
    cf.attn_prompt_window_grad(desc, w, q, k, v, out[1:-1], lse, dout, at, delta, dx[1:-1, :h], dx[1:-1, h:h + kv], dx[1:-1, h + kv:])
    torch.cuda.synchronize()
    for t in (out, dx):
        assert bool((t[0] == 3).all()) and bool((t[-1] == 3).all())
