"""Causal attention of packed prompts, and its gradient, on the GPU against the definition in 64 bits.  Needs an MI355X: ``-m gpu``.

Tolerances of the output.  Probabilities are rounded to bf16 (2^-8 of each, in numerator and, the rounded ones being summed, in the
denominator: the weights of the average sum to one, so a row moves by at most 2 * 2^-8 of the weighted mean of |v|), and the output by 2^-8
of itself.  The scores are fp32 sums of 128 exact products in fp32: off by at most 128 * 2^-24 of scale * sum |q k| (taken as 2^-17
of it), which moves a weight by as much, relatively.  lse: that much absolutely, and a few roundings of 2^-23 of |lse| + 1 (a sum of n
positive terms, lanes and tiles apart: under 2^-18)."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(ws)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)


@pytest.fixture(params=["4x100000", "8x100000", "4x1", "8x2", "4x3"])
def shape_of_launch(request, monkeypatch):
    """Waves of a workgroup, and key tiles of a split."""
    monkeypatch.setenv("COMMFUSE_CAUSAL", request.param)


def make(seed, T, h, kv, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(T, h + 2 * kv, D, generator=g, device=DEV)
    x[:, :h + kv] *= sigma
    return x.to(torch.bfloat16)


def starts(lens, before=0):
    at = [before]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def definition(q, k, v, at, scale):
    """(out, lse, weighted mean of |v|, largest scale * sum |q k| of a visible key) in 64 bits; rows of no sequence are NaN."""
    T, h = q.shape[:2]
    g = h // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, lse, mean, size = (torch.full(s, math.nan, dtype=torch.float64, device=DEV) for s in ((T, h, D), (h, T), (T, h, D), (h, T)))
    for a, b in zip(at[:-1].tolist(), at[1:].tolist()):
        hidden = torch.ones(b - a, b - a, dtype=torch.bool, device=DEV).triu(1)
        for i in range(h):
            kk, vv = k[a:b, i // g], v[a:b, i // g]
            s = (q[a:b, i] @ kk.t() * scale).masked_fill(hidden, -math.inf)
            lse[i, a:b] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            out[a:b, i] = p @ vv
            mean[a:b, i] = p @ vv.abs()
            size[i, a:b] = (q[a:b, i].abs() @ kk.abs().t() * scale).masked_fill(hidden, 0).amax(1) if b > a else 0
    return out, lse, mean, size


def check(out, lse, ref):
    want, wlse, mean, size = ref
    some = ~torch.isnan(wlse)
    moved = 2.0 ** -17 * size
    limit = 2.0 ** -8 * want.abs() + (2.0 ** -7 + 2 * moved.t()[..., None]) * mean
    bad = ~((out.double() - want).abs() <= limit) & some.t()[..., None]
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())
    if lse is not None:
        bad = ~((lse.double() - wlse).abs() <= moved + 2.0 ** -18 * (wlse.abs() + 1)) & some
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), float((lse.double() - wlse).abs()[some].max()))


def run(x, h, kv, at, scale, with_lse=True, o=None):
    T = x.shape[0]
    out = torch.full((T, h, D), -7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((h, T), -7.0, device=DEV) if with_lse else None
    s = x.stride()[:2]
    cf.attn_prompt(cf.prompt_desc(T, at.numel() - 1, h, kv, scale, q=s, k=s, v=s), x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, out, lse)
    torch.cuda.synchronize()
    return out, lse


CASES = [  # heads, key heads, lengths
    (1, 1, [1]), (8, 1, [1, 1, 1]), (4, 4, [2]), (4, 4, [63]), (4, 2, [64]), (4, 1, [65, 1]), (8, 1, [127, 129, 3]), (2, 2, [300]),
    (5, 1, [17, 0, 33, 0, 0, 260]), (6, 2, [1] * 70 + [200] + [2] * 40), (16, 2, [511, 513]), (1, 1, [1025, 7]), (3, 3, [640, 64, 128, 5]),
    (32, 1, [40, 100]), (12, 4, [700]), (8, 8, [0, 5, 0])]


@pytest.mark.parametrize("case", CASES)
def test_output_and_lse(case, shape_of_launch):
    h, kv, lens = case
    x = make(len(lens) * 100 + lens[0], sum(lens), h, kv)
    at = starts(lens)
    ref = definition(x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, 1 / math.sqrt(D))
    out, lse = run(x, h, kv, at, 1 / math.sqrt(D))
    check(out, lse, ref)
    check(run(x, h, kv, at, 1 / math.sqrt(D), False)[0], None, ref)
    again = run(x, h, kv, at, 1 / math.sqrt(D))
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("case", [(8, 1, [2000, 90]), (4, 4, [1, 3000]), (2, 1, [4097])])
def test_longer_prompts_without_overrides(case):
    h, kv, lens = case
    x = make(7, sum(lens), h, kv, 2.0)
    at = starts(lens)
    out, lse = run(x, h, kv, at, 0.05)
    check(out, lse, definition(x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, 0.05))


def test_rows_of_no_sequence_are_left_as_they_were(shape_of_launch):
    h, kv, lens = 4, 2, [70, 0, 130]
    x = make(3, 333, h, kv)
    x[:37] = math.nan                                                # in front of the first sequence, and behind the last
    x[237:] = math.inf
    at = starts(lens, 37)
    out, lse = run(x, h, kv, at, 0.1)
    check(out, lse, definition(x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, 0.1))
    for r in (slice(0, 37), slice(237, 333)):
        assert bool((out[r] == -7).all()) and bool((lse[:, r] == -7).all())


def test_peaked_flat_and_equal_scores(shape_of_launch):
    """Scores of sigma 60 (one key takes all), of zero (averages), and all equal and large."""
    at = starts([190, 200])
    for sigma, scale in ((8.0, 0.7), (1e-4, 1.0)):
        x = make(11, 390, 2, 1, sigma)
        check(*run(x, 2, 1, at, scale), definition(x[:, :2], x[:, 2:3], x[:, 3:], at, scale))
    x = make(12, 390, 2, 1)
    x[:, :3] = 8.0
    check(*run(x, 2, 1, at, 1.0), definition(x[:, :2], x[:, 2:3], x[:, 3:], at, 1.0))


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_a_token_does_not_see_has_no_influence(value, shape_of_launch):
    """K and V of two tokens are not finite: rows in front of them and of the other sequences are as with zeros there."""
    h, kv, lens = 4, 2, [150, 81, 160]
    clean = make(21, sum(lens), h, kv)
    at = starts(lens)
    spoilt = clean.clone()
    for t in (100, 190):
        clean[t, h:] = 0
        spoilt[t, h:] = value
    out, lse = run(spoilt, h, kv, at, 0.09)
    ref = definition(clean[:, :h], clean[:, h:h + kv], clean[:, h + kv:], at, 0.09)
    for part in ref:                                                 # those that see them are not looked at
        rows = part if part.ndim == 3 else part.t()
        rows[100:150] = math.nan
        rows[190:231] = math.nan
    check(out, lse, ref)
    # ... and V alone: what sees it is not finite, as the definition has it
    spoilt = clean.clone()
    spoilt[100, h + kv:] = value
    out, lse = run(spoilt, h, kv, at, 0.09)
    assert not bool(torch.isfinite(out[100:150]).any()) and bool(torch.isfinite(out[:100]).all()) and bool(torch.isfinite(out[150:]).all())


def test_layouts_of_heads_and_tokens():
    """Heads outermost; padded rows."""
    h, kv, lens = 4, 2, [100, 57]
    T = sum(lens)
    x = make(31, T, h, kv)
    at = starts(lens)
    want, lse0 = run(x, h, kv, at, 0.09)
    q, k, v = (t.transpose(0, 1).contiguous() for t in (x[:, :h], x[:, h:h + kv], x[:, h + kv:]))
    wide = torch.full((T, h + 3, D + 8), -7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(h, T, device=DEV)
    o = wide[:, 1:1 + h, :D]
    cf.attn_prompt(cf.prompt_desc(T, 2, h, kv, 0.09, q=(D, T * D), k=(D, T * D), v=(D, T * D), o=o.stride()[:2]), q, k, v, at, o, lse)
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(lse, lse0)
    assert bool((wide[:, 0] == -7).all()) and bool((wide[:, 1 + h:] == -7).all()) and bool((wide[..., D:] == -7).all())


def test_offsets_beyond_32_bits():
    """Tokens a MiB apart: keys 4 GiB from the first."""
    T, h, stride = 4200, 1, 1 << 19
    x = make(41, T, h, 1)
    big = torch.zeros((T - 1) * stride + 3 * D, dtype=torch.bfloat16, device=DEV)
    view = big.as_strided((T, 3, D), (stride, D, 1))
    view.copy_(x)
    at = starts([T])
    assert all(torch.equal(a, b) for a, b in zip(run(view, 1, 1, at, 0.09), run(x, 1, 1, at, 0.09)))


def test_graph_replays_with_other_sequences():
    h, kv, T = 4, 2, 600
    x, at = make(51, T, h, kv), starts([600, 0, 0])
    out, lse, s = torch.zeros(T, h, D, dtype=torch.bfloat16, device=DEV), torch.zeros(h, T, device=DEV), x.stride()[:2]
    desc = cf.prompt_desc(T, 3, h, kv, 0.09, q=s, k=s, v=s)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cf.attn_prompt(desc, x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, out, lse, side)
    for i, lens in enumerate(([600, 0, 0], [1, 599, 0], [200, 200, 200], [0, 0, 600])):
        at.copy_(starts(lens))
        x.copy_(make(60 + i, T, h, kv))
        graph.replay()
        torch.cuda.synchronize()
        eager = run(x, h, kv, at, 0.09)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
