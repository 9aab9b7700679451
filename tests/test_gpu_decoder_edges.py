"""Causal attention over packed prompts, its gradient and the paged cache where workspaces, numbers of sequences and values that are not
finite take paths of their own.  Needs an MI355X: ``-m gpu``.  Limits are those of the files that test each operator alone."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests import test_gpu_attn_grad as grad
from tests import test_gpu_attn_prompt as prompt
from tests.test_gpu_attn_paged import Batch
from tests.test_gpu_attn_paged import check as check_paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
SCALE = 1 / math.sqrt(D)
WORKSPACE = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    global WORKSPACE
    cf.load()
    WORKSPACE = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(WORKSPACE)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)
    WORKSPACE = None


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n, new", [(64, 1), (65, 1), (200, 1), (65, 3), (66, 30)])
def test_large_batches_in_the_workspace_that_they_ask_for(n, new, dtype):
    """One long context among short ones, in exactly the bytes asked for, with a guard behind."""
    ctx = [new + (i * 7) % 40 for i in range(n)]
    ctx[n // 2] += 6000
    b = Batch(300 + n, 8, 1, 16, dtype, [new] * n, ctx)
    ask = cf.attn_paged_workspace_bytes(b.cache()[0], cf.paged_desc(n, 8, b.total, new, max(ctx), b.table.shape[1], SCALE))
    assert ask > 64 << 10
    buf = torch.full((ask + (1 << 20),), 85, dtype=torch.uint8, device=DEV)
    cf.set_workspace(buf[:ask])
    try:
        check_paged(*b.run(), b.definition())
        assert bool((buf[ask:] == 85).all())
        assert bool((buf[64 << 10:ask] != 85).any())                          # keys were split
    finally:
        torch.cuda.synchronize()
        cf.set_workspace(WORKSPACE)


# ---- values that are not finite --------------------------------------------------------------------------------------------------
# A feature of V that is not finite makes that feature of the rows that see it so, with its sign, and nothing else: the probabilities of these
# problems are far above 2^-126.  All other elements are those of V with 0 there, up to that key's weight -- so the reference has 0 in the
# place, and the spoilt feature of the rows that see it is compared by itself.
SPOILT = [(math.inf, math.inf), (-math.inf, -math.inf), (math.nan, math.nan), ("both", math.nan)]      # value(s), what sees it


def _packed_case(lens, h, kv, tokens, value, seed):
    """(spoilt x, clean x, starts, [(row mask, feature, key head)])"""
    x = prompt.make(seed, sum(lens), h, kv)
    at, clean, marks = prompt.starts(lens), x.clone(), []
    ends = at[1:].tolist()
    for i, t in enumerate(tokens):
        head, d = h + kv + i % kv, (37 * i + 5) % D
        end = next(e for e in ends if e > t)
        seen = torch.zeros(x.shape[0], dtype=torch.bool, device=DEV)
        if value == "both":
            other = max([b for b in [0] + ends if b <= t]) if t + 1 >= end else t + 1
            x[t, head, d], x[other, head, d] = math.inf, -math.inf
            clean[t, head, d] = clean[other, head, d] = 0
            seen[max(t, other):end] = True
            one = torch.zeros_like(seen)
            one[min(t, other):max(t, other)] = True                       # see one of them only
            marks.append((one, d, i % kv, math.inf if t < other else -math.inf))
            marks.append((seen, d, i % kv, math.nan if other != t else -math.inf))
        else:
            x[t, head, d], clean[t, head, d] = value, 0
            seen[t:end] = True
            marks.append((seen, d, i % kv, value))
    return x, clean, at, marks


def _expect(out, marks, group):
    """Looks at the spoilt elements of out [tokens, heads, D] and puts 0 there; a later mark adds to an earlier one of the same feature."""
    for rows, d, kvh, value in marks:
        for head in range(kvh * group, (kvh + 1) * group):
            got = out[rows, head, d].float()
            want = torch.full_like(got, value)
            assert torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0)), (d, head, value, got[:5].tolist())
            out[rows, head, d] = 0


@pytest.mark.parametrize("value", [v for v, _ in SPOILT])
@pytest.mark.parametrize("chunk", [None, "4x1", "8x2", "4x100000"])
@pytest.mark.parametrize("case", [(4, 2, [150, 81, 160], [100, 190, 391 - 1]), (8, 1, [5, 3, 9, 1, 30, 2], [3, 6, 20, 49]), (1, 1, [300], [0, 130]),
                                  (6, 2, [1] * 70 + [200] + [2] * 40, [10, 75, 269, 300]), (3, 3, [700], [64, 65, 500])])
def test_one_feature_of_a_prompts_v(case, chunk, value, monkeypatch):
    h, kv, lens, tokens = case
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    x, clean, at, marks = _packed_case(lens, h, kv, tokens, value, 501)
    q, k, v = clean[:, :h], clean[:, h:h + kv], clean[:, h + kv:]
    ref = prompt.definition(q, k, v, at, SCALE)
    for with_lse in (True, False):
        out, lse = prompt.run(x, h, kv, at, SCALE, with_lse)
        for rows, d, kvh, _ in marks:
            for head in range(kvh * (h // kv), (kvh + 1) * (h // kv)):
                ref[0][rows, head, d] = 0
        _expect(out, marks, h // kv)
        prompt.check(out, lse, ref)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [None, "4x1", "8x3"])
@pytest.mark.parametrize("case", [(8, 2, 16, [4, 3, 1], [250, 64, 33]), (4, 4, 32, [7, 5], [7, 300]), (8, 1, 16, [60, 5], [700, 5]), (4, 2, 64, [33, 200], [333, 200])])
def test_one_feature_of_a_caches_v(case, chunk, dtype, monkeypatch):
    """Of one of the new tokens, and of an old one where there are any.  (e4m3 has NaN only.)"""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    heads, kv, page, new, ctx = case
    b = Batch(511, heads, kv, page, dtype, new, ctx)
    marks = []
    for s, (m, n) in enumerate(zip(new, ctx)):
        for i, key in enumerate({n - m + m // 2, (n - m) // 2}):
            d = (29 * s + 50 * i + 3) % D
            at = (int(b.table[s, key // page]), s % kv, key % page, d)
            b.pool[1][at] = 127 if dtype == "e4m3" else math.nan
            b.values[1][at] = 0
            rows = torch.zeros(b.total, dtype=torch.bool, device=DEV)
            first = int(b.starts[s]) + max(0, key - (n - m))
            rows[first:int(b.starts[s + 1])] = True
            marks.append((rows, d, s % kv, math.nan))
    ref = b.definition()
    out, lse = b.run()
    for rows, d, kvh, _ in marks:
        for head in range(kvh * (heads // kv), (kvh + 1) * (heads // kv)):
            ref[0][rows, head, d] = 0
    _expect(out, marks, heads // kv)
    check_paged(out, lse, ref)


def test_missing_pages_in_front_of_a_page_that_is_not_finite():
    """Keys of pages that do not exist are not seen, whatever page 0 holds."""
    for dtype in ("bf16", "e4m3"):
        for new in (1, 3, 40):
            b = Batch(521, 8, 2, 16, dtype, [new, new], [600, 90])
            page = int(b.table[0, 7])
            for pool in b.pool:                                               # page 0 becomes one of no sequence, NaN throughout
                pool[page].copy_(pool[0])
            for values in b.values:
                values[page].copy_(values[0])
            for e in b.exps:
                if e is not None:
                    e[page].copy_(e[0])
            b.table[b.table == 0] = page
            b.table[0, 7] = -1
            for pool in b.pool:
                pool[0] = 127 if dtype == "e4m3" else math.nan
            b.table[1, 2] = b.pages + 5
            check_paged(*b.run(), b.definition(absent=[(0, 7), (1, 2)]))


def _time(f):
    """Shortest of five, in milliseconds."""
    best = math.inf
    for _ in range(6):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


# Time with values that are not finite.  A wave whose results may be spoilt walks over its rows' keys once more, by itself, while others may have
# shared the first walk: 32 keys take it some five times as long as 64 keys take a workgroup, so a walk takes ten times as long as an unsplit one, and an
# unsplit one of these problems three times as long as the call.
SLOWER = 30


@pytest.mark.parametrize("tokens", [[100], [5000], list(range(20, 6000, 50))])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_time_of_prompts_with_a_value_that_is_not_finite(tokens, value):
    x, at = prompt.make(531, 6144, 4, 1), prompt.starts([6000, 144])
    out, lse, s = torch.empty(6144, 4, D, dtype=torch.bfloat16, device=DEV), torch.empty(4, 6144, device=DEV), x.stride()[:2]
    call = lambda: cf.attn_prompt(cf.prompt_desc(6144, 2, 4, 1, SCALE, q=s, k=s, v=s), x[:, :4], x[:, 4:5], x[:, 5:], at, out, lse)
    normal = _time(call)
    x[tokens, 5, 7] = value
    assert _time(call) <= SLOWER * normal


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 4, 100])
def test_time_of_a_cache_with_a_value_that_is_not_finite(new, dtype):
    b = Batch(541, 8, 1, 16, dtype, [new, new], [6000, 4000])
    out, lse = torch.empty(b.total, 8, D, dtype=torch.bfloat16, device=DEV), torch.empty(8, b.total, device=DEV)
    call = lambda: b.run(out=out, lse=lse, stream=torch.cuda.current_stream())
    normal = _time(call)
    for key in (70, 6000 - new + new // 2):
        b.pool[1][int(b.table[0, key // 16]), 0, key % 16, 9] = 127 if dtype == "e4m3" else math.inf
        assert _time(call) <= SLOWER * normal


# The gradient.  What a value that is not finite reaches by the formulas (all probabilities are above 2^-126, no element of Q, K, V or dout is 0):
#   dout[t, d]   dP and delta of row t: dQ of the row, dK of the keys that it sees; dV of those keys in feature d
#   V[t, d]      delta of the rows that see t: their dQ, and dK of all keys that those rows see; no dV
#   Q[t, d]      lse of row t: dQ of the row, dK and dV of the keys that it sees
#   K[t, d]      lse of the rows that see t: their dQ, dK and dV of all keys that those rows see        (NaN; an infinite score may be -inf)
# Everything else is as without it.
def _reached(what, t, a, b):
    """{result: tokens} of a sequence [a, b)"""
    row, keys, rows, every = slice(t, t + 1), slice(a, t + 1), slice(t, b), slice(a, b)
    return {"dout": dict(dq=row, dk=keys, dv=keys), "v": dict(dq=rows, dk=every), "q": dict(dq=row, dk=keys, dv=keys), "k": dict(dq=rows, dk=every, dv=every)}[what]


@pytest.mark.parametrize("what, value", [("dout", math.inf), ("dout", -math.inf), ("dout", math.nan), ("v", math.inf), ("v", math.nan), ("q", math.nan), ("k", math.nan)])
@pytest.mark.parametrize("chunk", [None, "4x1", "4x3", "4x100000"])
@pytest.mark.parametrize("case", [(4, 2, [150, 81, 160], [100, 151, 390]), (8, 1, [5, 3, 9, 1, 30, 2], [3, 6, 20, 48]), (1, 1, [300], [0, 130]),
                                  (6, 2, [1] * 70 + [200] + [2] * 40, [10, 75, 269, 300]), (3, 3, [420], [64, 65, 300]), (40, 1, [70], [33])])
def test_one_feature_of_a_gradients_operand(case, chunk, what, value, monkeypatch):
    h, kv, lens, tokens = case
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    ends = [sum(lens[:i + 1]) for i in range(len(lens))]
    for i, t in enumerate(tokens):                                            # one at a time
        x, dout, at = grad.problem(601, lens, h, kv)
        head, d = (3 * i + 1) % h, (37 * i + 5) % D
        kvh = head // (h // kv)
        clean = [y.clone() for y in (x, dout)]
        spot = dict(dout=(1, head), q=(0, head), k=(0, h + kvh), v=(0, h + kv + kvh))[what]
        (x, dout)[spot[0]][t, spot[1], d] = value
        clean[spot[0]][t, spot[1], d] = 0
        ref = grad.gradient(clean[0][:, :h], clean[0][:, h:h + kv], clean[0][:, h + kv:], clean[1], at, SCALE)
        got = grad.forward_and_gradient(x, dout, h, kv, at, SCALE)
        end = next(e for e in ends if e > t)
        a, group = end - lens[ends.index(end)], slice(kvh * (h // kv), (kvh + 1) * (h // kv))
        for n, rows in _reached(what, t, a, end).items():
            heads = kvh if n != "dq" else head if what in ("dout", "q") else group
            features = d if (what, n) == ("dout", "dv") else slice(None)
            part = got[n][rows, heads, features].float()
            if (what, n) == ("dout", "dv"):
                assert torch.equal(part.nan_to_num(7.0, 8.0, 9.0), torch.full_like(part, value).nan_to_num(7.0, 8.0, 9.0))
            else:
                assert not bool(torch.isfinite(part).any()), (n, t)
            got[n][rows, heads, features] = -7
            for r in ref:
                r[n][rows, heads, features] = math.nan
        grad.check(got, ref)


@pytest.mark.parametrize("new, ctx", [([1, 1, 1], [33, 600, 64]), ([2, 3], [50, 1000]), ([30, 50], [45, 700])])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
def test_infinite_v_of_a_caches_last_keys(new, ctx, value):
    """Places behind the last key may be read from it: the rows that see it are infinite in that feature, no row is NaN."""
    b = Batch(551, 8, 2, 16, "bf16", new, ctx)
    marks = []
    for s, n in enumerate(ctx):
        d, at = 11 + 40 * s, (int(b.table[s, (n - 1) // 16]), s % 2, (n - 1) % 16)
        b.pool[1][at][d], b.values[1][at][d] = value, 0
        rows = torch.zeros(b.total, dtype=torch.bool, device=DEV)
        rows[int(b.starts[s + 1]) - 1] = True
        marks.append((rows, d, s % 2, value))
    ref = b.definition()
    out, lse = b.run()
    for rows, d, kvh, _ in marks:
        ref[0][rows, kvh * 4:kvh * 4 + 4, d] = 0
    _expect(out, marks, 4)
    check_paged(out, lse, ref)


@pytest.mark.parametrize("what", ["dout", "v", "q"])
@pytest.mark.parametrize("tokens", [[100], [4000], [4095], list(range(20, 4096, 50))])
@pytest.mark.parametrize("h, kv, lens", [(8, 1, [4096]), (4, 4, [3000, 1096])])
def test_time_of_a_gradient_with_a_value_that_is_not_finite(h, kv, lens, tokens, what):
    x, dout, at = grad.problem(611, lens, h, kv)
    out, lse, delta, dx = torch.empty_like(dout), torch.empty(h, 4096, device=DEV), torch.empty(h, 4096, device=DEV), torch.empty_like(x)
    q, k, v, s = x[:, :h], x[:, h:h + kv], x[:, h + kv:], x.stride()[:2]
    desc = cf.prompt_desc(4096, len(lens), h, kv, SCALE, q=s, k=s, v=s)

    def call():
        cf.attn_prompt(desc, q, k, v, at, out, lse)
        cf.attn_prompt_grad(desc, q, k, v, out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:])

    normal = _time(call)
    dict(dout=dout, v=v, q=q)[what][tokens, 0, 7] = math.inf
    assert _time(call) <= SLOWER * normal


@pytest.mark.parametrize("chunk", [None, "4x1", "4x3"])
@pytest.mark.parametrize("n", [8, 9, 33, 63, 64, 65])
@pytest.mark.parametrize("h, kv", [(8, 1), (4, 4)])
def test_numbers_of_packed_sequences(n, h, kv, chunk, monkeypatch):
    """Up to 64 sequences walks are split by the starts that a wave holds, from nine on by a search over its lanes: uneven ones, empty ones at both
    ends and between, one long enough to be split, rows before the first and behind the last."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    lens = [(i * 13) % 40 if i % 5 else 0 for i in range(n)]
    lens[n // 2] = 1500
    lens[-2:] = [7, 0]
    x, dout, at = grad.problem(700 + n, lens, h, kv, 37, 96)
    for t in (x, dout):
        t[:37], t[37 + sum(lens):] = math.nan, math.inf
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    out, lse = prompt.run(x, h, kv, at, SCALE)
    prompt.check(out, lse, prompt.definition(q, k, v, at, SCALE))
    for r in (slice(0, 37), slice(37 + sum(lens), None)):
        assert bool((out[r] == -7).all()) and bool((lse[:, r] == -7).all())
    grad.check(grad.forward_and_gradient(x, dout, h, kv, at, SCALE), grad.gradient(q, k, v, dout, at, SCALE))


@pytest.mark.parametrize("power", [-110, -117, -118, -119, -121, -123, -126])
def test_rows_of_the_smallest_values_in_e4m3(power):
    """What a code and its exponent stand for, rounded to bf16: exact from e = -124 on, below that to a multiple of 2^-133, to nearest even.  Rotated
    rows: their values have more bits than bf16's subnormal numbers."""
    T, kv = 40, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(800 - power)
    k, v = ((torch.randn(T, kv, D, generator=g, device=DEV).double() * 2.0 ** power).to(torch.bfloat16) for _ in range(2))
    pools = [torch.zeros(3, kv, 16, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    exps = [torch.zeros(3, kv, 16, dtype=torch.uint8, device=DEV) for _ in range(2)]
    desc, cache = cf.cache_desc("e4m3", 3, 16, kv), cf.make_cache(*pools, *exps)
    at, slots = torch.arange(T, dtype=torch.int32, device=DEV) * 1000 + 7, torch.arange(T, dtype=torch.int64, device=DEV)
    cf.cache_write(desc, cache, cf.cache_rows(T), cf.rope_make(D), None, k, v, at, slots, None)
    back = [torch.empty_like(k) for _ in range(2)]
    cf.cache_read(desc, cache, cf.cache_rows(T), slots, *back)
    torch.cuda.synchronize()
    exact = 0
    for pool, exp, got in zip(pools, exps, back):
        codes = pool.view(torch.float8_e4m3fn).double().permute(0, 2, 1, 3).reshape(48, kv, D)[:T].cpu()
        e = exp.permute(0, 2, 1).reshape(48, kv)[:T, :, None].double().cpu() - 127
        stands_for = codes * torch.exp2(e)                                    # in 64 bits: exact
        step = torch.clamp(torch.floor(torch.log2(stands_for.abs().clamp(min=2.0 ** -140))) - 7, min=-133.0)
        want = torch.exp2(step) * torch.round(stands_for * torch.exp2(-step))
        assert torch.equal(got.double().cpu(), want)
        assert bool((want == stands_for)[(e >= -124).expand_as(want)].all())
        assert int(e.min()) >= -126
        exact += int((want == stands_for).all())
    assert exact >= (1 if power <= -118 else 2)                               # V is not rotated: exact at any size


@pytest.mark.parametrize("what", ["v", "dout"])
@pytest.mark.parametrize("chunk", [None, "4x1", "4x100000"])
@pytest.mark.parametrize("h, kv, lens, t", [(4, 2, [150, 81, 160], 180), (8, 1, [5, 30, 9, 60], 20), (1, 1, [300], 130)])
def test_finite_values_whose_products_overflow(h, kv, lens, t, what, chunk, monkeypatch):
    """One token's V (of 2^110) or dout (of 2^120): dP and delta overflow for what sees it, nothing else changes."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    x, dout, at = grad.problem(621, lens, h, kv)
    if what == "v":
        dout *= 2.0 ** 30
        part, factor = x[t, h + kv], 2.0 ** 110
    else:
        x[:, h + kv:] *= 2.0 ** 12
        part, factor = dout[t, 0], 2.0 ** 120
    clean_x, clean_g = x.clone(), dout.clone()
    (clean_x[t, h + kv] if what == "v" else clean_g[t, 0]).zero_()
    part *= factor
    ref = grad.gradient(clean_x[:, :h], clean_x[:, h:h + kv], clean_x[:, h + kv:], clean_g, at, SCALE)
    got = grad.forward_and_gradient(x, dout, h, kv, at, SCALE)
    ends = [sum(lens[:i + 1]) for i in range(len(lens))]
    end = next(e for e in ends if e > t)
    for n, rows in _reached(what, t, end - lens[ends.index(end)], end).items():
        heads = 0 if n != "dq" or what == "dout" else slice(0, h // kv)
        if n != "dv":
            assert not bool(torch.isfinite(got[n][rows, heads].float()).any()), n
        got[n][rows, heads] = -7
        for r in ref:
            r[n][rows, heads] = math.nan
    grad.check(got, ref)
