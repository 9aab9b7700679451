"""Attention of new tokens over the paged cache on the GPU against the definition in 64 bits.  Needs an MI355X: ``-m gpu``.

The cache's values are what the pages stand for (bf16, or codes times powers of two), so the tolerances are those of the same
attention over dense keys: probabilities rounded to bf16 in numerator and denominator (2 * 2^-8 of the weighted mean of |v|), the output's
own rounding (2^-8), fp32 scores (2^-17 of scale * sum |q k|, taken twice as a change of the weights), lse 2^-18 of |lse| + 1."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
WORKSPACE = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    global WORKSPACE
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    WORKSPACE = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(WORKSPACE)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)
    WORKSPACE = None


class Batch:
    """Sequences with `new` tokens each and `ctx` tokens in a pool of shuffled pages; what no sequence holds is NaN, or, in the
    exponents, 255."""

    def __init__(self, seed, heads, kv, page, dtype, new, ctx, spare=3, before=0, behind=0, tokens_outside=False):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.heads, self.kv, self.page, self.dtype, self.new, self.ctx = heads, kv, page, dtype, new, ctx
        need = [-(-c // page) for c in ctx]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=self.g, device=DEV).int()
        self.table = torch.full((len(new), max(need + [1]) + 1), -5, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        held = torch.zeros(self.pages, page, dtype=torch.bool, device=DEV)
        for i, c in enumerate(ctx):
            for j in range(need[i]):
                held[self.table[i, j].long(), :min(page, c - j * page)] = True
        shape = (self.pages, page, kv, D) if tokens_outside else (self.pages, kv, page, D)
        look = (lambda t: t.transpose(1, 2)) if tokens_outside else (lambda t: t)
        self.values, self.pool, self.exps = [], [], []
        for x in range(2):
            raw = look(torch.randn(shape, generator=self.g, device=DEV)) * torch.exp2(torch.randint(-3, 4, (self.pages, kv, page, 1), generator=self.g, device=DEV).float() * 0.5)
            free = ~held[:, None, :, None]
            if dtype == "e4m3":
                e = torch.ceil(torch.log2(raw.abs().amax(-1) / 448))
                code = (raw * torch.exp2(-e)[..., None]).to(torch.float8_e4m3fn)
                self.values.append((code.double() * torch.exp2(e.double())[..., None]))
                code = code.view(torch.uint8).masked_fill(free, 255)
                self.exps.append((e + 127).to(torch.uint8).masked_fill(free[..., 0], 255).contiguous())
            else:
                code = raw.to(torch.bfloat16)
                self.values.append(code.double())
                code = code.masked_fill(free, math.nan)
                self.exps.append(None)
            dense = torch.empty(shape, dtype=code.dtype, device=DEV)
            look(dense).copy_(code)
            self.pool.append(look(dense))
        self.strides = self.pool[0].stride()[:3] if tokens_outside else (0, 0, 0)
        self.total = before + sum(new) + behind
        self.starts = torch.tensor([before + sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV)
        self.lens = torch.tensor(ctx, dtype=torch.int32, device=DEV)
        self.qkv = torch.randn(self.total, heads + 2, D, generator=self.g, device=DEV).to(torch.bfloat16)
        self.q = self.qkv[:, 1:1 + heads]

    def cache(self):
        return cf.cache_desc(self.dtype, self.pages, self.page, self.kv, D, self.strides), cf.make_cache(*self.pool, *self.exps)

    def run(self, scale=1 / math.sqrt(D), max_q=None, max_kv=None, with_lse=True, stream=None, out=None, lse=None):
        if out is None:
            out = torch.full((self.total, self.heads, D), -7.0, dtype=torch.bfloat16, device=DEV)
            lse = torch.full((self.heads, self.total), -7.0, device=DEV) if with_lse else None
        desc = cf.paged_desc(len(self.new), self.heads, self.total, max(self.new) if max_q is None else max_q, max(self.ctx) if max_kv is None else max_kv,
                             self.table.shape[1], scale, q=self.q.stride()[:2])
        cf.attn_paged(*self.cache(), desc, self.q, self.starts, self.lens, self.table, out, lse, stream)
        if stream is None:
            torch.cuda.synchronize()
        return out, lse

    def definition(self, scale=1 / math.sqrt(D), absent=()):
        """(out, lse, weighted mean of |v|, largest scale * sum |q k|), rows of no sequence NaN; absent: (sequence, page index)."""
        T, h, g = self.total, self.heads, self.heads // self.kv
        out, lse, mean, size = (torch.full(s, math.nan, dtype=torch.float64, device=DEV) for s in ((T, h, D), (h, T), (T, h, D), (h, T)))
        for s, (m, n) in enumerate(zip(self.new, self.ctx)):
            a = int(self.starts[s])
            pages = self.table[s, :-(-n // self.page)].long().clamp(0, self.pages - 1)
            j = torch.arange(n, device=DEV)
            hidden = j[None, :] > n - m + torch.arange(m, device=DEV)[:, None]
            for (sq, pg) in absent:
                if sq == s:
                    hidden = hidden | (j // self.page == pg)[None, :]
            for u in range(h):
                k, v = (x[:, u // g][pages].reshape(-1, D)[:n] for x in self.values)
                q = self.q[a:a + m, u].double()
                sc = (q @ k.t() * scale).masked_fill(hidden, -math.inf)
                lse[u, a:a + m] = torch.logsumexp(sc, 1) if n else -math.inf
                p = torch.exp(sc - torch.nan_to_num(lse[u, a:a + m], neginf=0.0)[:, None])
                out[a:a + m, u], mean[a:a + m, u] = p @ v, p @ v.abs()
                size[u, a:a + m] = (q.abs() @ k.abs().t() * scale).masked_fill(hidden, 0).amax(1) if n else 0
        return out, lse, mean, size


def check(out, lse, ref):
    want, wlse, mean, size = ref
    some = ~torch.isnan(wlse)
    moved = 2.0 ** -17 * size
    bad = ~((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -7 + 2 * moved.t()[..., None]) * mean) & some.t()[..., None]
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())
    if lse is not None:
        empty = torch.isinf(wlse)
        assert bool((lse[empty] == -math.inf).all())
        bad = ~((lse.double() - wlse).abs() <= moved + 2.0 ** -18 * (wlse.abs() + 1)) & some & ~empty
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())
    assert bool((out.transpose(0, 1)[~some] == -7).all()) and (lse is None or bool((lse[~some] == -7).all()))


FEW = [  # heads, key heads, page, new, ctx
    (8, 1, 16, [1], [1]), (8, 1, 16, [1], [16]), (8, 1, 16, [1], [1003]), (4, 4, 16, [1] * 6, [33, 1, 32, 31, 257, 0]), (16, 1, 64, [1, 1], [700, 65]),
    (5, 1, 32, [1, 2, 3], [3, 2, 300]), (32, 1, 128, [1], [130]), (12, 4, 16, [4, 1, 5], [4, 1000, 77]), (1, 1, 1024, [16, 7], [20, 2100]),
    (2, 2, 256, [1, 0, 1, 5], [5, 9, 0, 513]), (6, 2, 16, [1] * 40, list(range(0, 400, 10))), (8, 8, 64, [2], [4096]), (8, 1, 16, [3], [1])]
MANY = [
    (8, 1, 16, [40], [40]), (8, 1, 32, [130, 5], [130, 700]), (4, 4, 64, [33, 64, 1], [333, 64, 65]), (4, 2, 16, [200], [1111]), (1, 1, 128, [129, 0, 300], [129, 4, 555]),
    (5, 1, 256, [77], [1200]), (16, 2, 1024, [100, 100], [50, 3000]), (2, 1, 16, [70, 70], [0, 69])]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [None, "4x1", "4x3", "8x2", "8x100000"])
@pytest.mark.parametrize("case", FEW + MANY)
def test_output_and_lse(case, dtype, chunk, monkeypatch):
    heads, kv, page, new, ctx = case
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    b = Batch(heads * 100 + sum(ctx) % 97, heads, kv, page, dtype, new, ctx, before=2, behind=3)
    ref = b.definition()
    out, lse = b.run()
    check(out, lse, ref)
    check(b.run(with_lse=False)[0], None, ref)
    again = b.run()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    check(*b.run(max_q=max(new) + 9, max_kv=max(ctx) + 5000), ref)            # bounds, not lengths


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", [(8, 1, 64, [1, 1], [40000, 3]), (4, 4, 16, [1] * 64, [(i * 61) % 2000 for i in range(64)]), (8, 1, 32, [700, 300], [5000, 300])])
def test_longer_contexts_without_overrides(case, dtype):
    heads, kv, page, new, ctx = case
    b = Batch(5, heads, kv, page, dtype, new, ctx)
    check(*b.run(), b.definition())
    cf.set_workspace(None)                                                    # without one keys are not split
    try:
        check(*b.run(), b.definition())
    finally:
        cf.set_workspace(WORKSPACE)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 90])
def test_tokens_outside_heads_and_shared_pages(dtype, new):
    b = Batch(6, 4, 2, 32, dtype, [new, new], [500, 300], tokens_outside=True)
    b.table[1, :5] = b.table[0, :5]                                           # a common prefix
    check(*b.run(), b.definition())


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 3, 100])
@pytest.mark.parametrize("chunk", [None, "4x2"])
def test_pages_that_do_not_exist_hold_no_tokens(dtype, new, chunk, monkeypatch):
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    b = Batch(7, 8, 2, 16, dtype, [new, new, new], [600, 170, 128])
    b.table[0, 3], b.table[0, 17], b.table[1, 0], b.table[2, :8] = -1, b.pages, 2 ** 31 - 1, -2 ** 31
    ref = b.definition(absent=[(0, 3), (0, 17), (1, 0)] + [(2, i) for i in range(8)])
    check(*b.run(), ref)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [4, 60])
@pytest.mark.parametrize("chunk", [None, "4x1"])
def test_what_a_token_does_not_see_has_no_influence(dtype, new, chunk, monkeypatch):
    """The last token's K and V are NaN: the rows before it are as without."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    b = Batch(8, 4, 2, 16, dtype, [new], [250])
    ref = b.definition()
    page, at = int(b.table[0, 249 // 16]), 249 % 16
    for pool in b.pool:
        pool[page, :, at] = 127 if dtype == "e4m3" else math.nan
    out, lse = b.run()
    for part in ref:
        (part if part.ndim == 3 else part.t())[new - 1] = math.nan
    assert bool(torch.isnan(out[new - 1]).all()) and bool(torch.isnan(lse[:, new - 1]).all())
    out[new - 1], lse[:, new - 1] = -7, -7
    check(out, lse, ref)


def test_rows_beyond_max_q_and_tokens_beyond_max_kv():
    b = Batch(9, 4, 2, 16, "bf16", [6, 3], [100, 80])
    out, lse = b.run(max_q=4)
    full, full_lse = b.run()
    for r in (slice(0, 4), slice(6, 9)):
        assert torch.equal(out[r], full[r]) and torch.equal(lse[:, r], full_lse[:, r])
    assert bool((out[4:6] == -7).all()) and bool((lse[:, 4:6] == -7).all())
    cut = b.run(max_kv=80)
    b.ctx, b.lens[0] = [80, 80], 80
    check(*cut, b.definition())


@pytest.mark.parametrize("new", [1, 70])
def test_pools_beyond_32_bits(new):
    """Two pages four GiB apart."""
    b = Batch(10, 4, 1, 64, "e4m3", [new], [128], spare=0)
    far = (1 << 32) + 8192
    want = b.run()
    big = [torch.zeros(far + 64 * D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for x, p in zip(big, b.pool):
        x.as_strided((2, 64 * D), (far, 1)).copy_(p.reshape(2, 64 * D))
    b.pool, b.strides = big, (far, 64 * D, D)
    got = b.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_graph_replays_with_other_lengths_and_tables():
    b = Batch(11, 8, 1, 16, "e4m3", [1, 1, 1], [900, 40, 333])
    side = torch.cuda.Stream()
    out, lse = torch.zeros(3, 8, D, dtype=torch.bfloat16, device=DEV), torch.zeros(8, 3, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.run(max_kv=4096, stream=side, out=out, lse=lse)
    for i, ctx in enumerate(([900, 40, 333], [1, 0, 17], [880, 40, 300], [900, 33, 1])):
        b.lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        b.q.copy_(torch.randn(3, 8, D, generator=b.g, device=DEV))
        out.fill_(-7), lse.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        b.ctx = ctx
        check(out, lse, b.definition())
        eager = b.run(max_kv=4096)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
