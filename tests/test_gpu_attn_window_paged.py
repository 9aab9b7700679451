"""Attention of new tokens over the paged cache with a sliding window and first tokens that stay visible, on the GPU against the definition in 64 bits.
Tolerances as for the same attention without a window: the mask changes only what the sums run over.  Needs an MI355X: ``-m gpu``."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_paged import Batch, D, DEV, check

pytestmark = pytest.mark.gpu
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


class Windowed(Batch):
    """A batch whose pages that no new token sees are not there: their entries of the table are nonsense."""

    def __init__(self, seed, heads, kv, page, dtype, new, ctx, window, sinks, **kw):
        super().__init__(seed, heads, kv, page, dtype, new, ctx, **kw)
        self.window, self.sinks, self.whole = window, sinks, self.table.clone()
        for s, (m, n) in enumerate(zip(new, ctx)):
            first = n - m - window + 1                               # of the first new token's window
            for i in range(-(-n // page)):
                if i * page >= sinks and (i + 1) * page <= first:
                    self.table[s, i] = (-3, self.pages, 2 ** 31 - 1)[i % 3]

    def run(self, scale=1 / math.sqrt(D), max_q=None, max_kv=None, with_lse=True, stream=None, out=None, lse=None):
        if out is None:
            out = torch.full((self.total, self.heads, D), -7.0, dtype=torch.bfloat16, device=DEV)
            lse = torch.full((self.heads, self.total), -7.0, device=DEV) if with_lse else None
        desc = cf.paged_desc(len(self.new), self.heads, self.total, max(self.new) if max_q is None else max_q, max(self.ctx) if max_kv is None else max_kv,
                             self.table.shape[1], scale, q=self.q.stride()[:2])
        cf.attn_paged_window(*self.cache(), desc, cf.window(self.window, self.sinks), self.q, self.starts, self.lens, self.table, out, lse, stream)
        if stream is None:
            torch.cuda.synchronize()
        return out, lse

    def definition(self, scale=1 / math.sqrt(D), absent=()):
        T, h, g = self.total, self.heads, self.heads // self.kv
        out, lse, mean, size = (torch.full(s, math.nan, dtype=torch.float64, device=DEV) for s in ((T, h, D), (h, T), (T, h, D), (h, T)))
        for s, (m, n) in enumerate(zip(self.new, self.ctx)):
            a = int(self.starts[s])
            pages = self.whole[s, :-(-n // self.page)].long().clamp(0, self.pages - 1)
            j, i = torch.arange(n, device=DEV)[None, :], n - m + torch.arange(m, device=DEV)[:, None]
            hidden = (j > i) | ((j <= i - self.window) & (j >= self.sinks))
            for (sq, pg) in absent:
                if sq == s:
                    hidden = hidden | (j // self.page == pg)
            for u in range(h):
                k, v = (x[:, u // g][pages].reshape(-1, D)[:n] for x in self.values)
                q = self.q[a:a + m, u].double()
                sc = (q @ k.t() * scale).masked_fill(hidden, -math.inf)
                lse[u, a:a + m] = torch.logsumexp(sc, 1) if n else -math.inf
                p = torch.exp(sc - torch.nan_to_num(lse[u, a:a + m], neginf=0.0)[:, None])
                out[a:a + m, u], mean[a:a + m, u] = p @ v, p @ v.abs()
                size[u, a:a + m] = (q.abs() @ k.abs().t() * scale).masked_fill(hidden, 0).amax(1) if n else 0
        return out, lse, mean, size


FEW = [  # heads, key heads, page, new, ctx, window, sinks
    (8, 1, 16, [1], [1], 1, 0), (8, 1, 16, [1], [2], 1, 0), (8, 1, 16, [1], [1003], 1, 0), (8, 1, 16, [1], [1003], 64, 4), (8, 1, 64, [1], [1003], 33, 70),
    (4, 4, 16, [1] * 6, [33, 1, 32, 31, 257, 0], 20, 2), (16, 1, 64, [1, 1], [700, 65], 64, 1), (5, 1, 32, [1, 2, 3], [3, 2, 300], 100, 0),
    (32, 1, 128, [1], [630], 200, 4), (12, 4, 16, [4, 1, 5], [4, 1000, 77], 31, 16), (1, 1, 1024, [16, 7], [20, 5100], 1500, 4),
    (2, 2, 256, [1, 0, 1, 5], [5, 9, 0, 1513], 300, 0), (6, 2, 16, [1] * 40, list(range(0, 400, 10)), 50, 3), (8, 8, 64, [2], [4096], 1024, 4),
    (8, 1, 16, [3], [1], 1, 1), (8, 1, 16, [1], [9000], 128, 4)]
MANY = [
    (8, 1, 16, [40], [40], 7, 0), (8, 1, 32, [130, 5], [130, 700], 100, 4), (4, 4, 64, [33, 64, 1], [333, 64, 65], 50, 1), (4, 2, 16, [200], [1111], 256, 0),
    (1, 1, 128, [129, 0, 300], [129, 4, 555], 64, 64), (5, 1, 256, [77], [2200], 500, 3), (16, 2, 1024, [100, 100], [50, 9000], 700, 65), (2, 1, 16, [70, 70], [0, 69], 5, 5),
    (8, 1, 16, [64], [9000], 300, 4), (2, 2, 16, [40, 300], [6000, 5000], 1000, 129)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [None, "4x1", "4x3", "8x2", "8x100000"])
@pytest.mark.parametrize("case", FEW + MANY)
def test_output_and_lse(case, dtype, chunk, monkeypatch):
    heads, kv, page, new, ctx, window, sinks = case
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    b = Windowed(heads * 100 + sum(ctx) % 97, heads, kv, page, dtype, new, ctx, window, sinks, before=2, behind=3)
    ref = b.definition()
    out, lse = b.run()
    check(out, lse, ref)
    check(b.run(with_lse=False)[0], None, ref)
    again = b.run()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    check(*b.run(max_q=max(new) + 9, max_kv=max(ctx) + 5000), ref)            # bounds, not lengths


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", [(8, 1, 64, [1, 1], [60000, 3], 4096, 4), (4, 4, 16, [1] * 64, [(i * 61) % 3000 for i in range(64)], 512, 1),
                                  (8, 1, 32, [700, 300], [9000, 300], 2048, 16)])
def test_longer_contexts_without_overrides(case, dtype):
    heads, kv, page, new, ctx, window, sinks = case
    b = Windowed(5, heads, kv, page, dtype, new, ctx, window, sinks)
    ref = b.definition()
    desc = cf.paged_desc(len(new), heads, b.total, max(new), max(ctx), b.table.shape[1], 0.1)
    assert cf.attn_paged_window_workspace_bytes(b.cache()[0], desc, cf.window(window, sinks)) <= WORKSPACE.numel()
    for ws in (WORKSPACE, None, WORKSPACE[:1 << 20]):
        cf.set_workspace(ws)
        try:
            check(*b.run(), ref)
        finally:
            cf.set_workspace(WORKSPACE)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 70])
def test_a_window_that_hides_nothing_is_causal_attention(new, dtype):
    for window, sinks in ((500, 0), (2 ** 31 - 1, 2 ** 31 - 1), (490, 10), (1, 500)):
        b = Windowed(3, 4, 2, 32, dtype, [new, new], [500, 300], window, sinks)
        want, got = Batch.run(b), b.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 3, 100])
@pytest.mark.parametrize("chunk", [None, "4x2"])
def test_pages_that_do_not_exist_hold_no_tokens(dtype, new, chunk, monkeypatch):
    """Missing pages inside the window, among the sinks, and all that a row sees."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    b = Windowed(7, 8, 2, 16, dtype, [new, new, new], [2600, 1170, 128], 150, 40, tokens_outside=True)
    missing = [(0, 1), (0, 155), (0, 162), (1, 0), (1, 1), (1, 2)] + [(2, i) for i in range(8)]
    for s, i in missing:
        b.table[s, i] = (-1, b.pages, 2 ** 31 - 1)[i % 3]
    check(*b.run(), b.definition(absent=missing))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 4, 60])
@pytest.mark.parametrize("chunk", [None, "4x1"])
def test_what_a_token_does_not_see_has_no_influence(dtype, new, chunk, monkeypatch):
    """Tokens that no row sees, next to what is seen, and one that some rows see: K and V not finite."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    n, window, sinks = 900, 100, 3
    b = Windowed(8, 4, 2, 16, dtype, [new], [n], window, sinks)
    b.table.copy_(b.whole)                                           # (all pages are there)
    first = n - new - window + 1                                     # of the first row's window
    at = [sinks, 15, first - 1] + ([n - 1, first] if new > 1 else [])
    for t in at:
        for values, pool in zip(b.values, b.pool):
            page = int(b.table[0, t // 16])
            values[page, :, t % 16] = 0
            pool[page, :, t % 16] = 127 if dtype == "e4m3" else math.nan
    ref = b.definition()
    out, lse = b.run()
    if new > 1:
        for r in (0, new - 1):                                       # the rows that see one
            for part in ref:
                (part if part.ndim == 3 else part.t())[r] = math.nan
            assert bool(torch.isnan(out[r]).all())
            out[r], lse[:, r] = -7, -7
    check(out, lse, ref)


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("new", [1, 40])
def test_one_feature_of_v(new, value):
    """One infinite feature of V among the sinks and one in the window: that feature of the rows that see it, and nothing else."""
    n, window, sinks = 700, 90, 2
    b = Windowed(12, 8, 1, 16, "bf16", [new], [n], window, sinks)
    for t, f in ((1, 5), (n - new - 30, 77), (sinks + 3, 9)):
        page = int(b.whole[0, t // 16])
        b.pool[1][page, :, t % 16, f] = value
        b.values[1][page, :, t % 16, f] = 0
    ref = b.definition()
    out, lse = b.run()
    rows = torch.arange(new, device=DEV) + n - new - window < n - new - 30         # those whose window has the second
    odd = torch.zeros(new, D, dtype=torch.bool, device=DEV)
    odd[:, 5], odd[rows, 77] = True, True
    assert bool((~torch.isfinite(out.float()) == odd[:, None, :]).all())
    out = torch.where(odd[:, None, :], ref[0].to(out.dtype), out)
    check(out, lse, ref)


@pytest.mark.parametrize("new", [1, 70])
def test_pools_beyond_32_bits(new):
    """Two pages four GiB apart."""
    b = Windowed(10, 4, 1, 64, "e4m3", [new], [128], 40, 3, spare=0)
    far = (1 << 32) + 8192
    want = b.run()
    big = [torch.zeros(far + 64 * D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for x, p in zip(big, b.pool):
        x.as_strided((2, 64 * D), (far, 1)).copy_(p.reshape(2, 64 * D))
    b.pool, b.strides = big, (far, 64 * D, D)
    got = b.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_graph_replays_with_other_lengths_and_tables():
    b = Windowed(11, 8, 1, 16, "e4m3", [1, 1, 1], [900, 40, 333], 64, 4)
    b.table.copy_(b.whole)
    side = torch.cuda.Stream()
    out, lse = torch.zeros(3, 8, D, dtype=torch.bfloat16, device=DEV), torch.zeros(8, 3, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.run(max_kv=4096, stream=side, out=out, lse=lse)
    for ctx in ([900, 40, 333], [1, 0, 17], [880, 40, 300], [900, 33, 1]):
        b.lens.copy_(torch.tensor(ctx, dtype=torch.int32))
        b.q.copy_(torch.randn(3, 8, D, generator=b.g, device=DEV))
        out.fill_(-7), lse.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        b.ctx = ctx
        check(out, lse, b.definition())


@pytest.mark.parametrize("table", ["starts", "lens", "pages"])
@pytest.mark.parametrize("max_q", [1, 64])
def test_tables_of_nonsense_touch_nothing_outside(table, max_q):
    """Whatever the tables hold, only rows of out and lse change, and the call ends."""
    b = Windowed(13, 8, 1, 16, "bf16", [max_q] * 3, [900, 300, 77], 50, 4)
    top = 2 ** 31 - 1
    {"starts": b.starts, "lens": b.lens, "pages": b.table}[table].copy_(
        torch.randint(-top, top, {"starts": b.starts, "lens": b.lens, "pages": b.table}[table].shape, generator=b.g, device=DEV, dtype=torch.int32))
    guard = torch.full((b.total + 2, 8, D), 3.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((8, b.total), 3.0, device=DEV)
    b.run(max_q=max_q, max_kv=900, out=guard[1:-1], lse=lse)
    torch.cuda.synchronize()
    assert bool((guard[0] == 3).all()) and bool((guard[-1] == 3).all())
