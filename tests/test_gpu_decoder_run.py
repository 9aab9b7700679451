"""The operators between a decoder layer's projections as they are used: one after the other, on what the projections leave and
take, on streams of their own, captured; and with tables that hold nonsense.  Needs an MI355X: ``-m gpu``.

Tolerances of the runs.  Each step is checked against the definition in 64 bits applied to the GPU's own output of the step before, so that its
limit is that operator's (stated in the files that test it alone); steps that only place the same numbers elsewhere are compared bit by bit."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests import test_gpu_attn_grad as grad
from tests import test_gpu_attn_prompt as prompt
from tests.test_gpu_attn_paged import Batch
from tests.test_gpu_attn_paged import check as check_paged
from tests.test_gpu_rope_cache import _turned

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


def _randn(seed, *shape, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * sigma).to(torch.bfloat16)


def _int(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


class Layer:
    """One rank's attention block: a QKV projection, the operators, an output projection; a cache of shuffled pages."""

    def __init__(self, heads, kv, hidden, dtype, page, seqs, room):
        self.heads, self.kv, self.hidden, self.page = heads, kv, hidden, page
        self.w_in, self.w_out = _randn(1, hidden, (heads + 2 * kv) * D, sigma=hidden ** -0.5), _randn(2, heads * D, hidden, sigma=(heads * D) ** -0.5)
        per = -(-room // page)
        g = torch.Generator(device=DEV)
        g.manual_seed(3)
        self.table = torch.randperm(seqs * per, generator=g, device=DEV).int().reshape(seqs, per)
        shape = (seqs * per, kv, page, D)
        if dtype == "e4m3":
            self.pool = [torch.full(shape, 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
            self.exps = [torch.full(shape[:3], 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        else:
            self.pool, self.exps = [torch.full(shape, math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)], [None, None]
        self.desc, self.cache = cf.cache_desc(dtype, seqs * per, page, kv), cf.make_cache(*self.pool, *self.exps)
        self.rope = cf.rope_make(D, scaling="wavelength", factor=8.0, trained_len=512, magnitude=1.0)

    def project(self, x, stream=None):
        T = x.shape[0]
        qkv = torch.empty(T, self.heads + 2 * self.kv, D, dtype=torch.bfloat16, device=DEV)
        cf.ag_step(cf.layer_desc(1, 0, T, qkv.shape[1] * D, self.hidden, out_dtype="bf16"), 0, x, self.w_in, qkv, stream)
        return qkv

    def store(self, qkv, new, before, stream=None):
        """Rotates Q into a tensor of its own and stores K and V; tokens `before` .. of every sequence."""
        positions = [b + i for n, b in zip(new, before) for i in range(n)]
        seq = [s for s, n in enumerate(new) for _ in range(n)]
        slots = [int(self.host_table[s][p // self.page]) * self.page + p % self.page for s, p in zip(seq, positions)]
        self.positions, self.slots = _int(positions), _int(slots, torch.int64)
        T, h, kv, s = qkv.shape[0], self.heads, self.kv, qkv.stride()[:2]
        q = torch.empty(T, h, D, dtype=torch.bfloat16, device=DEV)
        rows = cf.cache_rows(T, h, q=s, k=s, v=s)
        cf.cache_write(self.desc, self.cache, rows, self.rope, qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], self.positions, self.slots, q, stream)
        return q

    @property
    def host_table(self):
        return self.table.tolist()

    def attend(self, q, new, ctx, stream=None):
        T = q.shape[0]
        out, lse = torch.full_like(q, -7.0), torch.full((self.heads, T), -7.0, device=DEV)
        starts, lens = _int([sum(new[:i]) for i in range(len(new) + 1)]), _int(ctx)
        desc = cf.paged_desc(len(new), self.heads, T, max(new), max(ctx), self.table.shape[1], SCALE)
        cf.attn_paged(self.desc, self.cache, desc, q, starts, lens, self.table, out, lse, stream)
        self.kept = (starts, lens)
        return out, lse

    def finish(self, out, stream=None):
        T = out.shape[0]
        y = torch.empty(T, self.hidden, device=DEV)
        cf.rs_step(cf.layer_desc(1, 0, T, self.hidden, self.heads * D), 0, out, self.w_out, None, y, stream)
        return y

    def stored(self, seq, ctx):
        """K and V of a sequence, as the cache gives them back."""
        slots = [int(self.host_table[seq][p // self.page]) * self.page + p % self.page for p in range(ctx)]
        k, v = (torch.empty(ctx, self.kv, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        cf.cache_read(self.desc, self.cache, cf.cache_rows(ctx), _int(slots, torch.int64), k, v)
        torch.cuda.synchronize()
        return k, v

    def reference(self, q, new, ctx):
        parts = []
        for s, (m, n) in enumerate(zip(new, ctx)):
            k, v = self.stored(s, n)
            a = sum(new[:s])
            full = torch.zeros(n, self.heads, D, dtype=torch.bfloat16, device=DEV)
            full[n - m:] = q[a:a + m]
            ref = prompt.definition(full, k, v, _int([0, n]), SCALE)
            parts.append((ref[0][n - m:], ref[1][:, n - m:], ref[2][n - m:], ref[3][:, n - m:]))
        return tuple(torch.cat([p[i] for p in parts], i % 2) for i in range(4))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,kv", [(8, 1), (4, 4)])
def test_prefill_chunk_and_decode(heads, kv, dtype):
    """Prompts through the projections and the cache, a chunk more, then single tokens; the last output goes through the output projection."""
    layer = Layer(heads, kv, 256, dtype, 16, 3, 520)
    ctx = [0, 0, 0]
    for step, new in enumerate(([300, 17, 1], [130, 40, 2], [1, 1, 1], [1, 1, 1])):
        x = _randn(10 + step, sum(new), layer.hidden)
        qkv = layer.project(x)
        q = layer.store(qkv, new, ctx)
        before = ctx
        ctx = [c + n for c, n in zip(ctx, new)]
        out, lse = layer.attend(q, new, ctx)
        y = layer.finish(out)
        torch.cuda.synchronize()
        # the rotation in the write is the rotation by itself
        alone = torch.empty_like(q)
        cf.rope(layer.rope, cf.rope_rows(sum(new), heads, x=qkv.stride()[:2]), qkv[:, :heads], layer.positions, alone)
        assert torch.equal(alone, q)
        want = layer.reference(q, new, ctx)
        check_paged(out, lse, want)
        if dtype == "bf16":                                                   # the cache holds the rotated K and V themselves
            turned = torch.empty(sum(new), kv, D, dtype=torch.bfloat16, device=DEV)
            cf.rope(layer.rope, cf.rope_rows(sum(new), kv, x=qkv.stride()[:2]), qkv[:, heads:heads + kv], layer.positions, turned)
            for s, n in enumerate(new):
                k, v = layer.stored(s, ctx[s])
                a = sum(new[:s])
                assert torch.equal(k[before[s]:], turned[a:a + n]) and torch.equal(v[before[s]:], qkv[a:a + n, heads + kv:])
            if step == 0:                                                     # a whole prompt: the packed kernel sees the same keys
                packed, plse = torch.empty_like(out), torch.empty_like(lse)
                s = qkv.stride()[:2]
                cf.attn_prompt(cf.prompt_desc(sum(new), 3, heads, kv, SCALE, v=s), q, turned, qkv[:, heads + kv:], _int([0, 300, 317, 318]), packed, plse)
                torch.cuda.synchronize()
                check_paged(packed, plse, want)
        exact = out.reshape(-1, heads * D).double() @ layer.w_out.double()
        size = out.reshape(-1, heads * D).double().abs() @ layer.w_out.double().abs()
        assert bool(((y.double() - exact).abs() <= 2.0 ** -24 * heads * D * size).all())


def test_training_step_between_the_projections():
    """rope -> attention -> its gradient -> the rotation's gradient, on one tensor in place of Q, K, V side by side."""
    h, kv, lens = 8, 2, [257, 64, 1, 130]
    T, at = sum(lens), _int([0, 257, 321, 322, 452])
    qkv, dout = _randn(21, T, h + 2 * kv, D), _randn(22, T, h, D)
    plain = qkv.clone()
    positions = _int([i for n in lens for i in range(n)])
    rope, s = cf.rope_make(D, 64, layout="interleaved"), qkv.stride()[:2]
    rows = cf.rope_rows(T, h + kv, x=s, o=s)
    cf.rope(rope, rows, qkv, positions, qkv)                                  # Q and K in place
    got = grad.forward_and_gradient(qkv, dout, h, kv, at, SCALE)
    ref = grad.gradient(qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], dout, at, SCALE)
    grad.check(got, ref)
    dx = torch.cat([got["dq"], got["dk"], got["dv"]], 1)
    turned = dx.clone()
    cf.rope(rope, rows, dx, positions, dx, gradient=True)
    torch.cuda.synchronize()
    for have, (want, size) in ((qkv, _turned(plain[:, :h + kv], positions, rope)), (dx, _turned(turned[:, :h + kv], positions, rope, True))):
        assert bool(((have[:, :h + kv].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size).all())
    assert torch.equal(dx[:, h + kv:], turned[:, h + kv:]) and torch.equal(qkv[:, h + kv:], plain[:, h + kv:])


def test_one_captured_decoding_step():
    """Projection, write, attention and output projection of a decoded token in one graph, replayed as the sequences grow."""
    layer = Layer(8, 1, 256, "e4m3", 32, 3, 200)
    lens = [100, 31, 64]
    x = _randn(30, sum(lens), 256)
    layer.attend(layer.store(layer.project(x), lens, [0, 0, 0]), lens, lens)
    token = _randn(31, 3, 256)
    qkv, q, out = (torch.zeros(3, n, D, dtype=torch.bfloat16, device=DEV) for n in (10, 8, 8))
    y, lse = torch.zeros(3, 256, device=DEV), torch.zeros(8, 3, device=DEV)
    positions, slots, ctx, starts = _int(lens), _int([0, 0, 0], torch.int64), _int(lens), _int([0, 1, 2, 3])
    ag, rs = cf.layer_desc(1, 0, 3, 10 * D, 256, out_dtype="bf16"), cf.layer_desc(1, 0, 3, 256, 8 * D)
    rows, paged = cf.cache_rows(3, 8, *([qkv.stride()[:2]] * 3)), cf.paged_desc(3, 8, 3, 1, 200, layer.table.shape[1], SCALE)

    def step(stream):
        cf.ag_step(ag, 0, token, layer.w_in, qkv, stream)
        cf.cache_write(layer.desc, layer.cache, rows, layer.rope, qkv[:, :8], qkv[:, 8:9], qkv[:, 9:], positions, slots, q, stream)
        cf.attn_paged(layer.desc, layer.cache, paged, q, starts, ctx, layer.table, out, lse, stream)
        cf.rs_step(rs, 0, out, layer.w_out, None, y, stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for i in range(4):
        at = [n + i for n in lens]
        positions.copy_(_int(at)), ctx.copy_(_int([n + 1 for n in at]))
        slots.copy_(_int([layer.host_table[s][n // 32] * 32 + n % 32 for s, n in enumerate(at)], torch.int64))
        token.copy_(_randn(40 + i, 3, 256))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q, out, lse, y)]
        check_paged(out, lse, layer.reference(q, [1, 1, 1], [n + 1 for n in at]))
        for t in (qkv, q, out, lse, y):
            t.fill_(-7)
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (q, out, lse, y)))


def test_two_streams_with_workspaces_of_their_own():
    """Calls that split their keys, at once on two streams, give the bits that they give alone."""
    batches = [Batch(61, 8, 1, 16, "bf16", [1, 1], [3000, 1500]), Batch(62, 8, 1, 32, "e4m3", [60], [2500])]
    xs = [grad.problem(63 + i, [900, 300], 4, 1) for i in range(2)]
    alone = [b.run() for b in batches], [grad.forward_and_gradient(x, g, 4, 1, at, SCALE) for x, g, at in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(64 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for s, w in zip(streams, spaces):
        cf.set_workspace(w, stream=s)
    try:
        torch.cuda.synchronize()
        for _ in range(3):
            got = [[], []]
            outs = [(torch.full_like(a[0], -7), torch.full_like(a[1], -7)) for a in alone[0]]
            kept = []
            torch.cuda.synchronize()
            for i, s in enumerate(streams):
                x, dout, at = xs[i]
                t = [torch.full((x.shape[0], 4, D), -7.0, dtype=torch.bfloat16, device=DEV)] + [torch.full((4, x.shape[0]), -7.0, device=DEV) for _ in range(2)]
                kept.append((t, torch.full_like(x, -7)))
            torch.cuda.synchronize()
            for i, s in enumerate(streams):
                batches[i].run(stream=s, out=outs[i][0], lse=outs[i][1])
                x, dout, at = xs[i]
                (o, lse, delta), dx = kept[i]
                st = x.stride()[:2]
                desc = cf.prompt_desc(x.shape[0], 2, 4, 1, SCALE, q=st, k=st, v=st)
                cf.attn_prompt(desc, x[:, :4], x[:, 4:5], x[:, 5:], at, o, lse, s)
                cf.attn_prompt_grad(desc, x[:, :4], x[:, 4:5], x[:, 5:], o, lse, dout, at, delta, dx[:, :4], dx[:, 4:5], dx[:, 5:], s)
            torch.cuda.synchronize()
            for i in range(2):
                assert torch.equal(outs[i][0], alone[0][i][0]) and torch.equal(outs[i][1], alone[0][i][1])
                assert torch.equal(kept[i][1], torch.cat([alone[1][i][n] for n in ("dq", "dk", "dv")], 1))
    finally:
        for s in streams:
            cf.set_workspace(None, stream=s)


@pytest.mark.parametrize("size", ["none", "small", "asked for"])
def test_workspaces(size):
    """Without a workspace, with one that fits a few splits only, and with exactly what is asked for: results within the same limits."""
    x, dout, at = grad.problem(71, [1500, 200], 8, 1)
    ref = grad.gradient(x[:, :8], x[:, 8:9], x[:, 9:], dout, at, SCALE)
    b = Batch(72, 8, 1, 16, "bf16", [1, 1], [3000, 2000])
    c = Batch(73, 8, 1, 16, "e4m3", [70], [2000])
    ask = max(cf.attn_prompt_workspace_bytes(cf.prompt_desc(1700, 2, 8, 1, SCALE)), *[
        cf.attn_paged_workspace_bytes(y.cache()[0], cf.paged_desc(len(y.new), 8, y.total, max(y.new), max(y.ctx), y.table.shape[1], SCALE)) for y in (b, c)])
    assert ask > 64 * 1024
    guard = 1 << 20
    n = dict(none=0, small=(64 << 10) + (3 << 20) + 16, **{"asked for": ask})[size]
    buf = torch.full((n + guard,), 85, dtype=torch.uint8, device=DEV)
    cf.set_workspace(buf[:n] if n else None)
    try:
        grad.check(grad.forward_and_gradient(x, dout, 8, 1, at, SCALE), ref)
        for y in (b, c):
            check_paged(*y.run(), y.definition())
        assert bool((buf[n:] == 85).all())
    finally:
        torch.cuda.synchronize()
        cf.set_workspace(WORKSPACE)


@pytest.mark.parametrize("case", [(100, 2000, 1), (70, 40, 3), (300, 0, 1), (600, 25, 1)])
def test_many_sequences(case):
    """More sequences than a wave has lanes, one of them long, decoded and packed."""
    n, long, new = case
    ctx = [new + (i * 7) % 30 for i in range(n)]
    ctx[n // 2] += long
    b = Batch(81, 8, 1, 16, "bf16", [new] * n, ctx)
    check_paged(*b.run(), b.definition())
    lens = [1 + (i * 5) % 9 for i in range(n)]
    lens[n // 3] += min(long, 900)
    x, dout, at = grad.problem(82, lens, 4, 2, 3, 2)
    ref = prompt.definition(x[:, :4], x[:, 4:6], x[:, 6:], at, SCALE)
    prompt.check(*prompt.run(x, 4, 2, at, SCALE), ref)
    grad.check(grad.forward_and_gradient(x, dout, 4, 2, at, SCALE), grad.gradient(x[:, :4], x[:, 4:6], x[:, 6:], dout, at, SCALE))


@pytest.mark.parametrize("case", [(32, 1, [2100]), (8, 1, [8300])])
def test_more_blocks_than_are_looked_at(case):
    """Above 512 blocks of a key head walks are not split; sampled rows against the definition."""
    h, kv, lens = case
    T = lens[0]
    x, dout, at = grad.problem(91, lens, h, kv)
    out, lse = prompt.run(x, h, kv, at, SCALE)
    rows = torch.tensor([0, 1, 63, 64, 1000, T - 2, T - 1], device=DEV)
    k, v = (x[:, h + i].double() for i in range(2))
    for head in (0, h - 1):
        s = x[rows, head].double() @ k.t() * SCALE
        size = (x[rows, head].double().abs() @ k.abs().t() * SCALE).amax(1)
        s = s.masked_fill(torch.arange(T, device=DEV)[None, :] > rows[:, None], -math.inf)
        p = torch.softmax(s, 1)
        limit = 2.0 ** -8 * (p @ v).abs() + (2.0 ** -7 + 2.0 ** -16 * size[:, None]) * (p @ v.abs())
        assert bool(((out[rows, head].double() - p @ v).abs() <= limit).all())
        want = torch.logsumexp(s, 1)
        assert bool(((lse[head, rows].double() - want).abs() <= 2.0 ** -17 * size + 2.0 ** -18 * (want.abs() + 1)).all())


@pytest.mark.parametrize("what", ["all", "v", "dout"])
def test_nan_throughout(what):
    """Rows whose result is not finite are computed key by key: with NaN everywhere that ends with the first key."""
    x, dout, at = grad.problem(93, [6000, 144], 4, 1)
    (x if what == "all" else x[:, 5:] if what == "v" else dout).fill_(math.nan)
    out, lse = prompt.run(x, 4, 1, at, SCALE)
    assert bool(torch.isnan(out).all()) == (what != "dout") and bool(torch.isnan(lse).all()) == (what == "all")
    got = grad.forward_and_gradient(x, dout, 4, 1, at, SCALE)
    for n in ("dq", "dk") if what == "v" else ("dq", "dk", "dv"):
        assert bool(torch.isnan(got[n]).all()), n
    for new in (1, 100):
        b = Batch(94, 4, 1, 16, "bf16", [new], [5000])
        b.pool[1].fill_(math.nan)
        assert bool(torch.isnan(b.run()[0]).all())


NONSENSE = [[5, -2 ** 31, 2 ** 31 - 1, 7, 3], [2 ** 31 - 1, -2 ** 31, 60, 0, 2 ** 31 - 1], [90, 80, 70, 60, 50], [-9, 1000, -1000, 2 ** 30, 40], [-2 ** 31] * 5]


@pytest.mark.parametrize("table", NONSENSE)
@pytest.mark.parametrize("chunk", [None, "4x1"])
def test_tables_of_nonsense_touch_nothing_outside(table, chunk, monkeypatch):
    """Starts out of order and out of range, lengths and pages likewise: the calls end, and what lies around the outputs stays as it was."""
    if chunk:
        monkeypatch.setenv("COMMFUSE_CAUSAL", chunk)
    h, kv, T = 4, 2, 100
    x, dout, _ = grad.problem(95, [T], h, kv)
    at, s = _int(table), x.stride()[:2]

    def guarded(*shape, dtype=torch.bfloat16):
        n = math.prod(shape)
        whole = torch.full((n + 8192,), -7.0, dtype=dtype, device=DEV)
        return whole, whole[4096:4096 + n].view(shape)

    def intact(*wholes):
        torch.cuda.synchronize()
        assert all(bool((w[:4096] == -7).all()) and bool((w[-4096:] == -7).all()) for w in wholes)

    (wo, out), (wl, lse), (wd, delta), (wx, dx) = guarded(T, h, D), guarded(h, T, dtype=torch.float32), guarded(h, T, dtype=torch.float32), guarded(*x.shape)
    desc = cf.prompt_desc(T, 4, h, kv, SCALE, q=s, k=s, v=s)
    cf.attn_prompt(desc, x[:, :h], x[:, h:h + kv], x[:, h + kv:], at, out, lse)
    cf.attn_prompt_grad(desc, x[:, :h], x[:, h:h + kv], x[:, h + kv:], out, lse, dout, at, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:])
    intact(wo, wl, wd, wx)
    for dtype in ("bf16", "e4m3"):
        for most in (1, 40):
            b = Batch(96, h, kv, 16, dtype, [most] * 4, [100, 90, 80, 70])
            b.starts.copy_(at), b.lens.copy_(_int(table[1:]))
            b.table.view(-1)[:5] = at
            (wo, out), (wl, lse) = guarded(b.total, h, D), guarded(h, b.total, dtype=torch.float32)
            b.run(out=out, lse=lse, max_kv=100)
            intact(wo, wl)
