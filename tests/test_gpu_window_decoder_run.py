"""Normed heads, positions on several axes, the step's tables, the paged cache and windowed attention one after the other, as a serving loop and a
training step use them.  Needs an MI355X: ``-m gpu``.  Tolerances: those of the single operators' tests."""
import math
import os
import random

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_paged import check as check_attention
from tests.test_gpu_norm_rope import _backward, _close, _forward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
SCALE = 1 / math.sqrt(D)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(ws)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Server:
    """A batch of `places` requests over one layer: device tables that the step's call fills, and beside it what every request has cached."""

    def __init__(self, seed, places, heads, kv, page, dtype, window, sinks, pages, width, rows):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.places, self.heads, self.kv, self.page, self.dtype, self.window, self.sinks = places, heads, kv, page, dtype, window, sinks
        self.pages, self.width, self.rows = pages, width, rows
        self.rope = cf.rope_axes_make(D, D, base=5e5, sections=(24, 20, 20), order="interleaved")
        self.norm = cf.head_norm(1e-6)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=self.g, device=DEV)).bfloat16() for _ in range(2))
        t = torch.bfloat16 if dtype == "bf16" else torch.uint8
        self.pool = [torch.full((pages, kv, page, D), 127 if dtype == "e4m3" else math.nan, device=DEV).to(t) for _ in range(2)]      # (NaN in both)
        self.exps = [torch.full((pages, kv, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.desc, self.cache = cf.cache_desc(dtype, pages, page, kv), cf.make_cache(*self.pool, *self.exps)
        free = torch.randperm(pages, generator=self.g, device=DEV).int()
        self.t = dict(held=_i32([0] * places), new_tokens=_i32([0] * places), back_from=_i32([0] * places), back_to=_i32([0] * places),
                      page_table=torch.full((places, width), -1, dtype=torch.int32, device=DEV), free_pages=free, free_count=_i32([pages]),
                      q_start=_i32([0] * (places + 1)), kv_len=_i32([0] * places), positions=_i32([0] * rows),
                      slots=torch.zeros(rows, dtype=torch.int64, device=DEV))
        self.t["free_left"] = self.t["free_count"]
        self.tables, self.tdesc = cf.make_tables(**self.t), cf.tables_desc(places, page, pages, width, rows, clear_back=True)
        self.x = torch.zeros(rows, heads + 2 * kv, D, dtype=torch.bfloat16, device=DEV)
        self.q = torch.zeros(rows, heads, D, dtype=torch.bfloat16, device=DEV)
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(heads, rows, device=DEV)
        self.held, self.seen = [0] * places, [[] for _ in range(places)]

    def step(self, max_q, stream=None):
        """What the program enqueues: tables, cache, attention."""
        h, kv, x = self.heads, self.kv, self.x
        s = x.stride()[:2]
        cf.step_tables(self.tdesc, self.tables, stream)
        cf.cache_write_norm(self.desc, self.cache, cf.cache_rows(self.rows, h, q=s, k=s, v=s), self.rope, self.norm, x[:, :h], x[:, h:h + kv], x[:, h + kv:],
                            self.wq, self.wk, self.t["positions"], 0, self.t["slots"], self.q, stream)
        paged = cf.paged_desc(self.places, h, self.rows, max_q, self.width * self.page, self.width, SCALE)
        cf.attn_paged_window(self.desc, self.cache, paged, cf.window(self.window, self.sinks), self.q, self.t["q_start"], self.t["kv_len"], self.t["page_table"],
                             self.out, self.lse, stream)

    def prepare(self, new, finished=()):
        """The lengths of a step; pages of finished requests go back, and those that have left a window."""
        back = [(0, 0)] * self.places
        for s in range(self.places):
            if s in finished:
                back[s] = (0, -(-self.held[s] // self.page))
                self.held[s], self.seen[s] = 0, []
            else:                                                    # pages in front of the next token's window (what went back before is -1 by now)
                back[s] = (-(-self.sinks // self.page), (self.held[s] + 1 - self.window) // self.page)
        self.t["held"].copy_(_i32(self.held))
        self.t["new_tokens"].copy_(_i32(new))
        self.t["back_from"].copy_(_i32([a for a, _ in back]))
        self.t["back_to"].copy_(_i32([b for _, b in back]))
        self.x.copy_(torch.randn(self.x.shape, generator=self.g, device=DEV))
        self.out.fill_(-7), self.lse.fill_(-7)

    def check(self, new):
        torch.cuda.synchronize()
        h, kv, g = self.heads, self.kv, self.heads // self.kv
        starts, total = self.t["q_start"].tolist(), sum(new)
        assert starts == [sum(new[:i]) for i in range(self.places + 1)] and int(self.t["free_left"]) >= 0
        assert bool((self.t["slots"][:total] >= 0).all()) and bool((self.t["slots"][total:] == -1).all())
        # q as the operator alone has it, K and V as the cache stands for them
        s = self.x.stride()[:2]
        q, k = torch.empty_like(self.q), torch.empty(self.rows, kv, D, dtype=torch.bfloat16, device=DEV)
        cf.norm_rope(self.rope, self.norm, cf.head_rows(self.rows, h, kv, D, q=s, k=s), self.x[:, :h], self.x[:, h:h + kv], self.wq, self.wk, self.t["positions"], 0, q, k)
        back = torch.zeros(2, self.rows, kv, D, dtype=torch.bfloat16, device=DEV)
        cf.cache_read(self.desc, self.cache, cf.cache_rows(self.rows), self.t["slots"], back[0], back[1])
        torch.cuda.synchronize()
        assert torch.equal(q[:total], self.q[:total])
        if self.dtype == "bf16":
            assert torch.equal(back[0][:total], k[:total]) and torch.equal(back[1][:total], self.x[:total, h + kv:])
        want, wlse, mean, size = (torch.full(sh, math.nan, dtype=torch.float64, device=DEV) for sh in ((self.rows, h, D), (h, self.rows), (self.rows, h, D), (h, self.rows)))
        for s in range(self.places):
            a, m = starts[s], new[s]
            positions = self.t["positions"][a:a + m].tolist()
            assert positions == list(range(self.held[s], self.held[s] + m))
            self.seen[s].append(back[:, a:a + m].double())
            self.held[s] += m
            if m == 0:
                continue
            kk, vv = torch.cat(self.seen[s], 1)
            n = kk.shape[0]
            j, i = torch.arange(n, device=DEV)[None, :], n - m + torch.arange(m, device=DEV)[:, None]
            hidden = (j > i) | ((j <= i - self.window) & (j >= self.sinks))
            for u in range(h):
                qq = self.q[a:a + m, u].double()
                sc = (qq @ kk[:, u // g].t() * SCALE).masked_fill(hidden, -math.inf)
                p = torch.softmax(sc, 1)
                wlse[u, a:a + m], want[a:a + m, u], mean[a:a + m, u] = torch.logsumexp(sc, 1), p @ vv[:, u // g], p @ vv[:, u // g].abs()
                size[u, a:a + m] = (qq.abs() @ kk[:, u // g].abs().t() * SCALE).masked_fill(hidden, 0).amax(1)
        check_attention(self.out, self.lse, (want, wlse, mean, size))


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads, kv", [(8, 1), (4, 4)])
def test_serving_loop(heads, kv, dtype):
    """Prompts, chunks, decoded tokens, requests that end and places that are taken again, with fewer pages than all tokens would need."""
    rng = random.Random(heads)
    places = 6
    s = Server(3, places, heads, kv, 16, dtype, 60, 4, pages=64, width=40, rows=320)
    done = set()
    for step in range(20):
        new = []
        finished = {i for i in range(places) if s.held[i] > 120}
        for i in range(places):
            if i in finished or rng.random() < 0.15:
                new.append(0)
            elif s.held[i] == 0:
                new.append(rng.randint(1, 90))
            else:
                new.append(rng.choice([1, 1, 1, 3, 40]))
        while sum(new) > 320:
            new[new.index(max(new))] = 1
        done |= finished
        s.prepare(new, finished)
        s.step(max(max(new), 1))
        s.check(new)
    assert done                                                      # (places were given up, and used again)


def test_captured_decoding_steps():
    """One captured step, replayed with other lengths: every request brings up to two tokens, pages are taken and given back on the way."""
    places = 5
    s = Server(9, places, 8, 1, 16, "e4m3", 40, 2, pages=48, width=24, rows=16)
    prompt = [30, 1, 57, 16, 2]
    for i in range(places):                                          # the prompts, a few tokens at a time
        for at in range(0, prompt[i], 16):
            new = [min(16, prompt[i] - at) if j == i else 0 for j in range(places)]
            s.prepare(new)
            s.step(16)
            s.check(new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = {n: s.t[n].clone() for n in ("page_table", "free_pages", "free_count")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.step(2, side)
    for n, t in state.items():
        s.t[n].copy_(t)
    for step in range(12):
        new = [(1, 2, 1, 0, 1)[(i + step) % 5] for i in range(places)]
        s.prepare(new)
        graph.replay()
        s.check(new)


def test_training_step():
    """Norm and rotation, windowed attention and both gradients, against the formulas in 64 bits.  What the attention takes and gives is rounded to bf16
    (2^-8), and its gradients are off as its own test says, so that the gradients of x are compared with the formula applied to what arrived there, and
    those of the attention with its formula applied to the rounded operands."""
    from tests.test_gpu_attn_window import check_grad, definition
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    T, h, kv, window, sinks = 500, 4, 2, 90, 3
    lens = [310, 1, 189]
    at = _i32([0, 310, 311, 500])
    x = torch.randn(T, h + 2 * kv, D, generator=g, device=DEV).bfloat16()
    w = (1 + 0.2 * torch.randn(2, D, generator=g, device=DEV)).bfloat16()
    dout = torch.randn(T, h, D, generator=g, device=DEV).bfloat16()
    pos = torch.stack([torch.arange(T, device=DEV)] * 3).int()
    pos[1, 100:200] += 7
    rope, norm = cf.rope_axes_make(D, D, sections=(24, 20, 20), order="interleaved"), cf.head_norm(1e-6)
    y = x.clone()                                                    # q and k are normed and rotated in place, v stays
    s = x.stride()[:2]
    rows = cf.head_rows(T, h, kv, D, q=s, k=s, oq=s, ok=s)
    q, k, v = (slice(0, h), slice(h, h + kv), slice(h + kv, h + 2 * kv))
    cf.norm_rope(rope, norm, rows, y[:, q], y[:, k], w[0], w[1], pos, T, y[:, q], y[:, k])
    desc, win = cf.prompt_desc(T, 3, h, kv, SCALE, q=s, k=s, v=s), cf.window(window, sinks)
    out, lse, delta = torch.empty(T, h, D, dtype=torch.bfloat16, device=DEV), torch.empty(h, T, device=DEV), torch.empty(h, T, device=DEV)
    dy, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(2, D, device=DEV)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    cf.attn_prompt_window(desc, win, y[:, q], y[:, k], y[:, v], at, out, lse)
    cf.attn_prompt_window_grad(desc, win, y[:, q], y[:, k], y[:, v], out, lse, dout, at, delta, dy[:, q], dy[:, k], dy[:, v])
    cf.norm_rope_grad(rope, norm, rows, x[:, q], x[:, k], w[0], w[1], pos, T, dy[:, q], dy[:, k], dx[:, q], dx[:, k], dw[0], dw[1], scratch)
    torch.cuda.synchronize()
    for part, wt in ((q, w[0]), (k, w[1])):
        want, size = _forward(x[:, part], wt, 0.0, 1e-6, pos, rope)
        assert _close(y[:, part], want, "bf16", 2.0 ** -18 * size)
    ref, gref = definition(y, h, kv, at, SCALE, window, sinks, dout)
    check_attention(out, lse, ref)
    check_grad(dict(dq=dy[:, q], dk=dy[:, k], dv=dy[:, v]), gref)
    for part, wt, dwt in ((q, w[0], dw[0]), (k, w[1], dw[1])):
        want, slack, want_w, slack_w = _backward(x[:, part], wt, 0.0, 1e-6, pos, rope, dy[:, part])
        assert _close(dx[:, part], want, "bf16", 2.0 ** -16 * slack)
        assert bool(((dwt.double() - want_w).abs() <= 2.0 ** -15 * slack_w).all())


def test_two_streams():
    """Two requests' batches on two streams at once, with a workspace each: the bits of one after the other."""
    servers = [Server(20 + i, 3, 8, 1, 16, "bf16", 50, 4, pages=80, width=40, rows=256) for i in range(2)]
    new = [[200, 5, 40], [1, 120, 60]]
    for s, n in zip(servers, new):
        s.prepare(n)
    torch.cuda.synchronize()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.empty(64 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]
    for st, ws in zip(streams, spaces):
        cf.set_workspace(ws, 0, st)
    try:
        for s, st in zip(servers, streams):
            s.step(200, st)
        torch.cuda.synchronize()
        for s, n in zip(servers, new):
            s.check(n)
    finally:
        for st in streams:
            cf.set_workspace(None, 0, st)
