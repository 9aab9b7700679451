"""What the operators of a decoder layer with normed heads, positions on several axes and a sliding window are measured on, and the tables
that a serving step hands to them.

A case is a dict of plain numbers and texts.  ``kind`` names the path:

  tables   a serving step's page table, slots, positions and lengths from the requests' lengths; pages are taken from a stack of free
           ones, those of finished requests go back onto it first
  norm     every head of Q and K divided by its root mean square, times a weight, and rotated by positions on one to four axes, and
           the gradient of that: outputs, dQ, dK and the weights' gradients
  cache    the same on the way into the paged cache, and the values that the cache stands for read back
  prompt   causal attention of packed sequences (``lens``) in which a token sees the last ``window`` tokens, itself among them, and the first
           ``sinks`` of its sequence: output and log-sum-exp
  train    the same forward, then its gradient: output, dQ, dK, dV
  paged    the new tokens of every sequence (``new``) over its cache (``ctx`` tokens, the new ones among them), seen in the same way

Q, K and V come as the QKV projection leaves them: side by side in one row per token.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 128                                      # features of a head (attention)
EPS = 1e-6
WORKSPACE_BYTES = 256 << 20                  # what launches split their work into, registered once
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INF = math.inf


def _text(values):
    return ",".join(str(v) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def listed():
    rng = random.Random(11)
    return [
        # one step of a serving batch: every request brings a token, a few need a page, two have just finished
        dict(name="tables_decode", kind="tables", n=64, page=16, pick=1, most=4096, prompts=0, longest=1, done=2),
        # a step with prompts among decoded tokens, large batch, small pages
        dict(name="tables_prefill", kind="tables", n=512, page=16, pick=2, most=8192, prompts=24, longest=2048, done=40),
        # training, 70B shapes: text, images and video on three axes that take the pairs in turn
        dict(name="norm_70b", kind="norm", heads=8, kv=1, head=128, tokens=8192, dtype="bf16", layout="half", rot=128, base=5e5,
             sections="24,20,20", order="interleaved", spectrum="shared", offset=0.0, far=8192),
        # training in fp32 on images: height and width with a spectrum each, half of each head rotated, neighbours paired
        dict(name="norm_odd", kind="norm", heads=5, kv=2, head=128, tokens=4099, dtype="f32", layout="interleaved", rot=64, base=1e4,
             sections="16,16", order="sections", spectrum="own", offset=1.0, far=1000000),
        # a prefill's keys and values into an 8-bit cache, 70B shapes, text only
        dict(name="cache_70b", kind="cache", heads=8, kv=1, head=128, tokens=8192, page=64, cache="e4m3", layout="half", rot=128, base=5e5,
             sections="64", order="sections", spectrum="shared", offset=0.0, far=131072),
        # one step of a serving batch into a bf16 cache, 7B shapes, three axes in a row
        dict(name="cache_decode_7b", kind="cache", heads=4, kv=4, head=128, tokens=64, page=16, cache="bf16", layout="half", rot=128, base=1e6,
             sections="16,24,24", order="sections", spectrum="shared", offset=0.0, far=4096),
        # prefill of uneven long prompts, one of a single token, 70B shapes: eight query heads on one key head
        dict(name="prompt_70b_packed", kind="prompt", heads=8, kv=1, lens="9001,1,517,4096,2769", window=4096, sinks=0),
        # training on packed documents, 7B shapes, a short window
        dict(name="train_7b_packed", kind="train", heads=4, kv=4, lens="2048,1365,683", window=512, sinks=4),
        # training on one long document, 70B shapes
        dict(name="train_70b", kind="train", heads=8, kv=1, lens="8192", window=1024, sinks=16),
        # one user's next token far behind a long context: latency
        dict(name="decode_one", kind="paged", heads=8, kv=1, page=64, cache="e4m3", new="1", ctx="100003", window=4096, sinks=4),
        # decoding 64 sequences of a serving batch, 7B shapes, contexts shorter and longer than the window; two places of the batch are idle
        dict(name="decode_7b", kind="paged", heads=4, kv=4, page=16, cache="bf16", new=_text([1] * 64),
             ctx=_text([rng.randint(33, 16384) for _ in range(62)] + [0, 0]), window=2048, sinks=4),
        # chunked prefill: two thousand new tokens of three prompts over what the cache holds already
        dict(name="chunk_70b", kind="paged", heads=8, kv=1, page=32, cache="e4m3", new="1024,1024,333", ctx="8192,30003,333", window=4096, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cut(rng, total, pieces):
    """``total`` tokens in ``pieces`` uneven sequences of one token at the least."""
    at = sorted(rng.sample(range(1, total), pieces - 1)) if pieces > 1 else []
    return [b - a for a, b in zip([0] + at, at + [total])]


def _draw_sections(rng, pairs):
    """(sections, order) of one to four axes that share out the pairs."""
    n = rng.choice([1, 2, 3, 3, 4])
    if n == 1:
        return _text([pairs]), "sections"
    if rng.random() < 0.5:
        return _text(_cut(rng, pairs, n)), "sections"
    some = [rng.randint(1, pairs // n) for _ in range(n - 1)]        # axes behind the first take every n-th pair as long as they last
    return _text([pairs - sum(some)] + some), "interleaved"


def _draw_any(rng):
    kind = rng.choice(["tables", "norm", "norm", "cache", "cache", "prompt", "prompt", "train", "train", "paged", "paged", "paged"])
    c = dict(kind=kind)
    if kind == "tables":
        c["n"], c["page"], c["pick"] = _log_int(rng, 1, 512), rng.choice([16, 32, 64, 128, 256]), rng.randint(3, 1 << 30)
        c["most"], c["longest"] = _log_int(rng, 16, 8192), _log_int(rng, 1, 2048)
        c["prompts"], c["done"] = rng.randint(0, min(24, c["n"])), rng.randint(0, c["n"] // 8)
        return c
    c["heads"], c["kv"] = rng.choice([(4, 4), (8, 1), (8, 2), (8, 8), (4, 1), (16, 2), (1, 1), (6, 2), (12, 4), (5, 1), (32, 1)])
    if kind in ("norm", "cache"):
        c["head"] = rng.choice([128, 128, 128, 64, 256, 96])
        c["rot"] = rng.choice([c["head"], c["head"], c["head"] // 2])
        c["tokens"], c["far"] = _log_int(rng, 1, 8192), _log_int(rng, 1000, 1000000)
        c["layout"], c["base"] = rng.choice(["half", "interleaved"]), rng.choice([1e4, 5e5, 1e6])
        c["sections"], c["order"] = _draw_sections(rng, c["rot"] // 2)
        c["spectrum"], c["offset"] = rng.choice(["shared", "own"]), rng.choice([0.0, 0.0, 1.0])
        if kind == "cache":
            c["page"], c["cache"] = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"])
        else:
            c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        return c
    c["window"], c["sinks"] = _log_int(rng, 16, 8192), rng.choice([0, 0, 1, 4, 4, 16, 64, 130])
    if kind in ("prompt", "train"):
        # (dQ and dK of a sequence of one token are differences of equal numbers: such sequences come among longer ones)
        total = _log_int(rng, 1, 16384) if kind == "prompt" else _log_int(rng, 32, 8192)
        c["lens"] = _text(_cut(rng, total, min(total if kind == "prompt" else total // 8, _log_int(rng, 1, 64))))
    else:
        c["page"], c["cache"] = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"])
        if rng.random() < 0.6:                                       # decoding, now and then several tokens at once
            n, most = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
            ctx = [_log_int(rng, 1, max(16, 262144 // n)) for _ in range(n)]
            new = [min(x, rng.randint(1, most)) for x in ctx]
            if n > 4 and rng.random() < 0.5:
                ctx[-1] = 0                                          # an idle place of the batch
        else:
            n = rng.randint(1, 4)
            new = [_log_int(rng, 1, 1500) for _ in range(n)]
            ctx = [x + rng.choice([0, _log_int(rng, 1, 16384)]) for x in new]
        c["new"], c["ctx"] = _text(new), _text(ctx)
    return c


def _plain_cost(c):
    """What the plain form's products and its largest tensors come to, in its own manner (masked places are computed)."""
    if c["kind"] == "tables":
        return c["n"] * (c["most"] + c["longest"]) // c["page"]
    if c["kind"] in ("prompt", "train"):
        return c["heads"] * sum(_ints(c["lens"])) ** 2 * (3 if c["kind"] == "train" else 1)
    if c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        return len(new) * max(ctx) * (c["heads"] * max(new) + 2 * c["kv"] * D)
    return c["tokens"] * (c["heads"] + c["kv"]) * c["head"]


def draw(rng):
    limit = {}
    for c in listed():
        limit[c["kind"]] = max(limit.get(c["kind"], 0), _plain_cost(c))
    while True:
        c = _draw_any(rng)
        if _plain_cost(c) <= limit[c["kind"]]:
            return c


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def _pages(tokens, page):
    return -(-tokens // page)


def _requests(c):
    """(held, new, finished) of every place of the batch: what requests have in the cache, what they bring; a finished place is idle."""
    rng = random.Random(c["pick"])
    held = [rng.randint(1, c["most"]) for _ in range(c["n"])]
    new = [1] * c["n"]
    for i in rng.sample(range(c["n"]), c["prompts"]):
        held[i], new[i] = rng.choice([0, 0, held[i]]), rng.randint(1, c["longest"])
    finished = set(rng.sample(range(c["n"]), c["done"]))
    for i in finished:
        new[i] = 0
    return held, new, finished


def _pairs(c, first, rows):
    """(token, key) pairs of tokens first .. first + rows - 1 of a sequence."""
    at = np.arange(max(first, 0), first + rows, dtype=np.int64)
    return int((np.minimum(at + 1, c["window"]) + np.minimum(c["sinks"], np.maximum(0, at + 1 - c["window"]))).sum())


def work(case):
    c = case
    if c["kind"] == "tables":
        held, new, finished = _requests(c)
        taken = sum(_pages(h + m, c["page"]) - _pages(h, c["page"]) for h, m in zip(held, new))
        back = sum(_pages(held[i], c["page"]) for i in finished)
        return {"bytes": 24 * c["n"] + 8 * (taken + back) + 12 * sum(new), "flops": 8 * sum(new)}
    if c["kind"] in ("prompt", "train"):
        lens = _ints(c["lens"])
        T, pairs = sum(lens), c["heads"] * sum(_pairs(c, 0, n) for n in lens)
        qo, kv = T * c["heads"] * D * 2, T * c["kv"] * D * 2
        if c["kind"] == "prompt":
            return {"bytes": 2 * qo + 2 * kv + T * c["heads"] * 4, "flops": 4 * D * pairs}
        return {"bytes": 4 * qo + 4 * kv, "flops": 14 * D * pairs}
    if c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        pairs = sum(_pairs(c, n - q, q) for q, n in zip(new, ctx))
        keys = sum(min(n, c["window"] + q - 1) + min(c["sinks"], max(0, n - c["window"] - q + 1)) for q, n in zip(new, ctx))
        row = D * 2 if c["cache"] == "bf16" else D + 1
        return {"bytes": 2 * keys * c["kv"] * row + sum(new) * c["heads"] * (D * 4 + 4), "flops": 4 * D * pairs * c["heads"]}
    axes, rows, d = len(_ints(c["sections"])), c["heads"] + c["kv"], c["head"]
    if c["kind"] == "cache":
        row = d * 2 if c["cache"] == "bf16" else d + 1
        moved = c["heads"] * d * 4 + 2 * c["kv"] * (d * 2 + row + row + d * 2) + 4 * axes + 16
        return {"bytes": c["tokens"] * moved, "flops": c["tokens"] * rows * (4 * d + 3 * c["rot"])}
    e = 2 if c["dtype"] == "bf16" else 4
    return {"bytes": c["tokens"] * (rows * d * 5 * e + 4 * axes), "flops": c["tokens"] * rows * (17 * d + 6 * c["rot"])}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=self.g)

    def qkv(self, tokens, heads, kv, head=D, dtype=torch.bfloat16):
        """A projection's output: some features of the keys are larger than others, as in trained layers."""
        x = self.normal(tokens, heads + 2 * kv, head)
        x[:, heads:heads + kv] *= torch.exp(0.5 * self.normal(kv, head))
        return x.to(dtype)

    def permutation(self, n):
        return torch.randperm(n, device=DEV, generator=self.g)

    def uniform(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, device=DEV, generator=self.g)


def _starts(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _exponents(x):
    """The smallest e of each row with max|x| <= 448 * 2^e, from the bits of the maximum (448 = 1.75 * 2^8)."""
    bits = x.float().abs().amax(-1).view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()
    return torch.where(bits == 0, torch.zeros_like(e), e.clamp(-126, 127))


def _pow2(e):
    """2^e for e in [-126, 127], from its bits."""
    return ((e + 127) << 23).view(torch.float32)


def _prepare_tables(c, mk):
    held, new, finished = _requests(c)
    page, n = c["page"], c["n"]
    width = max(_pages(h + m, page) for h, m in zip(held, new)) + 1
    owned = [_pages(h, page) for h in held]
    pool = sum(owned) + sum(_pages(h + m, page) - o for h, m, o in zip(held, new, owned)) + 5
    order = mk.permutation(pool).int()
    table = mk.uniform(-3, pool + 3, n, width).int()                 # (what lies behind a request's pages is anything)
    count = _i32(owned)
    mask = torch.arange(width, device=DEV)[None, :] < count[:, None]
    table[mask] = order[:sum(owned)]
    free = torch.full((pool,), -1, dtype=torch.int32, device=DEV)
    free[:pool - sum(owned)] = order[sum(owned):]
    back = [owned[i] if i in finished else 0 for i in range(n)]
    return dict(held=_i32([0 if i in finished else h for i, h in enumerate(held)]), new=_i32(new), back_from=_i32([0] * n), back_to=_i32(back),
                table=table, free=free, free_count=_i32([pool - sum(owned)]), rows=_pages(sum(new), 64) * 64)


def _positions(c, mk):
    """[axes, tokens]: text counts on along all axes at once; a stretch in the middle is an image, row by row on the second and third."""
    T, axes = c["tokens"], len(_ints(c["sections"]))
    at = torch.arange(T, device=DEV) + mk.uniform(0, max(1, c["far"] - T), 1)
    p = at[None, :].repeat(axes, 1)
    a, b = T // 4, 3 * T // 4
    i = torch.arange(b - a, device=DEV)
    for axis in range(1, axes):
        p[axis, a:b] = at[a:a + 1] + (i // 32 if axis == 1 else i % 32 if axis == 2 else i % 7)
    if axes > 1:
        p[0, a:b] = at[a:a + 1]
    return p.int()


def prepare(case, seed):
    c, mk = case, _Maker(seed)
    st = dict(case=c)
    if c["kind"] == "tables":
        st.update(_prepare_tables(c, mk))
    elif c["kind"] in ("prompt", "train"):
        lens = _ints(c["lens"])
        T, h, kv = sum(lens), c["heads"], c["kv"]
        x = mk.qkv(T, h, kv)
        st.update(q=x[:, :h], k=x[:, h:h + kv], v=x[:, h + kv:], starts=_starts(lens))
        if c["kind"] == "train":
            st["dout"] = mk.normal(T, h, D).to(torch.bfloat16)
    elif c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        h, kv, page, n = c["heads"], c["kv"], c["page"], len(new)
        need = [_pages(x, page) for x in ctx]
        pool, width = sum(need) + 3, max(need)
        order = mk.permutation(pool).int()
        table = torch.zeros(n, width, dtype=torch.int32, device=DEV)
        table[torch.arange(width, device=DEV)[None, :] < _i32(need)[:, None]] = order[:sum(need)]
        x = [mk.normal(pool, kv, page, D) for _ in range(2)]
        x[0] *= torch.exp(0.5 * mk.normal(1, kv, 1, D))
        if c["cache"] == "e4m3":
            e = [_exponents(t) for t in x]
            st.update(k=(x[0] * _pow2(-e[0])[..., None]).to(torch.float8_e4m3fn), v=(x[1] * _pow2(-e[1])[..., None]).to(torch.float8_e4m3fn),
                      k_exp=(e[0] + 127).to(torch.uint8), v_exp=(e[1] + 127).to(torch.uint8))
        else:
            st.update(k=x[0].to(torch.bfloat16), v=x[1].to(torch.bfloat16), k_exp=None, v_exp=None)
        st.update(q=mk.qkv(sum(new), h, kv)[:, :h], starts=_starts(new), lens=_i32(ctx), table=table)
    else:
        T, h, kv, d = c["tokens"], c["heads"], c["kv"], c["head"]
        dt = DTYPES[c.get("dtype", "bf16")]
        x = mk.qkv(T, h, kv, d, dt)
        wq, wk = ((1.0 - c["offset"] + 0.2 * mk.normal(d)).to(dt) for _ in range(2))      # as trained: around one in all
        st.update(x=x, positions=_positions(c, mk), wq=wq, wk=wk)
        if c["kind"] == "norm":
            st["dy"] = mk.normal(T, h + kv, d).to(dt)
        else:
            page = c["page"]
            pool = _pages(T, page) + 3
            order = mk.permutation(pool)
            i = torch.arange(T, device=DEV)
            st["slots"] = order[i // page] * page + i % page
            shape, dt = (pool, kv, page, d), torch.float8_e4m3fn if c["cache"] == "e4m3" else torch.bfloat16
            st["k"], st["v"] = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV).to(dt) for _ in range(2))
            st["k_exp"], st["v_exp"] = (torch.full(shape[:3], 127, dtype=torch.uint8, device=DEV) for _ in range(2)) if c["cache"] == "e4m3" else (None, None)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# one pass, plain
# ---------------------------------------------------------------------------------------------------------------------
def _plain_tables(st):
    c, table, free = st["case"], st["table"], st["free"]
    page, (n, width), pool, rows = c["page"], table.shape, free.numel(), st["rows"]
    held, new = st["held"].long(), st["new"].long()
    q_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), torch.cumsum(new, 0)]).clamp(max=rows)
    m = q_start[1:] - q_start[:-1]
    at = torch.arange(width, device=DEV)[None, :]
    # the pages that come back, in the order of the batch
    back = (at >= st["back_from"][:, None]) & (at < st["back_to"][:, None]) & (table >= 0) & (table < pool)
    order = torch.cumsum(back.reshape(-1).long(), 0)
    count = st["free_count"].long()
    longer = torch.cat([free, free[:1]])                             # (the last place takes what does not come back)
    longer[torch.where(back.reshape(-1), count + order - 1, torch.full_like(order, pool))] = table.reshape(-1)
    free.copy_(longer[:pool])
    count = count + order[-1]
    # the pages that are taken, from the top
    take = (at >= ((held + page - 1) // page)[:, None]) & (at < ((held + m + page - 1) // page)[:, None])
    order = torch.cumsum(take.reshape(-1).long(), 0).reshape(n, width)
    src = count - order
    page_of = torch.where(src >= 0, free[src.clamp(min=0)], torch.full_like(table, -1))
    table.copy_(torch.where(take, page_of, table))
    t = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(q_start, t, right=True) - 1
    there = seq < n
    seq = seq.clamp(max=n - 1)
    pos = held[seq] + t - q_start[seq]
    number = table[seq, (pos // page).clamp(max=width - 1)].long()
    real = there & (pos // page < width) & (number >= 0) & (number < pool)
    slots = torch.where(real, number * page + pos % page, torch.full_like(pos, -1))
    return dict(table=table, free=free, free_left=(count - order[-1, -1]).int(), q_start=q_start.int(), kv_len=(held + m).int(), slots=slots,
                positions=torch.where(there, pos, torch.zeros_like(pos)).int())


def _axes(c):
    """(axis of each pair, its index among the pairs that its frequency counts, the dimension that it is relative to)"""
    pairs, s = c["rot"] // 2, _ints(c["sections"])
    axis = np.zeros(pairs, dtype=np.int64)
    if c["order"] == "sections":
        axis = np.repeat(np.arange(len(s)), s)
    else:
        for a in range(1, len(s)):
            axis[a:a + len(s) * s[a]:len(s)] = a
    if c["spectrum"] == "shared":
        return axis, np.arange(pairs), np.full(pairs, c["rot"])
    nth, dim = np.zeros(pairs, dtype=np.int64), np.zeros(pairs, dtype=np.int64)
    for a in range(len(s)):
        mine = axis == a
        nth[mine], dim[mine] = np.arange(mine.sum()), 2 * mine.sum()
    return axis, nth, dim


def _turned(x, positions, c, sign=1.0):
    """x [tokens, heads, features] rotated, in 32 bits (the angles in 64)."""
    axis, nth, dim = (torch.tensor(v, device=DEV) for v in _axes(c))
    f = c["base"] ** (-2.0 * nth.double() / dim)
    angle = positions.double()[axis].t() * f[None, :]
    cos, sin = torch.cos(angle).float()[:, None, :], (torch.sin(angle) * sign).float()[:, None, :]
    y, rot = x.clone(), c["rot"]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    xa, xb = x[..., a], x[..., b]
    y[..., a] = xa * cos - xb * sin
    y[..., b] = xb * cos + xa * sin
    return y


def _normed(x, w, offset):
    """(x over its root mean square, the weight in 32 bits, one over the root)"""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, w.float() + offset, r


def _plain_norm(st):
    c, x, h = st["case"], st["x"], st["case"]["heads"]
    out = {}
    for name, part, w, dy in (("q", x[:, :h], st["wq"], st["dy"][:, :h]), ("k", x[:, h:h + c["kv"]], st["wk"], st["dy"][:, h:])):
        n, w, r = _normed(part.float(), w, c["offset"])
        out[name] = _turned(n * w, st["positions"], c).to(x.dtype)
        g = _turned(dy.float(), st["positions"], c, -1.0)
        out["dw" + name] = (g * n).sum((0, 1))
        g = g * w
        out["d" + name] = (r * (g - n * (g * n).mean(-1, keepdim=True))).to(x.dtype)
    return out


def _plain_cache(st):
    c, x, slots = st["case"], st["x"], st["slots"]
    h, kv, page = c["heads"], c["kv"], c["page"]
    q, k = (n * w for n, w, _ in (_normed(x[:, :h].float(), st["wq"], c["offset"]), _normed(x[:, h:h + kv].float(), st["wk"], c["offset"])))
    out = [_turned(q, st["positions"], c).to(torch.bfloat16)]
    for rows, pool, exps in ((_turned(k, st["positions"], c), st["k"], st["k_exp"]), (x[:, h + kv:].float(), st["v"], st["v_exp"])):
        p, s = slots // page, slots % page
        if exps is None:
            pool[p, :, s] = rows.to(torch.bfloat16)
            out.append(pool[p, :, s])
        else:
            e = _exponents(rows)
            pool.view(torch.uint8)[p, :, s] = (rows * _pow2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            exps[p, :, s] = (e + 127).to(torch.uint8)
            code = pool.view(torch.uint8)[p, :, s].view(torch.float8_e4m3fn).float()
            out.append((code * _pow2(exps[p, :, s].int() - 127)[..., None]).to(torch.bfloat16))
    return dict(q=out[0], k=out[1], v=out[2])


def _by_key_head(x, kv):
    """[tokens, heads, D] -> [kv, heads / kv, tokens, D] in 32 bits"""
    T, h = x.shape[:2]
    return x.float().permute(1, 0, 2).reshape(kv, h // kv, T, D)


def _products(a, b):
    """a [kv, group, rows, n] times b [kv, n, columns]"""
    kv, g, r, n = a.shape
    return torch.matmul(a.reshape(kv, g * r, n), b.contiguous()).reshape(kv, g, r, b.shape[-1])


def _softmax_(s):
    """Probabilities (in place) and log-sum-exp over the last axis; rows with nothing but -inf have probabilities of 0."""
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -INF, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(torch.where(total == 0, torch.ones_like(total), total)), (m + torch.log(total))[..., 0]


def _plain_prompt(st):
    c, q, k, v, starts = st["case"], st["q"], st["k"], st["v"], st["starts"]
    (T, h), kv, scale = q.shape[:2], k.shape[1], 1.0 / math.sqrt(D)
    at = torch.arange(T, device=DEV)
    seq = torch.bucketize(at, starts[1:].long(), right=True)
    place = at - starts.long()[seq]                                  # in its sequence
    seen = (seq[:, None] == seq[None, :]) & (at[None, :] <= at[:, None])
    seen &= (at[None, :] > at[:, None] - c["window"]) | (place[None, :] < c["sinks"])
    qf, kf, vf = _by_key_head(q, kv), k.float().permute(1, 0, 2), v.float().permute(1, 0, 2)
    p, lse = _softmax_(_products(qf, kf.transpose(1, 2)).mul_(scale).masked_fill_(~seen, -INF))
    o = _products(p, vf)
    out = o.reshape(h, T, D).permute(1, 0, 2).to(torch.bfloat16).contiguous()
    if "dout" not in st:
        return dict(out=out, lse=lse.reshape(h, T))
    do = _by_key_head(st["dout"], kv)
    ds = p * (_products(do, vf.transpose(1, 2)) - (do * o).sum(-1, keepdim=True)) * scale
    dq = _products(ds, kf).reshape(h, T, D).permute(1, 0, 2)
    over = lambda a, b: torch.matmul(a.reshape(kv, -1, T).transpose(1, 2).contiguous(), b.reshape(kv, -1, D)).permute(1, 0, 2)
    return dict(out=out, dq=dq.to(torch.bfloat16), dk=over(ds, qf).to(torch.bfloat16), dv=over(p, do).to(torch.bfloat16))


def _plain_paged(st):
    q, table, lens, starts = st["q"], st["table"].long(), st["lens"].long(), st["starts"].long()
    c, (rows, h), (n, width), (_, kv, page, _) = st["case"], st["q"].shape[:2], st["table"].shape, st["k"].shape
    new, most = starts[1:] - starts[:-1], max(_ints(c["new"]))
    gathered = []
    for x, e in ((st["k"], st["k_exp"]), (st["v"], st["v_exp"])):
        x = x[table.reshape(-1)].float() if e is None else x.view(torch.uint8)[table.reshape(-1)].view(torch.float8_e4m3fn).float()
        if e is not None:
            x = x * _pow2(e[table.reshape(-1)].int() - 127)[..., None]
        gathered.append(x.reshape(n, width, kv, page, D).transpose(1, 2).reshape(n * kv, width * page, D))
    k, v = gathered
    i = torch.arange(most, device=DEV)
    there = i[None, :] < new[:, None]                                                # [n, most]
    row = (starts[:-1, None] + i[None, :]).clamp(max=rows - 1)
    qf = q[row].float().permute(0, 2, 1, 3).reshape(n * kv, h // kv, most, D)
    key = torch.arange(width * page, device=DEV)[None, None, :]
    end = (lens - new)[:, None, None] + i[None, :, None] + 1                         # [n, most, 1]
    seen = (key < end) & ((key >= end - c["window"]) | (key < c["sinks"]))
    s = _products(qf, k.transpose(1, 2)).mul_(1.0 / math.sqrt(D))
    p, lse = _softmax_(s.reshape(n, h, most, -1).masked_fill_(~seen[:, None], -INF))
    o = _products(p.reshape(n * kv, h // kv, most, -1), v).reshape(n, h, most, D).permute(0, 2, 1, 3)
    return dict(out=o[there].to(torch.bfloat16), lse=lse.permute(0, 2, 1)[there].t().contiguous())


# ---------------------------------------------------------------------------------------------------------------------
# one pass, by the framework
# ---------------------------------------------------------------------------------------------------------------------
_workspace = None


def _plan(st):
    """Descriptors, the workspace and output buffers: what a program sets up once and keeps."""
    global _workspace
    from paper_2604_24013_amd import binding as cf

    c, kind = st["case"], st["case"]["kind"]
    if _workspace is None:
        cf.load()
        _workspace = torch.empty(WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
        cf.set_workspace(_workspace, WORKSPACE_BYTES)
        torch.cuda.synchronize()
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=DEV)
    pair = lambda t: (t.stride(0), t.stride(1))
    p = dict(cf=cf)
    if kind == "tables":
        n, width = st["table"].shape
        out = dict(q_start=empty(n + 1, dtype=torch.int32), kv_len=empty(n, dtype=torch.int32), slots=empty(st["rows"], dtype=torch.int64),
                   positions=empty(st["rows"], dtype=torch.int32), free_left=empty(1, dtype=torch.int32))
        p.update(desc=cf.tables_desc(n, c["page"], st["free"].numel(), width, st["rows"]),
                 tables=cf.make_tables(held=st["held"], new_tokens=st["new"], back_from=st["back_from"], back_to=st["back_to"], page_table=st["table"],
                                       free_pages=st["free"], free_count=st["free_count"], **out),
                 out=dict(out, table=st["table"], free=st["free"]))
    elif kind in ("norm", "cache"):
        T, h, kv, d, x = c["tokens"], c["heads"], c["kv"], c["head"], st["x"]
        dt = "f32" if x.dtype == torch.float32 else "bf16"
        p.update(rope=cf.rope_axes_make(d, c["rot"], c["layout"], base=c["base"], sections=_ints(c["sections"]), order=c["order"], spectrum=c["spectrum"]),
                 norm=cf.head_norm(EPS, c["offset"], dt), q=x[:, :h], k=x[:, h:h + kv], v=x[:, h + kv:])
        if kind == "norm":
            y, g = torch.empty(T, h + kv, d, dtype=x.dtype, device=DEV), torch.empty_like(x)
            rows = cf.head_rows(T, h, kv, d, dt, q=pair(x), k=pair(x), oq=pair(y), ok=pair(y))
            p.update(rows=rows, q_out=y[:, :h], k_out=y[:, h:], dyq=st["dy"][:, :h], dyk=st["dy"][:, h:], dq=g[:, :h], dk=g[:, h:h + kv],
                     dwq=empty(d, dtype=torch.float32), dwk=empty(d, dtype=torch.float32),
                     scratch=empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8))
        else:
            pool, _, page, _ = st["k"].shape
            p.update(cache_desc=cf.cache_desc(c["cache"], pool, page, kv, d), cache=cf.make_cache(st["k"], st["v"], st["k_exp"], st["v_exp"]),
                     rows=cf.cache_rows(T, h, q=pair(x), k=pair(x), v=pair(x)), back=cf.cache_rows(T), q_out=empty(T, h, d),
                     k_back=empty(T, kv, d), v_back=empty(T, kv, d))
    elif kind in ("prompt", "train"):
        q, k, v = st["q"], st["k"], st["v"]
        T, h, kv = q.shape[0], c["heads"], c["kv"]
        p.update(desc=cf.prompt_desc(T, st["starts"].numel() - 1, h, kv, 1.0 / math.sqrt(D), q=pair(q), k=pair(k), v=pair(v)),
                 window=cf.window(c["window"], c["sinks"]), out=empty(T, h, D), lse=empty(h, T, dtype=torch.float32))
        if kind == "train":
            g = empty(T, h + 2 * kv, D)
            p.update(dq=g[:, :h], dk=g[:, h:h + kv], dv=g[:, h + kv:], delta=empty(h, T, dtype=torch.float32))
    else:
        q, (pool, kv, page, _) = st["q"], st["k"].shape
        rows, h = q.shape[:2]
        p.update(cache_desc=cf.cache_desc(c["cache"], pool, page, kv), cache=cf.make_cache(st["k"], st["v"], st["k_exp"], st["v_exp"]),
                 desc=cf.paged_desc(st["lens"].numel(), h, rows, max(_ints(c["new"])), max(_ints(c["ctx"])), st["table"].shape[1],
                                    1.0 / math.sqrt(D), q=pair(q)),
                 window=cf.window(c["window"], c["sinks"]), out=empty(rows, h, D), lse=empty(h, rows, dtype=torch.float32))
    return p


def _own_run(st):
    p = st.get("plan")
    if p is None:
        p = st["plan"] = _plan(st)
    cf, kind, s = p["cf"], st["case"]["kind"], torch.cuda.current_stream()
    if kind == "tables":
        cf.step_tables(p["desc"], p["tables"], s)
        return dict(p["out"])
    if kind == "norm":
        pos, axis = st["positions"], st["positions"].stride(0)
        cf.norm_rope(p["rope"], p["norm"], p["rows"], p["q"], p["k"], st["wq"], st["wk"], pos, axis, p["q_out"], p["k_out"], s)
        cf.norm_rope_grad(p["rope"], p["norm"], p["rows"], p["q"], p["k"], st["wq"], st["wk"], pos, axis, p["dyq"], p["dyk"], p["dq"], p["dk"],
                          p["dwq"], p["dwk"], p["scratch"], s)
        return dict(q=p["q_out"], k=p["k_out"], dq=p["dq"], dk=p["dk"], dwq=p["dwq"], dwk=p["dwk"])
    if kind == "cache":
        cf.cache_write_norm(p["cache_desc"], p["cache"], p["rows"], p["rope"], p["norm"], p["q"], p["k"], p["v"], st["wq"], st["wk"], st["positions"],
                            st["positions"].stride(0), st["slots"], p["q_out"], s)
        cf.cache_read(p["cache_desc"], p["cache"], p["back"], st["slots"], p["k_back"], p["v_back"], s)
        return dict(q=p["q_out"], k=p["k_back"], v=p["v_back"])
    if kind == "paged":
        cf.attn_paged_window(p["cache_desc"], p["cache"], p["desc"], p["window"], st["q"], st["starts"], st["lens"], st["table"], p["out"], p["lse"], s)
        return dict(out=p["out"], lse=p["lse"])
    q, k, v, out, lse = st["q"], st["k"], st["v"], p["out"], p["lse"]
    cf.attn_prompt_window(p["desc"], p["window"], q, k, v, st["starts"], out, lse, s)
    if kind == "prompt":
        return dict(out=out, lse=lse)
    cf.attn_prompt_window_grad(p["desc"], p["window"], q, k, v, out, lse, st["dout"], st["starts"], p["delta"], p["dq"], p["dk"], p["dv"], s)
    return dict(out=out, dq=p["dq"], dk=p["dk"], dv=p["dv"])


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    return {"tables": _plain_tables, "norm": _plain_norm, "cache": _plain_cache, "prompt": _plain_prompt, "train": _plain_prompt,
            "paged": _plain_paged}[kind](state)


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits: request by request, sequence by sequence and head by head
# ---------------------------------------------------------------------------------------------------------------------
def _exact_tables(st):
    page, rows = st["case"]["page"], st["rows"]
    held, new, b0, b1, free = (st[x].tolist() for x in ("held", "new", "back_from", "back_to", "free"))
    table, count = st["table"].cpu().numpy().copy(), int(st["free_count"])
    pool = len(free)
    for s in range(len(held)):
        for x in table[s, b0[s]:b1[s]]:
            if 0 <= x < pool:
                free[count] = int(x)
                count += 1
    q_start, kv_len, slots, positions = [0], [], [-1] * rows, [0] * rows
    for s, (have, m) in enumerate(zip(held, new)):
        m = min(m, rows - q_start[-1])
        for i in range(_pages(have, page), min(_pages(have + m, page), table.shape[1])):
            count -= 1
            table[s, i] = free[count] if count >= 0 else -1
        for i in range(m):
            at = have + i
            number = int(table[s, at // page]) if at // page < table.shape[1] else -1
            positions[q_start[-1] + i] = at
            if 0 <= number < pool:
                slots[q_start[-1] + i] = number * page + at % page
        q_start.append(q_start[-1] + m)
        kv_len.append(have + m)
    return dict(table=torch.from_numpy(table), free=_i32(free), free_left=_i32([count]), q_start=_i32(q_start), kv_len=_i32(kv_len),
                slots=torch.tensor(slots), positions=_i32(positions))


def _exact_angles(positions, c):
    s, pairs, n = _ints(c["sections"]), c["rot"] // 2, len(_ints(c["sections"]))
    used, columns = [0] * n, []
    for j in range(pairs):
        if c["order"] == "sections":
            a = next(a for a in range(n) if j < sum(s[:a + 1]))
        else:
            a = j % n if j < n * s[j % n] else 0
        mine = pairs if c["spectrum"] == "shared" else s[a]
        f = math.pow(c["base"], -(j if c["spectrum"] == "shared" else used[a]) / mine)
        used[a] += 1
        columns.append(positions[a].double() * f)
    return torch.stack(columns, 1)                                   # [tokens, pairs]


def _exact_turn(x, angle, c):
    """x [tokens, heads, features] by complex numbers; a negative angle turns back."""
    y, z, rot = x.clone(), x[..., :c["rot"]], c["rot"]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    pairs = torch.stack([z[..., :rot // 2], z[..., rot // 2:]], -1) if c["layout"] == "half" else z.reshape(*z.shape[:2], -1, 2)
    w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y[..., :rot] = torch.cat([w[..., 0], w[..., 1]], -1) if c["layout"] == "half" else w.reshape(*z.shape)
    return y


def _exact_cached(x, dtype):
    """The values a cache stands for: rounded to bf16, or to e4m3 (four significant bits, steps of 2^-9 at the least) over 2^e."""
    if dtype == "bf16":
        return x.to(torch.bfloat16).double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(top == 0, torch.zeros_like(e), e)
    z = torch.ldexp(x, -e)
    step = torch.ldexp(torch.ones_like(z), torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.ldexp(torch.round(z / step) * step, e)


def _exact_heads(st):
    c, x, h = st["case"], st["x"].double(), st["case"]["heads"]
    angle, out = _exact_angles(st["positions"], c), {}
    for name, lo, hi, w in (("q", 0, h, st["wq"]), ("k", h, h + c["kv"], st["wk"])):
        part, w = x[:, lo:hi], w.double() + c["offset"]
        root = torch.sqrt(part.pow(2).sum(-1, keepdim=True) / c["head"] + EPS)
        out[name] = _exact_turn(part / root * w, angle, c)
        if c["kind"] == "norm":                                      # the derivative of x / root, term by term
            g = _exact_turn(st["dy"][:, lo:hi].double(), -angle, c)
            out["dw" + name] = torch.einsum("thd,thd->d", g, part / root)
            out["d" + name] = g * w / root - part * (g * w * part).sum(-1, keepdim=True) / (c["head"] * root ** 3)
    if c["kind"] == "norm":
        return out
    return dict(q=out["q"], k=_exact_cached(out["k"], c["cache"]), v=_exact_cached(x[:, h + c["kv"]:], c["cache"]))


def _exact_head(c, q, k, v, first, do=None):
    """One head of one sequence; row i is at place first + i.  (out, lse, dq, dk, dv)"""
    i, j = torch.arange(first, first + q.shape[0], device=DEV)[:, None], torch.arange(k.shape[0], device=DEV)[None, :]
    s = q @ k.t() / math.sqrt(D)
    s[(j > i) | ((i - j >= c["window"]) & (j >= c["sinks"]))] = -INF
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -INF, dtype=torch.float64, device=DEV)
    p = torch.exp(s - torch.nan_to_num(lse, neginf=0.0)[:, None])
    out = p @ v
    if do is None:
        return out, lse
    ds = p * (do @ v.t() - (do * out).sum(1)[:, None]) / math.sqrt(D)
    return out, lse, ds @ k, ds.t() @ q, p.t() @ do


def _exact_prompt(st):
    c = st["case"]
    q, k, v = (st[x].double() for x in "qkv")
    g = c["heads"] // c["kv"]
    out, lse = torch.zeros_like(q), torch.zeros(c["heads"], q.shape[0], dtype=torch.float64, device=DEV)
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    at = 0
    for n in _ints(c["lens"]):
        r = slice(at, at + n)
        for h in range(c["heads"]):
            args = (c, q[r, h], k[r, h // g], v[r, h // g], 0)
            if c["kind"] == "prompt":
                out[r, h], lse[h, r] = _exact_head(*args)
            else:
                out[r, h], _, dq[r, h], a, b = _exact_head(*args, st["dout"][r, h].double())
                dk[r, h // g] += a
                dv[r, h // g] += b
        at += n
    return dict(out=out, lse=lse) if c["kind"] == "prompt" else dict(out=out, dq=dq, dk=dk, dv=dv)


def _exact_paged(st):
    c = st["case"]
    g = c["heads"] // c["kv"]
    q = st["q"].double()
    out, lse = torch.zeros_like(q), torch.full((c["heads"], q.shape[0]), -INF, dtype=torch.float64, device=DEV)
    at = 0
    for i, (m, n) in enumerate(zip(_ints(c["new"]), _ints(c["ctx"]))):
        r = slice(at, at + m)
        at += m
        if n == 0:
            continue
        pages = st["table"][i, :_pages(n, c["page"])].long()
        for h in range(c["kv"]):
            kv = []
            for x, e in ((st["k"], st["k_exp"]), (st["v"], st["v_exp"])):
                rows = x[:, h][pages].double() if e is None else x.view(torch.uint8)[:, h][pages].view(torch.float8_e4m3fn).double()
                if e is not None:
                    rows = torch.ldexp(rows, (e[:, h][pages].int() - 127)[..., None])
                kv.append(rows.reshape(-1, D)[:n])
            for u in range(h * g, (h + 1) * g):
                out[r, u], lse[u, r] = _exact_head(c, q[r, u], *kv, n - m)
    return dict(out=out, lse=lse)


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    return {"tables": _exact_tables, "norm": _exact_heads, "cache": _exact_heads, "prompt": _exact_prompt, "train": _exact_prompt,
            "paged": _exact_paged}[kind](st)
