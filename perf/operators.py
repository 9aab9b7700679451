"""What the operators between a decoder layer's two projections are measured on: rotary positions, the paged cache, causal
attention over packed prompts with its gradient, and attention of new tokens over the cache.

A case is a dict of plain numbers and texts.  ``kind`` names the path:

  prompt   causal attention of packed sequences (``lens``), query heads sharing key heads: output and log-sum-exp
  train    the same forward, then its gradient: output, dQ, dK, dV
  paged    the new tokens of every sequence (``new``) over its cache (``ctx`` tokens, the new ones among them)
  cache    rotation of Q and K, K and V written into cache pages, and read back as the values that the cache now stands for
  rope     rotation of some heads of a projection's output, or its gradient

Q, K and V come as the QKV projection leaves them: side by side in one row per token.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 128                                      # features of a head
WORKSPACE_BYTES = 256 << 20                  # key splits of one launch, registered once
ROPES = {
    # base 10000, as trained
    "plain": dict(base=1e4, scaling="linear", factor=1.0, trained_len=4096, low=1.0, high=4.0, magnitude=1.0),
    # twice the trained length, positions squeezed
    "linear": dict(base=1e4, scaling="linear", factor=2.0, trained_len=4096, low=1.0, high=4.0, magnitude=1.0),
    # slow frequencies slowed down by eight, fast ones kept, a ramp by wavelength between
    "wavelength": dict(base=5e5, scaling="wavelength", factor=8.0, trained_len=8192, low=1.0, high=4.0, magnitude=1.0),
    # the ramp over the pair's index, cosines and sines enlarged
    "index": dict(base=1e6, scaling="index", factor=4.0, trained_len=32768, low=1.0, high=32.0, magnitude=0.1 * math.log(4.0) + 1.0),
}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _text(values):
    return ",".join(str(v) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def listed():
    rng = random.Random(7)
    return [
        # prefill of one 4096-token prompt, 7B shapes on 8 ranks: four heads with keys of their own
        dict(name="prompt_7b", kind="prompt", heads=4, kv=4, lens="4096"),
        # prefill of a batch of uneven prompts, one of a single token, 70B shapes: eight query heads on one key head
        dict(name="prompt_70b_packed", kind="prompt", heads=8, kv=1, lens="2809,1,517,4096,769"),
        # training on packed documents, 7B shapes
        dict(name="train_7b_packed", kind="train", heads=4, kv=4, lens="2048,1365,683"),
        # training on one long document, 70B shapes: the gradient of the key head sums over eight query heads
        dict(name="train_70b", kind="train", heads=8, kv=1, lens="4096"),
        # one user's next token: latency
        dict(name="decode_one", kind="paged", heads=8, kv=1, page=16, cache="bf16", new="1", ctx="1003"),
        # decoding 64 sequences of a serving batch, 7B shapes; two places of the batch are idle
        dict(name="decode_7b", kind="paged", heads=4, kv=4, page=16, cache="bf16", new=_text([1] * 64),
             ctx=_text([rng.randint(33, 4096) for _ in range(62)] + [0, 0])),
        # decoding eight long contexts from an 8-bit cache, 70B shapes
        dict(name="decode_70b_long", kind="paged", heads=8, kv=1, page=64, cache="e4m3", new=_text([1] * 8),
             ctx=_text([65536, 50001, 40000, 65000, 30011, 65536, 12345, 61234])),
        # chunked prefill: a thousand new tokens of three prompts over what the cache holds already
        dict(name="chunk_70b", kind="paged", heads=8, kv=1, page=32, cache="e4m3", new="1024,1024,333", ctx="8192,5003,333"),
        # a prefill's keys and values into an 8-bit cache, contexts beyond the trained length
        dict(name="cache_prefill_70b", kind="cache", heads=8, kv=1, page=64, cache="e4m3", tokens=8192, rope="wavelength", layout="half", rot=128, far=131072),
        # one step of a serving batch into a bf16 cache
        dict(name="cache_decode_7b", kind="cache", heads=4, kv=4, page=16, cache="bf16", tokens=64, rope="plain", layout="half", rot=128, far=4096),
        # training: Q and K of a projection rotated in one call
        dict(name="rope_70b", kind="rope", heads=9, tokens=8192, dtype="bf16", rope="wavelength", layout="half", rot=128, far=8192, gradient=False),
        # the gradient of a rotation of half of each head, neighbours paired, in fp32
        dict(name="rope_gradient_odd", kind="rope", heads=5, tokens=4099, dtype="f32", rope="index", layout="interleaved", rot=64, far=1000000, gradient=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cut(rng, total, pieces):
    """``total`` tokens in ``pieces`` uneven sequences of one token at the least."""
    at = sorted(rng.sample(range(1, total), pieces - 1)) if pieces > 1 else []
    return [b - a for a, b in zip([0] + at, at + [total])]


def _draw_any(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "paged", "paged", "paged", "cache", "rope"])
    c = dict(kind=kind)
    if kind != "rope":
        c["heads"], c["kv"] = rng.choice([(4, 4), (8, 1), (8, 2), (8, 8), (4, 1), (16, 2), (1, 1), (6, 2), (12, 4), (5, 1), (32, 1)])
    if kind in ("prompt", "train"):
        # (dQ and dK of a sequence of one token are differences of equal numbers: such sequences come among longer ones)
        total = _log_int(rng, 1, 8192) if kind == "prompt" else _log_int(rng, 32, 4096)
        c["lens"] = _text(_cut(rng, total, min(total if kind == "prompt" else total // 8, _log_int(rng, 1, 64))))
    elif kind == "paged":
        c["page"], c["cache"] = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"])
        if rng.random() < 0.6:                                     # decoding, now and then several tokens at once
            n, most = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
            ctx = [_log_int(rng, 1, max(16, 262144 // n)) for _ in range(n)]
            new = [min(x, rng.randint(1, most)) for x in ctx]
            if n > 4 and rng.random() < 0.5:
                ctx[-1] = 0                                        # an idle place of the batch
        else:
            n = rng.randint(1, 4)
            new = [_log_int(rng, 1, 1500) for _ in range(n)]
            ctx = [x + rng.choice([0, _log_int(rng, 1, 8192)]) for x in new]
        c["new"], c["ctx"] = _text(new), _text(ctx)
    else:
        c["tokens"] = _log_int(rng, 1, 8192)
        c["rope"], c["layout"], c["rot"] = rng.choice(sorted(ROPES)), rng.choice(["half", "interleaved"]), rng.choice([128, 128, 64, 32, 96])
        c["far"] = _log_int(rng, 1000, 1000000)
        if kind == "cache":
            c["page"], c["cache"] = rng.choice([16, 32, 64, 128, 256]), rng.choice(["bf16", "e4m3"])
        else:
            c["heads"], c["dtype"], c["gradient"] = rng.choice([1, 4, 5, 9, 10, 16]), rng.choice(["bf16", "f32"]), rng.choice([True, False])
    return c


def _plain_cost(c):
    """What the plain form's products and its largest tensors come to, in its own manner (masked places are computed)."""
    if c["kind"] in ("prompt", "train"):
        return c["heads"] * sum(_ints(c["lens"])) ** 2 * (3 if c["kind"] == "train" else 1)
    if c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        return len(new) * max(ctx) * (c["heads"] * max(new) + 2 * c["kv"] * D)
    return c["tokens"] * (c["heads"] + 2 * c.get("kv", 0)) * D


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
def work(case):
    c = case
    if c["kind"] in ("prompt", "train"):
        lens = _ints(c["lens"])
        T, pairs = sum(lens), c["heads"] * sum(n * (n + 1) // 2 for n in lens)
        qo, kv = T * c["heads"] * D * 2, T * c["kv"] * D * 2
        if c["kind"] == "prompt":
            return {"bytes": 2 * qo + 2 * kv + T * c["heads"] * 4, "flops": 4 * D * pairs}
        return {"bytes": 4 * qo + 4 * kv, "flops": 14 * D * pairs}
    if c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        pairs = sum(sum(max(0, n - q + i + 1) for i in range(q)) for q, n in zip(new, ctx))
        row = D * 2 if c["cache"] == "bf16" else D + 1
        return {"bytes": 2 * sum(ctx) * c["kv"] * row + sum(new) * c["heads"] * (D * 4 + 4), "flops": 4 * D * pairs * c["heads"]}
    if c["kind"] == "cache":
        row = D * 2 if c["cache"] == "bf16" else D + 1
        moved = c["heads"] * D * 4 + 2 * c["kv"] * (D * 2 + row + row + D * 2) + 4 + 16
        return {"bytes": c["tokens"] * moved, "flops": c["tokens"] * (c["heads"] + c["kv"]) * c["rot"] * 3}
    e = 2 if c["dtype"] == "bf16" else 4
    return {"bytes": c["tokens"] * (c["heads"] * D * 2 * e + 4), "flops": c["tokens"] * c["heads"] * c["rot"] * 3}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
class _Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=self.g)

    def qkv(self, tokens, heads, kv, dtype=torch.bfloat16):
        """A projection's output: some features of the keys are larger than others, as in trained layers."""
        x = self.normal(tokens, heads + 2 * kv, D)
        x[:, heads:heads + kv] *= torch.exp(0.5 * self.normal(kv, D))
        return x.to(dtype)

    def permutation(self, n):
        return torch.randperm(n, device=DEV, generator=self.g)


def _starts(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)


def _exponents(x):
    """The smallest e of each row with max|x| <= 448 * 2^e, from the bits of the maximum (448 = 1.75 * 2^8)."""
    bits = x.float().abs().amax(-1).view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()
    return torch.where(bits == 0, torch.zeros_like(e), e.clamp(-126, 127))


def _pow2(e):
    """2^e for e in [-126, 127], from its bits."""
    return ((e + 127) << 23).view(torch.float32)


def prepare(case, seed):
    c, mk = case, _Maker(seed)
    st = dict(case=c)
    if c["kind"] in ("prompt", "train"):
        lens = _ints(c["lens"])
        T, h, kv = sum(lens), c["heads"], c["kv"]
        x = mk.qkv(T, h, kv)
        st.update(qkv=x, q=x[:, :h], k=x[:, h:h + kv], v=x[:, h + kv:], starts=_starts(lens))
        if c["kind"] == "train":
            st["dout"] = mk.normal(T, h, D).to(torch.bfloat16)
    elif c["kind"] == "paged":
        new, ctx = _ints(c["new"]), _ints(c["ctx"])
        h, kv, page, n = c["heads"], c["kv"], c["page"], len(new)
        need = [-(-x // page) for x in ctx]
        pool, width = sum(need) + 3, max(need)
        order = mk.permutation(pool).int()
        table = torch.zeros(n, width, dtype=torch.int32, device=DEV)
        at = 0
        for i, m in enumerate(need):
            table[i, :m] = order[at:at + m]
            at += m
        x = [mk.normal(pool, kv, page, D) for _ in range(2)]
        x[0] *= torch.exp(0.5 * mk.normal(1, kv, 1, D))
        if c["cache"] == "e4m3":
            e = [_exponents(t) for t in x]
            st.update(k=(x[0] * _pow2(-e[0])[..., None]).to(torch.float8_e4m3fn), v=(x[1] * _pow2(-e[1])[..., None]).to(torch.float8_e4m3fn),
                      k_exp=(e[0] + 127).to(torch.uint8), v_exp=(e[1] + 127).to(torch.uint8))
        else:
            st.update(k=x[0].to(torch.bfloat16), v=x[1].to(torch.bfloat16), k_exp=None, v_exp=None)
        st.update(q=mk.qkv(sum(new), h, kv)[:, :h], starts=_starts(new), lens=torch.tensor(ctx, dtype=torch.int32, device=DEV), table=table)
    else:
        T, h, kv = c["tokens"], c["heads"], c.get("kv", 0)
        x = mk.qkv(T, h, kv, DTYPES[c.get("dtype", "bf16")])
        st.update(x=x, positions=torch.randint(0, c["far"], (T,), device=DEV, generator=mk.g, dtype=torch.int32))
        if c["kind"] == "cache":
            page = c["page"]
            pool = -(-T // page) + 3
            order = mk.permutation(pool)
            i = torch.arange(T, device=DEV)
            st["slots"] = order[i // page] * page + i % page
            shape, dt = (pool, kv, page, D), torch.float8_e4m3fn if c["cache"] == "e4m3" else torch.bfloat16
            st["k"], st["v"] = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV).to(dt) for _ in range(2))
            st["k_exp"], st["v_exp"] = (torch.full(shape[:3], 127, dtype=torch.uint8, device=DEV) for _ in range(2)) if c["cache"] == "e4m3" else (None, None)
    return st


# ---------------------------------------------------------------------------------------------------------------------
# one pass, plain
# ---------------------------------------------------------------------------------------------------------------------
def _by_key_head(x, kv):
    """[tokens, heads, D] -> [kv, heads / kv, tokens, D] in 32 bits"""
    T, h = x.shape[:2]
    return x.float().permute(1, 0, 2).reshape(kv, h // kv, T, D)


def _products(a, b):
    """a [kv, group, rows, n] times b [kv, n, columns]"""
    kv, g, r, n = a.shape
    return torch.matmul(a.reshape(kv, g * r, n), b.contiguous()).reshape(kv, g, r, b.shape[-1])


def _softmax(s):
    """Probabilities and log-sum-exp over the last axis; rows with nothing but -inf have probabilities of 0."""
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total), (m + torch.log(total))[..., 0]


def _plain_prompt(st):
    q, k, v, starts = st["q"], st["k"], st["v"], st["starts"]
    (T, h), kv, scale = q.shape[:2], k.shape[1], 1.0 / math.sqrt(D)
    at = torch.arange(T, device=DEV)
    seq = torch.bucketize(at, starts[1:].long(), right=True)
    hidden = (seq[:, None] != seq[None, :]) | (at[None, :] > at[:, None])
    qf, kf, vf = _by_key_head(q, kv), k.float().permute(1, 0, 2), v.float().permute(1, 0, 2)
    p, lse = _softmax((_products(qf, kf.transpose(1, 2)) * scale).masked_fill_(hidden, -math.inf))
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
    there = i[None, :] < new[:, None]                                              # [n, most]
    row = (starts[:-1, None] + i[None, :]).clamp(max=rows - 1)
    qf = q[row].float().permute(0, 2, 1, 3).reshape(n * kv, h // kv, most, D)
    key = torch.arange(width * page, device=DEV)
    seen = key[None, None, :] < (lens - new)[:, None, None] + i[None, :, None] + 1  # [n, most, keys]
    s = _products(qf, k.transpose(1, 2)) * (1.0 / math.sqrt(D))
    p, lse = _softmax(s.reshape(n, h, most, -1).masked_fill_(~seen[:, None], -math.inf))
    o = _products(p.reshape(n * kv, h // kv, most, -1), v).reshape(n, h, most, D).permute(0, 2, 1, 3)
    return dict(out=o[there].to(torch.bfloat16), lse=lse.permute(0, 2, 1)[there].t().contiguous())


def _turns(r, rot, far):
    """Frequencies of the rotated pairs in radians a position, 64 bits."""
    j = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    f = r["base"] ** (-2.0 * j / rot)
    if r["scaling"] == "linear":
        return f / r["factor"]
    if r["scaling"] == "wavelength":
        keep = ((r["trained_len"] * f / (2 * math.pi) - r["low"]) / (r["high"] - r["low"])).clamp(0, 1)
    else:
        d = [rot * math.log(r["trained_len"] / (2 * math.pi * t)) / (2 * math.log(r["base"])) for t in (r["high"], r["low"])]
        lo, hi = max(0, math.floor(d[0])), min(rot // 2 - 1, math.ceil(d[1]))
        keep = 1 - ((j - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
    return f * (keep + (1 - keep) / r["factor"])


def _rotate(x, positions, c, sign=1.0):
    """x [tokens, heads, D] rotated, in 32 bits (the angles in 64)."""
    r, rot = ROPES[c["rope"]], c["rot"]
    angle = positions.double()[:, None] * _turns(r, rot, c["far"])[None, :]
    cos, sin = ((t * r["magnitude"]).float()[:, None, :] for t in (torch.cos(angle), torch.sin(angle) * sign))
    y = x.float().clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    xa, xb = y[..., a].clone(), y[..., b].clone()
    y[..., a] = xa * cos - xb * sin
    y[..., b] = xb * cos + xa * sin
    return y


def _plain_cache(st):
    c, x, slots = st["case"], st["x"], st["slots"]
    h, kv, page = c["heads"], c["kv"], c["page"]
    turned = _rotate(x[:, :h + kv], st["positions"], c)
    out = [turned[:, :h].to(torch.bfloat16)]
    for new, pool, exps in ((turned[:, h:], st["k"], st["k_exp"]), (x[:, h + kv:].float(), st["v"], st["v_exp"])):
        p, s = slots // page, slots % page
        if exps is None:
            pool[p, :, s] = new.to(torch.bfloat16)
            out.append(pool[p, :, s])
        else:
            e = _exponents(new)
            pool.view(torch.uint8)[p, :, s] = (new * _pow2(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            exps[p, :, s] = (e + 127).to(torch.uint8)
            code = pool.view(torch.uint8)[p, :, s].view(torch.float8_e4m3fn).float()
            out.append((code * _pow2(exps[p, :, s].int() - 127)[..., None]).to(torch.bfloat16))
    return dict(q=out[0], k=out[1], v=out[2])


def _plain_rope(st):
    c, x = st["case"], st["x"]
    return _rotate(x, st["positions"], c, -1.0 if c["gradient"] else 1.0).to(x.dtype)


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
    if kind in ("prompt", "train"):
        q, k, v = st["q"], st["k"], st["v"]
        T, h, kv = q.shape[0], c["heads"], c["kv"]
        p.update(desc=cf.prompt_desc(T, st["starts"].numel() - 1, h, kv, 1.0 / math.sqrt(D), q=pair(q), k=pair(k), v=pair(v)),
                 out=empty(T, h, D), lse=empty(h, T, dtype=torch.float32))
        if kind == "train":
            g = empty(T, h + 2 * kv, D)
            p.update(dq=g[:, :h], dk=g[:, h:h + kv], dv=g[:, h + kv:], delta=empty(h, T, dtype=torch.float32))
    elif kind == "paged":
        q, (pool, kv, page, _) = st["q"], st["k"].shape
        rows, h = q.shape[:2]
        p.update(cache_desc=cf.cache_desc(c["cache"], pool, page, kv), cache=cf.make_cache(st["k"], st["v"], st["k_exp"], st["v_exp"]),
                 desc=cf.paged_desc(st["lens"].numel(), h, rows, max(_ints(c["new"])), max(_ints(c["ctx"])), st["table"].shape[1],
                                    1.0 / math.sqrt(D), q=pair(q)),
                 out=empty(rows, h, D), lse=empty(h, rows, dtype=torch.float32))
    else:
        r = ROPES[c["rope"]]
        p["rope"] = cf.rope_make(D, c["rot"], c["layout"], base=r["base"], scaling=r["scaling"], factor=r["factor"],
                                 trained_len=r["trained_len"], low=r["low"], high=r["high"], magnitude=r["magnitude"])
        x = st["x"]
        T, h = x.shape[0], c["heads"]
        if kind == "rope":
            p.update(rows=cf.rope_rows(T, h, c["dtype"], x=pair(x)), out=torch.empty_like(x))
        else:
            kv, (pool, _, page, _) = c["kv"], st["k"].shape
            p.update(cache_desc=cf.cache_desc(c["cache"], pool, page, kv), cache=cf.make_cache(st["k"], st["v"], st["k_exp"], st["v_exp"]),
                     q=x[:, :h], k=x[:, h:h + kv], v=x[:, h + kv:], q_out=empty(T, h, D), k_back=empty(T, kv, D), v_back=empty(T, kv, D))
            p.update(rows=cf.cache_rows(T, h, q=pair(x), k=pair(x), v=pair(x)), back=cf.cache_rows(T))
    return p


def _own_run(st):
    p = st.get("plan")
    if p is None:
        p = st["plan"] = _plan(st)
    cf, kind, s = p["cf"], st["case"]["kind"], torch.cuda.current_stream()
    if kind in ("prompt", "train"):
        q, k, v, out, lse = st["q"], st["k"], st["v"], p["out"], p["lse"]
        cf.attn_prompt(p["desc"], q, k, v, st["starts"], out, lse, s)
        if kind == "prompt":
            return dict(out=out, lse=lse)
        cf.attn_prompt_grad(p["desc"], q, k, v, out, lse, st["dout"], st["starts"], p["delta"], p["dq"], p["dk"], p["dv"], s)
        return dict(out=out, dq=p["dq"], dk=p["dk"], dv=p["dv"])
    if kind == "paged":
        cf.attn_paged(p["cache_desc"], p["cache"], p["desc"], st["q"], st["starts"], st["lens"], st["table"], p["out"], p["lse"], s)
        return dict(out=p["out"], lse=p["lse"])
    if kind == "cache":
        cf.cache_write(p["cache_desc"], p["cache"], p["rows"], p["rope"], p["q"], p["k"], p["v"], st["positions"], st["slots"], p["q_out"], s)
        cf.cache_read(p["cache_desc"], p["cache"], p["back"], st["slots"], p["k_back"], p["v_back"], s)
        return dict(q=p["q_out"], k=p["k_back"], v=p["v_back"])
    cf.rope(p["rope"], p["rows"], st["x"], st["positions"], p["out"], st["case"]["gradient"], s)
    return p["out"]


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    if kind in ("prompt", "train"):
        return _plain_prompt(state)
    return {"paged": _plain_paged, "cache": _plain_cache, "rope": _plain_rope}[kind](state)


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, sequence by sequence and head by head
# ---------------------------------------------------------------------------------------------------------------------
def _exact_head(q, k, v, first, do=None):
    """One head of one sequence; row i sees keys 0 .. first + i.  (out, lse, dq, dk, dv)"""
    i, j = torch.arange(q.shape[0], device=DEV)[:, None], torch.arange(k.shape[0], device=DEV)[None, :]
    s = q @ k.t() / math.sqrt(D)
    s[j > first + i] = -math.inf
    lse = torch.logsumexp(s, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=DEV)
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
            args = (q[r, h], k[r, h // g], v[r, h // g], 0)
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
    out, lse = torch.zeros_like(q), torch.full((c["heads"], q.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for i, (m, n) in enumerate(zip(_ints(c["new"]), _ints(c["ctx"]))):
        r = slice(at, at + m)
        at += m
        if n == 0:
            continue
        pages = st["table"][i, :-(-n // c["page"])].long()
        for h in range(c["kv"]):
            kv = []
            for x, e in ((st["k"], st["k_exp"]), (st["v"], st["v_exp"])):
                rows = x[:, h][pages].double() if e is None else x.view(torch.uint8)[:, h][pages].view(torch.float8_e4m3fn).double()
                if e is not None:
                    rows = torch.ldexp(rows, (e[:, h][pages].int() - 127)[..., None])
                kv.append(rows.reshape(-1, D)[:n])
            for u in range(h * g, (h + 1) * g):
                out[r, u], lse[u, r] = _exact_head(q[r, u], *kv, n - m)
    return dict(out=out, lse=lse)


def _exact_rotation(x, positions, c, sign):
    r, rot = ROPES[c["rope"]], c["rot"]
    freq = []
    for j in range(rot // 2):
        f = math.pow(r["base"], -2.0 * j / rot)
        keep = 0.0
        if r["scaling"] == "wavelength":
            keep = min(1.0, max(0.0, (r["trained_len"] * f / math.tau - r["low"]) / (r["high"] - r["low"])))
        elif r["scaling"] == "index":
            where = lambda t: rot * math.log(r["trained_len"] / (math.tau * t)) / (2.0 * math.log(r["base"]))
            lo, hi = max(0, math.floor(where(r["high"]))), min(rot // 2 - 1, math.ceil(where(r["low"])))
            keep = 1.0 - min(1.0, max(0.0, (j - lo) / max(hi - lo, 1e-3)))
        freq.append(f * keep + f * (1.0 - keep) / r["factor"])
    turn = torch.polar(torch.full((len(x), rot // 2), r["magnitude"], dtype=torch.float64, device=DEV),
                       sign * positions.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV))[:, None]
    y, z = x.double(), x[..., :rot].double()
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


def exact(case, seed):
    st, c = prepare(case, seed), case
    if c["kind"] in ("prompt", "train"):
        return _exact_prompt(st)
    if c["kind"] == "paged":
        return _exact_paged(st)
    if c["kind"] == "rope":
        return _exact_rotation(st["x"], st["positions"], c, -1.0 if c["gradient"] else 1.0)
    h, kv, x = c["heads"], c["kv"], st["x"]
    y = _exact_rotation(x[:, :h + kv], st["positions"], c, 1.0)
    return dict(q=y[:, :h], k=_exact_cached(y[:, h:], c["cache"]), v=_exact_cached(x[:, h + kv:].double(), c["cache"]))
