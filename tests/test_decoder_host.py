"""Rotary positions, the paged cache and causal attention without a GPU: struct layouts, frequencies, and what is refused.
Every call below fails validation, or has nothing to do, before any kernel is launched."""
import ctypes
import math
from fractions import Fraction

import pytest

from paper_2604_24013_amd import binding as cf

A, B, C, D, E, F = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000      # fake, aligned, never dereferenced


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import os
    if not os.path.exists(cf.LIB_PATH):
        from paper_2604_24013_amd import build
        build.build()
    cf.load()


def status(f, *args):
    try:
        f(*args)
    except cf.CommFuseError as e:
        return e.status
    return cf.CF_OK


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(cf.RopeDesc) == 64 and cf.RopeDesc.base.offset == 24
    assert ctypes.sizeof(cf.Rope) == 1040 and cf.Rope.turn.offset == 16
    assert ctypes.sizeof(cf.RopeRows) == 48
    assert ctypes.sizeof(cf.CacheDesc) == 48 and cf.CacheDesc.n_pages.offset == 16
    assert ctypes.sizeof(cf.Cache) == 32
    assert ctypes.sizeof(cf.CacheRows) == 80 and cf.CacheRows.q_token.offset == 16


# ---- frequencies: to 2^-50 of the formula in 64 bits (powers and logarithms of 64 bits are good to a few 2^-53) --------
def _frequency(j, rot, base, scaling, factor, trained, low, high):
    f = base ** (-2.0 * j / rot)
    r = 0.0
    if scaling == "wavelength":
        r = (trained * f / (2 * math.pi) - low) / (high - low)
    elif scaling == "index":
        d = lambda t: rot * math.log(trained / (2 * math.pi * t)) / (2 * math.log(base))
        first, last = max(0, math.floor(d(high))), min(rot // 2 - 1, math.ceil(d(low)))
        r = 1 - (j - first) / max(last - first, 1e-3)
    r = min(1.0, max(0.0, r))
    return f * (r + (1 - r) / factor)


@pytest.mark.parametrize("rot", [2, 24, 64, 96, 128, 256])
@pytest.mark.parametrize("base, scaling, factor, trained, low, high", [
    (1e4, "linear", 1.0, 0, 1.0, 4.0), (1e4, "linear", 2.5, 0, 1.0, 4.0), (5e5, "wavelength", 8.0, 8192, 1.0, 4.0),
    (1e6, "index", 4.0, 32768, 1.0, 32.0), (1e4, "index", 40.0, 4096, 1.0, 32.0), (2.0, "index", 2.0, 7, 1.0, 1.1)])
def test_frequencies(rot, base, scaling, factor, trained, low, high):
    r = cf.rope_make(256, rot, "half", base=base, scaling=scaling, factor=factor, trained_len=trained, low=low, high=high, magnitude=1.5)
    assert (r.head_dim, r.rot_dim, r.layout, r.magnitude) == (256, rot, 0, 1.5)
    for j in range(rot // 2):
        turns = _frequency(j, rot, base, scaling, factor, trained, low, high) / (2 * math.pi)
        assert abs(Fraction(r.turn[j], 2 ** 64) - Fraction(turns)) <= Fraction(turns) / 2 ** 46 + Fraction(1, 2 ** 64)
    assert all(r.turn[j] == 0 for j in range(rot // 2, 128))


def test_rope_make_refusals():
    make = lambda **kw: status(lambda: cf.rope_make(**{"head_dim": 128, **kw}))
    assert make() == cf.CF_OK
    assert make(head_dim=264) == make(head_dim=0) == make(head_dim=60) == cf.CF_ERR_UNSUPPORTED
    assert make(rot_dim=130) == make(rot_dim=3) == make(rot_dim=-2) == cf.CF_ERR_INVALID_ARG
    assert make(layout=2) == make(scaling=3) == cf.CF_ERR_UNSUPPORTED
    nan = float("nan")
    for kw in (dict(base=1.0), dict(base=nan), dict(base=float("inf")), dict(factor=0.5), dict(factor=nan), dict(magnitude=0.0), dict(magnitude=nan),
               dict(scaling="wavelength"), dict(scaling="index", trained_len=4096, low=4.0, high=4.0), dict(scaling="index", trained_len=4096, low=0.0),
               dict(scaling="wavelength", trained_len=4096, high=float("inf"))):
        assert make(**kw) == cf.CF_ERR_INVALID_ARG, kw
    assert cf.load().commfuse_rope_make(None, None) == cf.CF_ERR_NULL_PTR


def test_rope_refusals():
    r = cf.rope_make(128, 128)
    call = lambda rows, x=A, pos=B, out=C, rope=r: status(cf.rope, rope, rows, x, pos, out)
    assert call(cf.rope_rows(0, 4)) == call(cf.rope_rows(7, 0)) == cf.CF_OK                      # nothing to do
    assert call(cf.rope_rows(7, 4), rope=cf.Rope()) == cf.CF_ERR_INVALID_ARG                     # never made
    assert call(cf.rope_rows(-1, 4)) == call(cf.rope_rows(7, -4)) == call(cf.rope_rows(2 ** 31, 1)) == cf.CF_ERR_INVALID_ARG
    assert call(cf.rope_rows(2 ** 30, 4)) == cf.CF_ERR_INVALID_ARG
    assert call(cf.rope_rows(7, 4, "e4m3")) == cf.CF_ERR_UNSUPPORTED
    assert call(cf.rope_rows(7, 4, x=(516, 128))) == call(cf.rope_rows(7, 4, o=(528, 132))) == cf.CF_ERR_MISALIGNED
    assert call(cf.rope_rows(7, 4, "f32", x=(518, 128))) == cf.CF_ERR_MISALIGNED
    for rows in (cf.rope_rows(7, 4, x=(64, 128)), cf.rope_rows(7, 4, o=(504, 128)), cf.rope_rows(7, 4, o=(512, 64)), cf.rope_rows(7, 4, x=(-512, 128)),
                 cf.rope_rows(7, 4, o=(128, 800))):
        assert call(rows) == cf.CF_ERR_INVALID_ARG
    assert call(cf.rope_rows(7, 4), None) == call(cf.rope_rows(7, 4), A, None) == call(cf.rope_rows(7, 4), A, B, None) == cf.CF_ERR_NULL_PTR
    assert call(cf.rope_rows(7, 4), A + 8) == call(cf.rope_rows(7, 4), A, B + 2) == call(cf.rope_rows(7, 4), A, B, C + 2) == cf.CF_ERR_MISALIGNED
    assert call(cf.rope_rows(7, 4, x=(640, 128)), A, B, A) == cf.CF_ERR_INVALID_ARG              # in place with other strides
    assert cf.load().commfuse_rope(r, None, A, B, C, 0, None) == cf.CF_ERR_NULL_PTR


def test_cache_refusals():
    r = cf.rope_make(128, 128)
    cache, rows = cf.make_cache(A, B, C, D), cf.cache_rows(5, 4)
    desc = lambda dtype="e4m3", pages=9, page=16, kv=2, dim=128, strides=(0, 0, 0): cf.cache_desc(dtype, pages, page, kv, dim, strides)
    write = lambda d=desc(), c=cache, w=rows, rope=r, q=A, k=B, v=C, pos=D, slots=E, out=F: status(cf.cache_write, d, c, w, rope, q, k, v, pos, slots, out)
    read = lambda d=desc(), c=cache, w=rows, slots=E, k=B, v=C: status(cf.cache_read, d, c, w, slots, k, v)
    none = cf.cache_rows(0, 4)
    for call in (write, read):
        assert call(w=none) == call(d=desc("bf16"), c=cf.make_cache(A, B), w=none) == cf.CF_OK
        assert call(d=desc("f32")) == call(d=desc(dim=8)) == call(d=desc(dim=264)) == call(d=desc(dim=272)) == cf.CF_ERR_UNSUPPORTED
        for bad in (desc(page=8), desc(page=48), desc(page=2048), desc(kv=0), desc(pages=-1), desc(pages=2 ** 31), desc(strides=(4096, 2048, 64)),
                    desc(strides=(4096, 1024, 128)), desc(strides=(2048, 2048, 128)), desc(strides=(4096, 2048, -128)), desc(strides=(4096, 0, 128))):
            assert call(d=bad) == cf.CF_ERR_INVALID_ARG
        assert call(d=desc(strides=(4096 + 8, 2048, 128))) == cf.CF_ERR_MISALIGNED
        assert call(d=desc("bf16", strides=(4096 + 4, 2048, 128))) == cf.CF_ERR_MISALIGNED
        assert call(d=desc(strides=(2 ** 40, 2 ** 35, 2 ** 21)), w=none) == cf.CF_ERR_UNSUPPORTED
        for bad in ((None, B, C, D), (A, None, C, D), (A, B, None, D), (A, B, C, None)):
            assert call(c=cf.make_cache(*bad)) == cf.CF_ERR_NULL_PTR
        assert call(c=cf.make_cache(A + 8, B, C, D)) == cf.CF_ERR_MISALIGNED
        assert call(w=cf.cache_rows(-1)) == call(w=cf.cache_rows(2 ** 30)) == cf.CF_ERR_INVALID_ARG
        assert call(w=cf.cache_rows(5, 4, k=(128, 128))) == call(w=cf.cache_rows(5, 4, v=(-256, 128))) == cf.CF_ERR_INVALID_ARG
        assert call(w=cf.cache_rows(5, 4, v=(260, 128))) == cf.CF_ERR_MISALIGNED
        assert call(k=None) == call(v=None) == call(slots=None) == cf.CF_ERR_NULL_PTR
        assert call(k=B + 8) == call(v=C + 2) == call(slots=E + 4) == cf.CF_ERR_MISALIGNED
    assert write(rope=cf.Rope()) == write(rope=cf.rope_make(64, 64)) == cf.CF_ERR_INVALID_ARG
    assert write(rope=cf.rope_make(128, 24)) == cf.CF_ERR_UNSUPPORTED
    assert write(rope=None) == write(pos=None) == write(out=None) == cf.CF_ERR_NULL_PTR         # Q without a rotation
    assert write(q=A + 8) == write(out=F + 2) == write(pos=D + 2) == cf.CF_ERR_MISALIGNED
    assert write(w=cf.cache_rows(5, 4, q=(256, 128))) == write(w=cf.cache_rows(5, 4, o=(256, 128))) == cf.CF_ERR_INVALID_ARG
    assert write(w=cf.cache_rows(5, -1)) == cf.CF_ERR_INVALID_ARG
    assert write(w=cf.cache_rows(5, 4, q=(640, 128)), out=A) == cf.CF_ERR_INVALID_ARG           # in place with other strides


def test_prompt_refusals():
    assert ctypes.sizeof(cf.PromptDesc) == 96 and cf.PromptDesc.q_token.offset == 24 and cf.PromptDesc.scale.offset == 88
    desc = lambda tokens=9, n=2, h=4, kv=2, scale=0.1, **kw: cf.prompt_desc(tokens, n, h, kv, scale, **kw)
    call = lambda d=desc(), q=A, k=B, v=C, at=D, out=E, lse=F: status(cf.attn_prompt, d, q, k, v, at, out, lse)
    assert call(desc(tokens=0)) == call(desc(n=0)) == cf.CF_OK
    assert call(desc(head_dim=64)) == cf.CF_ERR_UNSUPPORTED
    assert call(desc(q=(2 ** 28, 128))) == cf.CF_ERR_UNSUPPORTED
    nan = float("nan")
    for d in (desc(tokens=-1), desc(tokens=2 ** 30), desc(n=-1), desc(h=0), desc(kv=0), desc(kv=3), desc(scale=0.0), desc(scale=nan), desc(scale=-1.0),
              desc(q=(256, 128)), desc(k=(128, 128)), desc(v=(-512, 128)), desc(o=(512, 64))):
        assert call(d) == cf.CF_ERR_INVALID_ARG
    assert call(desc(q=(516, 128))) == call(desc(o=(528, 132))) == cf.CF_ERR_MISALIGNED
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(at=None), dict(out=None)):
        assert call(**kw) == cf.CF_ERR_NULL_PTR
    for kw in (dict(q=A + 8), dict(k=B + 2), dict(v=C + 4), dict(at=D + 2), dict(out=E + 8), dict(lse=F + 2)):
        assert call(**kw) == cf.CF_ERR_MISALIGNED
    assert call(out=A) == call(out=B) == call(out=C) == cf.CF_ERR_INVALID_ARG
    assert cf.load().commfuse_attn_prompt(None, A, B, C, D, E, F, None) == cf.CF_ERR_NULL_PTR
    assert cf.attn_prompt_workspace_bytes(desc(kv=3)) == cf.attn_prompt_workspace_bytes(desc(tokens=0)) == 0


def test_paged_refusals():
    assert ctypes.sizeof(cf.PagedDesc) == 64 and cf.PagedDesc.scale.offset == 20 and cf.PagedDesc.total_q.offset == 24
    pool = lambda dtype="e4m3", dim=128, kv=2: cf.cache_desc(dtype, 9, 16, kv, dim)
    cache = cf.make_cache(A, B, C, D)
    desc = lambda n=2, h=4, total=9, max_q=5, max_kv=100, pages=7, scale=0.1, **kw: cf.paged_desc(n, h, total, max_q, max_kv, pages, scale, **kw)
    call = lambda d=desc(), p=pool(), c=cache, q=A + 256, at=B, n=C, table=D, out=E, lse=F: status(cf.attn_paged, p, c, d, q, at, n, table, out, lse)
    assert call(desc(n=0)) == call(desc(total=0)) == call(desc(max_q=0)) == cf.CF_OK
    assert call(p=pool(dim=64)) == call(p=pool("f32")) == cf.CF_ERR_UNSUPPORTED
    nan = float("nan")
    for d in (desc(n=-1), desc(h=0), desc(h=3), desc(total=-1), desc(total=2 ** 30), desc(max_q=-1), desc(max_q=2 ** 30), desc(max_kv=-1), desc(max_kv=2 ** 31 - 1),
              desc(pages=-1), desc(scale=0.0), desc(scale=nan), desc(q=(256, 128)), desc(o=(-512, 128))):
        assert call(d) == cf.CF_ERR_INVALID_ARG
    assert call(desc(q=(516, 128))) == cf.CF_ERR_MISALIGNED
    for kw in (dict(q=None), dict(at=None), dict(n=None), dict(table=None), dict(out=None), dict(c=cf.make_cache(A, B))):
        assert call(**kw) == cf.CF_ERR_NULL_PTR
    for kw in (dict(q=A + 8), dict(at=B + 2), dict(n=C + 1), dict(table=D + 2), dict(out=E + 8), dict(lse=F + 2), dict(c=cf.make_cache(A, B, C + 4, D))):
        assert call(**kw) == cf.CF_ERR_MISALIGNED
    assert call(out=A) == call(out=B) == call(out=A + 256) == cf.CF_ERR_INVALID_ARG
    assert cf.load().commfuse_attn_paged(pool(), cache, None, A, B, C, D, E, F, None) == cf.CF_ERR_NULL_PTR
    assert cf.attn_paged_workspace_bytes(pool(), desc(h=3)) == cf.attn_paged_workspace_bytes(pool(), desc(n=0)) == 0


def test_prompt_gradient_refusals():
    desc = lambda tokens=9, n=2, h=4, kv=2, **kw: cf.prompt_desc(tokens, n, h, kv, 0.1, **kw)
    names = ["q", "k", "v", "out", "lse", "dout", "at", "delta", "dq", "dk", "dv"]
    good = {n: 0x10000 * (i + 1) for i, n in enumerate(names)}
    call = lambda d=desc(), **kw: status(cf.attn_prompt_grad, d, *({**good, **kw}[n] for n in names))
    assert call(desc(tokens=0)) == call(desc(n=0)) == cf.CF_OK
    assert call(desc(head_dim=64)) == cf.CF_ERR_UNSUPPORTED
    for d in (desc(tokens=-1), desc(tokens=2 ** 29), desc(kv=3), desc(q=(256, 128)), desc(o=(512, 64))):
        assert call(d) == cf.CF_ERR_INVALID_ARG
    for n in names:
        assert call(**{n: None}) == cf.CF_ERR_NULL_PTR
        assert call(**{n: good[n] + 2}) == cf.CF_ERR_MISALIGNED
    for n in ("dq", "dk", "dv"):
        for m in names:
            if m != n:
                assert call(**{n: good[m]}) == cf.CF_ERR_INVALID_ARG
