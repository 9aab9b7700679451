"""Normed heads on several axes and a step's tables without a GPU: struct layouts, which pair turns by which axis and how fast, and what is
refused.  Every call below fails validation, or has nothing to do, before any kernel is launched."""
import ctypes

import pytest

from paper_2604_24013_amd import binding as cf

A, B, C, D, E, F, G, H = (0x10000 * i for i in range(1, 9))          # fake, aligned, never dereferenced


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import os
    if not os.path.exists(cf.LIB_PATH):
        from paper_2604_24013_amd import build
        build.build()
    cf.load()


def status(f, *args, **kw):
    try:
        f(*args, **kw)
    except cf.CommFuseError as e:
        return e.status
    return cf.CF_OK


def test_struct_layouts_match_the_header():
    assert ctypes.sizeof(cf.AxesDesc) == 28 and cf.AxesDesc.sections.offset == 12
    assert ctypes.sizeof(cf.RopeAxes) == 1176 and cf.RopeAxes.n_axes.offset == 1040 and cf.RopeAxes.axis.offset == 1044
    assert ctypes.sizeof(cf.HeadNorm) == 16
    assert ctypes.sizeof(cf.HeadRows) == 88 and cf.HeadRows.q_token.offset == 24
    assert ctypes.sizeof(cf.TablesDesc) == 32 and cf.TablesDesc.n_pages.offset == 16
    assert ctypes.sizeof(cf.Tables) == 96


@pytest.mark.parametrize("spectrum", ["shared", "own"])
@pytest.mark.parametrize("scaling", ["linear", "wavelength", "index"])
def test_axes_and_frequencies(spectrum, scaling):
    kw = dict(base=5e5, scaling=scaling, factor=4.0, trained_len=8192, low=1.0, high=32.0, magnitude=1.5)
    for rot, sections, order in ((128, (24, 20, 20), "interleaved"), (128, (16, 24, 24), "sections"), (96, (40, 8), "sections"), (24, (3, 3, 3, 3), "interleaved"),
                                 (6, (1, 1, 1), "interleaved"), (2, (1,), "interleaved"), (64, (30, 1, 1), "interleaved")):
        r = cf.rope_axes_make(128, rot, "interleaved", sections=sections, order=order, spectrum=spectrum, **kw)
        assert (r.n_axes, r.rope.head_dim, r.rope.rot_dim, r.rope.layout, r.rope.magnitude) == (len(sections), 128, rot, 1, 1.5)
        n, want, used = len(sections), [], [0] * len(sections)
        if order == "sections":
            want = [a for a in range(n) for _ in range(sections[a])]
        else:
            for j in range(rot // 2):
                want.append(j % n if j // n < sections[j % n] else 0)
        assert list(r.axis[:rot // 2]) == want and [want.count(a) for a in range(n)] == list(sections)
        one = [cf.rope_make(128, rot if spectrum == "shared" else 2 * s, "half", **kw) for s in sections]
        for j, a in enumerate(want):
            assert r.rope.turn[j] == one[a].turn[j if spectrum == "shared" else used[a]]
            used[a] += 1
        assert not any(r.rope.turn[rot // 2:]) and not any(r.axis[rot // 2:])


def test_axes_are_refused():
    make = lambda **kw: status(cf.rope_axes_make, 128, 64, **kw)
    assert make(sections=(32,)) == cf.CF_OK
    assert make(sections=()) == cf.CF_ERR_INVALID_ARG
    assert make(sections=(8, 8, 8, 4, 4)) == cf.CF_ERR_INVALID_ARG
    assert make(sections=(16, 15)) == cf.CF_ERR_INVALID_ARG
    assert make(sections=(33, -1)) == cf.CF_ERR_INVALID_ARG
    assert make(sections=(32, 0)) == cf.CF_ERR_INVALID_ARG
    assert make(sections=(10, 22), order="interleaved") == cf.CF_ERR_INVALID_ARG
    assert make(sections=(22, 10), order="interleaved") == cf.CF_OK
    assert make(sections=(32,), order=2) == cf.CF_ERR_UNSUPPORTED
    assert make(sections=(32,), spectrum=2) == cf.CF_ERR_UNSUPPORTED
    assert make(sections=(32,), base=1.0) == cf.CF_ERR_INVALID_ARG
    lib, d, a, r = cf.load(), cf.RopeDesc(), cf.AxesDesc(), cf.RopeAxes()
    assert lib.commfuse_rope_axes_make(None, a, r) == cf.CF_ERR_INVALID_ARG          # (n_axes 0 is looked at first)
    a.n_axes, a.sections[0] = 1, 4
    assert lib.commfuse_rope_axes_make(None, a, r) == cf.CF_ERR_NULL_PTR
    assert lib.commfuse_rope_axes_make(d, None, r) == cf.CF_ERR_NULL_PTR and lib.commfuse_rope_axes_make(d, a, None) == cf.CF_ERR_NULL_PTR


def _norm_rope(rope="make", norm="make", rows=None, Q=A, K=B, wq=C, wk=D, pos=E, axis=0, qo=F, ko=G):
    rope = cf.rope_axes_make(128, sections=(32, 32)) if rope == "make" else rope
    norm = cf.head_norm(1e-6) if norm == "make" else norm
    return status(cf.norm_rope, rope, norm, rows or cf.head_rows(0, 8, 1), Q, K, wq, wk, pos, axis, qo, ko)


def test_norm_rope_is_refused():
    rows, ok = cf.head_rows, cf.CF_OK
    assert _norm_rope() == ok and _norm_rope(rows=rows(0, 0, 0)) == ok and _norm_rope(rows=rows(5, 0, 0)) == ok
    assert _norm_rope(rope=None) == ok and _norm_rope(norm=None) == ok and _norm_rope(rope=None, norm=None) == cf.CF_ERR_NULL_PTR
    assert _norm_rope(rope=cf.RopeAxes()) == cf.CF_ERR_INVALID_ARG
    bad = cf.rope_axes_make(128, sections=(32, 32))
    bad.axis[5] = 2
    assert _norm_rope(rope=bad) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(rope=cf.rope_axes_make(64)) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(norm=cf.head_norm(0.0)) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(norm=cf.head_norm(float("nan"))) == cf.CF_ERR_INVALID_ARG and _norm_rope(norm=cf.head_norm(float("inf"))) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(norm=cf.head_norm(1e-6, float("inf"))) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(norm=cf.head_norm(1e-6, 0.0, "e4m3")) == cf.CF_ERR_UNSUPPORTED
    assert _norm_rope(norm=cf.HeadNorm(0, 1e-6, 0.0, 1)) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(rows=rows(4, 8, 1, 128, "e4m3")) == cf.CF_ERR_UNSUPPORTED
    assert _norm_rope(rows=rows(4, 8, 1, 264)) == cf.CF_ERR_UNSUPPORTED and _norm_rope(rows=rows(4, 8, 1, 124)) == cf.CF_ERR_UNSUPPORTED
    assert _norm_rope(rows=rows(4, -1, 1)) == cf.CF_ERR_INVALID_ARG and _norm_rope(rows=rows(-1, 8, 1)) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(rows=rows(2 ** 31 // 8, 8, 1)) == cf.CF_ERR_INVALID_ARG
    for name in ("q", "k", "oq", "ok"):
        assert _norm_rope(rows=rows(4, 8, 8, **{name: (1024, 64)})) == cf.CF_ERR_INVALID_ARG         # heads overlap
        assert _norm_rope(rows=rows(4, 8, 8, **{name: (-1024, 128)})) == cf.CF_ERR_INVALID_ARG
        assert _norm_rope(rows=rows(4, 8, 8, **{name: (1028, 128)})) == cf.CF_ERR_MISALIGNED
        assert _norm_rope(rows=rows(4, 8, 8, 128, "f32", **{name: (1030, 128)})) == cf.CF_ERR_MISALIGNED
    some = rows(4, 8, 1)
    for name in ("Q", "K", "qo", "ko", "pos"):
        assert _norm_rope(rows=some, **{name: None}) == cf.CF_ERR_NULL_PTR, name
        assert _norm_rope(rows=some, **{name: A + 2}) == cf.CF_ERR_MISALIGNED, name
    assert _norm_rope(rows=some, wq=A + 1) == cf.CF_ERR_MISALIGNED and _norm_rope(rows=some, wk=A + 1) == cf.CF_ERR_MISALIGNED
    assert _norm_rope(rows=some, axis=3) == cf.CF_ERR_INVALID_ARG and _norm_rope(rows=some, axis=-4) == cf.CF_ERR_INVALID_ARG
    assert _norm_rope(rows=rows(4, 8, 1, oq=(2048, 128)), qo=A) == cf.CF_ERR_INVALID_ARG             # in place, other strides
    assert _norm_rope(rows=rows(4, 8, 2, ok=(2048, 128)), ko=B) == cf.CF_ERR_INVALID_ARG


def test_norm_rope_grad_is_refused():
    rope, norm, rows = cf.rope_axes_make(128), cf.head_norm(1e-6), cf.head_rows(4, 8, 1)

    def grad(rope=rope, norm=norm, rows=rows, Q=A, K=B, pos=E, gq=C, gk=D, dq=F, dk=G, dwq=H, dwk=H + 512, scratch=A):
        return status(cf.norm_rope_grad, rope, norm, rows, Q, K, None, None, pos, 0, gq, gk, dq, dk, dwq, dwk, scratch)

    assert cf.norm_rope_scratch_bytes(rows) >= 2 * 128 * 4
    for name in ("Q", "K", "pos", "gq", "gk", "dq", "dk"):
        assert grad(**{name: None}) == cf.CF_ERR_NULL_PTR, name
        assert grad(**{name: A + 2}) == cf.CF_ERR_MISALIGNED, name
    assert grad(scratch=None) == cf.CF_ERR_NULL_PTR and grad(scratch=A + 4) == cf.CF_ERR_MISALIGNED
    assert grad(dwq=H + 2) == cf.CF_ERR_MISALIGNED and grad(dwk=H) == cf.CF_ERR_INVALID_ARG
    assert grad(norm=None) == cf.CF_ERR_INVALID_ARG                  # no weights, no gradients of theirs
    assert grad(rope=None, norm=None, dwq=None, dwk=None) == cf.CF_ERR_NULL_PTR
    assert grad(rows=cf.head_rows(4, 8, 1, oq=(2048, 128)), dq=C) == cf.CF_ERR_INVALID_ARG
    assert grad(rows=cf.head_rows(0, 8, 1), dwq=None, dwk=None, scratch=None) == cf.CF_OK


def test_cache_write_norm_is_refused():
    rope, norm, cache = cf.rope_axes_make(128), cf.head_norm(1e-6), cf.make_cache(A, B)
    desc, rows = cf.cache_desc("bf16", 8, 16, 1), cf.cache_rows(4, 8)

    def write(desc=desc, rows=rows, rope=rope, norm=norm, Q=C, K=D, V=E, wq=None, pos=F, axis=0, slots=G, out=H):
        return status(cf.cache_write_norm, desc, cache, rows, rope, norm, Q, K, V, wq, None, pos, axis, slots, out)

    assert write(rows=cf.cache_rows(0, 8)) == cf.CF_OK
    for name in ("K", "V", "pos", "slots", "out"):
        assert write(**{name: None}) == cf.CF_ERR_NULL_PTR, name
        assert write(**{name: A + 2}) == cf.CF_ERR_MISALIGNED, name
    assert write(rope=None, norm=None) == cf.CF_ERR_NULL_PTR
    assert write(rope=cf.rope_axes_make(128, 24)) == cf.CF_ERR_UNSUPPORTED
    assert write(rope=cf.rope_axes_make(64)) == cf.CF_ERR_INVALID_ARG
    assert write(rope=cf.rope_axes_make(128, sections=(32, 32)), axis=2) == cf.CF_ERR_INVALID_ARG
    assert write(norm=cf.head_norm(-1.0)) == cf.CF_ERR_INVALID_ARG and write(wq=A + 1) == cf.CF_ERR_MISALIGNED
    assert write(rows=cf.cache_rows(4, 8, o=(2048, 128)), out=C) == cf.CF_ERR_INVALID_ARG
    assert write(rows=cf.cache_rows(-1, 8)) == cf.CF_ERR_INVALID_ARG and write(desc=cf.cache_desc("f32", 8, 16, 1)) == cf.CF_ERR_UNSUPPORTED


def test_step_tables_is_refused():
    names = ("held", "new_tokens", "page_table", "free_pages", "free_count", "free_left", "q_start", "kv_len", "positions", "slots")

    def step(desc=None, **kw):
        t = dict({n: 0x10000 * (i + 1) for i, n in enumerate(names)}, **kw)
        return status(cf.step_tables, desc or cf.tables_desc(4, 16, 100, 8, 64), cf.make_tables(**t))

    d = cf.tables_desc
    for name in names:
        assert step(**{name: None}) == cf.CF_ERR_NULL_PTR, name
        assert step(**{name: 0x10002}) == cf.CF_ERR_MISALIGNED, name
    assert step(slots=0x10004) == cf.CF_ERR_MISALIGNED
    assert step(back_from=0x90000) == cf.CF_ERR_NULL_PTR and step(back_to=0x90000) == cf.CF_ERR_NULL_PTR
    assert step(back_from=0x90000, back_to=0x90002) == cf.CF_ERR_MISALIGNED
    assert step(kv_len=0x10000) == cf.CF_ERR_INVALID_ARG             # over held
    for bad in (d(4, 15, 100, 8, 64), d(4, 8, 100, 8, 64), d(4, 2048, 100, 8, 64), d(-1, 16, 100, 8, 64), d(4, 16, -1, 8, 64), d(4, 16, 2 ** 31, 8, 64),
                d(4, 16, 100, -1, 64), d(4, 16, 100, 8, -1), d(4, 16, 100, 8, 2 ** 31), cf.TablesDesc(4, 16, 8, 2, 100, 64), cf.TablesDesc(4, 16, 8, -1, 100, 64)):
        assert step(bad) == cf.CF_ERR_INVALID_ARG
    assert step(d(4097, 16, 100, 8, 64)) == cf.CF_ERR_UNSUPPORTED
    lib = cf.load()
    assert lib.commfuse_step_tables(None, cf.Tables(), None) == cf.CF_ERR_NULL_PTR and lib.commfuse_step_tables(d(4, 16, 100, 8, 64), None, None) == cf.CF_ERR_NULL_PTR
