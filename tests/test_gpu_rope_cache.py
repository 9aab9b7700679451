"""Rotary positions and the paged cache on the GPU against plain forms in 64 bits.  Needs an MI355X: ``-m gpu``.

Tolerances.  A rotated value y = m (x_a cos - x_b sin) is computed in fp32 from an angle of at most an eighth of a turn rounded to fp32
(off by 2^-23.3 rad at most), cosines good to a few units of 2^-24 (taken as 2^-22) and three roundings of 2^-24 of the
products: under 2^-20 m (|x_a| + |x_b|) in all.  Then it is rounded to the type: 2^-24 |y| (fp32), 2^-8 |y| (bf16), to e4m3 2^-4 |y|
and half of the smallest step, 2^-10 2^e.  What is not rotated is copied, so equal; codes of unrotated rows are equal to those of the
definition."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    yield
    torch.cuda.synchronize()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _turned(x, positions, rope, gradient=False):
    """(y in 64 bits, |x_a| + |x_b| of each value's pair)"""
    rot, x = rope.rot_dim, x.double()
    turn = torch.tensor([rope.turn[j] / 2.0 ** 64 for j in range(rot // 2)], dtype=torch.float64, device=DEV)
    t = positions.double()[:, None] * turn
    angle = (t - t.round())[:, None, :] * (2 * math.pi)
    c, s = torch.cos(angle) * rope.magnitude, torch.sin(angle) * rope.magnitude * (-1 if gradient else 1)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if rope.layout == cf.CF_ROPE_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = rope.magnitude * (x[..., a].abs() + x[..., b].abs())
    return y, size


def _positions(g, n, far):
    p = torch.randint(-far, far, (n,), generator=g, device=DEV, dtype=torch.int32)
    p[0] = 0
    p[-1] = far - 1
    return p


SHAPES = [  # tokens, heads, head_dim, rot_dim
    (1, 1, 128, 128), (3, 5, 128, 64), (64, 9, 128, 96), (257, 3, 64, 64), (33, 2, 256, 256), (17, 4, 80, 32), (9, 2, 96, 24), (5, 3, 8, 2),
    (70, 2, 128, 126), (2049, 10, 128, 128), (11, 3, 72, 72)]


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rope(shape, dtype, layout, gradient):
    n, h, d, rot = shape
    g = _gen(n * 1000 + rot)
    rope = cf.rope_make(d, rot, layout, base=5e5, scaling="wavelength", factor=8.0, trained_len=8192, magnitude=1.25)
    pos = _positions(g, n, 2 ** 31 - 1 if n % 2 else 100000)
    wide = _normal(g, n, h + 2, d).to(TYPES[dtype])                  # the heads lie inside a wider row
    x = wide[:, 1:1 + h]
    out = torch.full((n, h, d), float("nan"), dtype=TYPES[dtype], device=DEV)
    cf.rope(rope, cf.rope_rows(n, h, dtype, x=x.stride()[:2]), x, pos, out, gradient)
    torch.cuda.synchronize()
    y, size = _turned(x, pos, rope, gradient)
    assert torch.equal(out[..., rot:], x[..., rot:])
    assert bool(((out.double() - y).abs() <= HALF_STEP[dtype] * y.abs() + 2.0 ** -20 * size).all())
    # in place, heads outermost
    first = x.transpose(0, 1).clone(memory_format=torch.contiguous_format)
    keep = wide.clone()
    cf.rope(rope, cf.rope_rows(n, h, dtype, x=(d, n * d), o=(d, n * d)), first, pos, first, gradient)
    torch.cuda.synchronize()
    assert torch.equal(first.transpose(0, 1), out) and torch.equal(wide, keep)


def test_rope_gradient_is_the_transposed_rotation():
    """<R x, g> = <x, R' g>, and the directional difference of the loss sum(R x * g) along v is <R' g, v> (R is linear)."""
    g = _gen(5)
    rope = cf.rope_make(128, 64, "interleaved", base=1e4, magnitude=1.5)
    n, h = 129, 3
    pos = _positions(g, n, 1 << 20)
    x, go, v = (_normal(g, n, h, 128) for _ in range(3))
    rows, out = cf.rope_rows(n, h, "f32"), torch.empty(4, n, h, 128, device=DEV)
    cf.rope(rope, rows, x, pos, out[0])
    cf.rope(rope, rows, go, pos, out[1], True)
    cf.rope(rope, rows, x + 0.5 * v, pos, out[2])
    cf.rope(rope, rows, x - 0.5 * v, pos, out[3])
    torch.cuda.synchronize()
    dot = lambda a, b: float((a.double() * b.double()).sum())
    # n h 128 products of values of order 1, each off by 2^-20 of the pair's size
    slack = 2.0 ** -20 * 4 * float((x.abs().double() * go.abs().double()).sum() + (v.abs().double() * go.abs().double()).sum() + n * h * 128)
    assert abs(dot(out[0], go) - dot(x, out[1])) <= slack
    assert abs(dot(out[2], go) - dot(out[3], go) - dot(out[1], v)) <= slack


def _exponents(y):
    y = torch.where(torch.isfinite(y), y, torch.zeros_like(y))
    top = y.abs().amax(-1).double()
    e = torch.ceil(torch.log2(top / 448.0))
    return torch.where(top == 0, torch.zeros_like(e), e.clamp(-126, 127)), top


def _pool(n_pages, kv, page, d, dtype, order):
    """K, V and exponents of a pool whose memory is laid out in `order`, as views [pages, kv, page, d]."""
    shape = (n_pages, kv, page, d)
    if order == "tokens":                                            # [pages, page, kv, d]
        k, v = (torch.zeros(n_pages, page, kv, d, dtype=torch.uint8 if dtype == "e4m3" else torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2))
    else:
        k, v = (torch.zeros(shape, dtype=torch.uint8 if dtype == "e4m3" else torch.bfloat16, device=DEV) for _ in range(2))
    e = [torch.full(shape[:3], 77, dtype=torch.uint8, device=DEV) for _ in range(2)] if dtype == "e4m3" else [None, None]
    return k, v, e


CACHES = [  # tokens, query heads, key heads, head_dim, rot_dim, page
    (1, 8, 1, 128, 128, 16), (37, 4, 4, 128, 64, 16), (64, 3, 2, 64, 64, 32), (300, 2, 3, 80, 32, 64), (5, 0, 1, 256, 0, 128), (2000, 9, 1, 128, 96, 256),
    (130, 5, 5, 16, 16, 16), (4099, 4, 2, 128, 128, 64)]


@pytest.mark.parametrize("order", ["packed", "tokens"])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("case", CACHES)
def test_cache_write_and_read(case, layout, dtype, order):
    n, h, kv, d, rot, page = case
    g = _gen(n + page)
    rope = cf.rope_make(d, rot, layout, base=1e4) if rot else None
    x = (_normal(g, n, h + 2 * kv, d) * torch.exp2(torch.randint(-20, 20, (n, h + 2 * kv, 1), generator=g, device=DEV).float())).to(torch.bfloat16)
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    k[0, 0] = 0                                                       # a row of zeros
    pos = _positions(g, n, 1 << 17)
    pages = -(-n // page) + 2
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:n]
    away = torch.zeros(n, dtype=torch.bool, device=DEV)
    if n > 3:                                                        # padding in the batch
        slots[1], slots[2] = -1, pages * page
        away[1:3] = True
    pk, pv, (ek, ev) = _pool(pages, kv, page, d, dtype, order)
    desc = cf.cache_desc(dtype, pages, page, kv, d, (0, 0, 0) if order == "packed" else pk.stride()[:3])
    cache = cf.make_cache(pk, pv, ek, ev)
    out = torch.full((n, h, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    s = x.stride()[:2]
    cf.cache_write(desc, cache, cf.cache_rows(n, h, q=s, k=s, v=s), rope, q if h else None, k, v, pos if rope else None, slots, out if h else None)
    back = torch.full((2, n, kv + 1, d), -7.0, dtype=torch.bfloat16, device=DEV)
    bs = back[0].stride()[:2]
    cf.cache_read(desc, cache, cf.cache_rows(n, k=bs, v=bs), slots, back[0], back[1])
    torch.cuda.synchronize()
    assert bool((back[:, :, kv] == -7).all()) and bool((back[:, away] == -7).all())             # left as they were
    if h:
        y, size = _turned(q, pos, rope)
        assert bool(((out.double() - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -20 * size).all())
    stay = ~away
    for src, turned, got, pool, exps in ((k, rope is not None, back[0], pk, ek), (v, False, back[1], pv, ev)):
        y, size = _turned(src, pos, rope) if turned else (src.double(), torch.zeros_like(src, dtype=torch.float64))
        y, size, got = y[stay], size[stay], got[:, :kv][stay].double()
        p, i = (slots // page)[stay], (slots % page)[stay]
        # what lies in the pool is what comes back, and nothing else was touched
        held = pool[p, :, i]
        if dtype == "bf16":
            assert torch.equal(held.double(), got)
            assert bool(((got - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -20 * size).all())
        else:
            e = exps[p, :, i].double() - 127
            assert torch.equal(held.view(torch.float8_e4m3fn).double() * torch.exp2(e)[..., None], got)
            want, top = _exponents(y)
            near = (size.amax(-1) * 2.0 ** -20 >= (top / 448 - torch.exp2(torch.round(torch.log2(top / 448)))).abs() * 448)
            assert bool(((e == want) | (near & ((e - want).abs() <= 1))).all())
            assert bool(((got - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -10 * torch.exp2(e)[..., None] + 2.0 ** -20 * size).all())
            if not turned:
                code = (y * torch.exp2(-want)[..., None]).float().to(torch.float8_e4m3fn)      # exact, then to nearest even
                assert torch.equal(held, code.view(torch.uint8))
        left = torch.ones(pages, page, dtype=torch.bool, device=DEV)
        left[p, i] = False
        assert bool((pool.transpose(1, 2)[left] == 0).all())
        if exps is not None:
            assert bool((exps.transpose(1, 2)[left] == 77).all())


def test_e4m3_borders_zeros_infinities_and_nan():
    """Rows around the largest code, of denormal and of the largest size, and with values that are not finite."""
    inf, nan = float("inf"), float("nan")
    rows = [[448.0, 1.0], [450.0, 1.0], [1.75, 1.7421875], [1.7578125, 0.0], [2.0 ** -126, 2.0 ** -130], [3.3895314e38, -1.0], [2.0 ** -9, 2.0 ** -18],
            [inf, 3.0], [nan, 448.0], [-inf, 0.0], [0.0, 0.0], [-0.0, 5.0], [0.0146484375 * 448, 0.0146484375 / 2 ** 10]]
    n = len(rows)
    k = torch.zeros(n, 1, 128, dtype=torch.bfloat16, device=DEV)
    k[:, 0, ::64] = torch.tensor(rows, device=DEV).to(torch.bfloat16)
    pk, pv, (ek, ev) = _pool(1, 1, 16, 128, "e4m3", "packed")
    desc, cache, w = cf.cache_desc("e4m3", 1, 16, 1), cf.make_cache(pk, pv, ek, ev), cf.cache_rows(n)
    slots = torch.arange(n, device=DEV)
    cf.cache_write(desc, cache, w, None, None, k, k, None, slots, None)
    back = torch.empty(2, n, 1, 128, dtype=torch.bfloat16, device=DEV)
    cf.cache_read(desc, cache, w, slots, back[0], back[1])
    torch.cuda.synchronize()
    assert torch.equal(pk, pv) and torch.equal(ek, ev)
    e, _ = _exponents(k.double())
    assert torch.equal(ek[0, 0, :n].double() - 127, e[:, 0])
    x = k.double()
    most = torch.where(e == 120, 240.0, 448.0)[..., None]             # 256 * 2^120 is no finite number of 32 bits
    y = torch.minimum(torch.maximum(x * torch.exp2(-e)[..., None], -most), most)
    want = torch.where(torch.isfinite(x), y.float().to(torch.float8_e4m3fn).double() * torch.exp2(e)[..., None], torch.full_like(x, nan))
    assert torch.equal(back[0].double().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))


def test_a_slot_read_into_several_rows_and_pools_beyond_32_bits():
    """Two pages four GiB apart."""
    n, page, d = 20, 16, 128
    stride = (1 << 32) + 4096
    pool = torch.zeros(stride + page * d, dtype=torch.uint8, device=DEV)
    v = torch.zeros(2 * page * d, dtype=torch.uint8, device=DEV)
    e = [torch.zeros(2, 1, page, dtype=torch.uint8, device=DEV) for _ in range(2)]
    desc = cf.cache_desc("e4m3", 2, page, 1, d, (stride, page * d, d))
    g = _gen(3)
    k = _normal(g, n, 1, d).to(torch.bfloat16)
    slots = torch.arange(n, device=DEV) + 5
    big = cf.make_cache(pool, torch.zeros_like(pool), e[0], e[1])
    cf.cache_write(desc, big, cf.cache_rows(n), None, None, k, k, None, slots, None)
    again = torch.tensor([5, 24, 24, 21, 5], device=DEV)
    back = torch.empty(2, 5, 1, d, dtype=torch.bfloat16, device=DEV)
    cf.cache_read(desc, big, cf.cache_rows(5), again, back[0], back[1])
    torch.cuda.synchronize()
    y = k[again - 5].double()
    assert torch.equal(back[0], back[1])
    assert bool(((back[0].double() - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -10 * torch.exp2(_exponents(y)[0])[..., None]).all())
    assert bool((pool[stride:stride + 9 * d].view(9, d) != 0).any(1).all()) and not bool(pool[page * d:stride].any())


def test_graph_replays_with_other_positions_and_slots():
    g = _gen(11)
    n, h, kv, page = 48, 4, 2, 16
    rope = cf.rope_make(128, 128)
    x = _normal(g, n, h + 2 * kv, 128).to(torch.bfloat16)
    pk, pv, (ek, ev) = _pool(8, kv, page, 128, "e4m3", "packed")
    desc, cache = cf.cache_desc("e4m3", 8, page, kv), cf.make_cache(pk, pv, ek, ev)
    s = x.stride()[:2]
    rows, pos, slots = cf.cache_rows(n, h, q=s, k=s, v=s), torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, device=DEV)
    out, back = torch.zeros(n, h, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, n, kv, 128, dtype=torch.bfloat16, device=DEV)

    def step(stream):
        cf.cache_write(desc, cache, rows, rope, x[:, :h], x[:, h:h + kv], x[:, h + kv:], pos, slots, out, stream)
        cf.cache_read(desc, cache, cf.cache_rows(n), slots, back[0], back[1], stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for i in range(4):
        pos.copy_(_positions(g, n, 5000))
        slots.copy_(torch.randperm(8 * page, generator=g, device=DEV)[:n])
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), back.clone()
        out.zero_(), back.zero_()
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], back)
