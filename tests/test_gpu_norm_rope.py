"""Normed and rotated heads on the GPU against plain forms in 64 bits: forward, gradient, and on the way into the cache.  Needs an MI355X: ``-m gpu``.

Tolerances.  A sum of squares of up to 256 features, in threads of 16 at the most and a tree of six: off by (16 + 6) 2^-24 of itself at the most, the
root by half of that; with mean, eps, root, quotient, and the products with r and (offset + w), eight more roundings, a normed value is off
by less than 2^-19 of itself.  Rotation adds 2^-20 of its pair's size (|x_a| + |x_b|, see the tests of the rotation alone) and passes on the
pair's own 2^-19: less than 2^-18 of the size.  Then half a step of the type.
Gradient, with G the pair's size of dy times |offset + w| >= |h|: g is off by 2^-20 G, n by 2^-19, the mean of h n by (2^-20 + 2^-19 +
2^-19) of that of G |n|, so dx by less than 2^-16 r (G + |n| mean(G |n|)).  The sums over tokens and heads go through chains of fewer than 400
additions: (2^-17 + 400 2^-24) of the sum of the magnitudes, less than 2^-15."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
NAN = float("nan")


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


def _pair(t):
    return t.stride(0), t.stride(1)


def _turned(x, positions, rope, sign=1.0):
    """(rotated in 64 bits, |x_a| + |x_b| of each value's pair; positions [axes, tokens]"""
    r = rope.rope
    rot = r.rot_dim
    turn = torch.tensor([r.turn[j] / 2.0 ** 64 for j in range(rot // 2)], dtype=torch.float64, device=DEV)
    axis = torch.tensor([rope.axis[j] for j in range(rot // 2)], device=DEV)
    t = positions.double()[axis].t() * turn
    angle = (t - t.round())[:, None, :] * (2 * math.pi)
    c, s = torch.cos(angle) * r.magnitude, torch.sin(angle) * r.magnitude * sign
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if r.layout == cf.CF_ROPE_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    y, size = x.clone(), x.abs()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = r.magnitude * (x[..., a].abs() + x[..., b].abs())
    return y, size


def _factor(w, offset, d):
    return torch.ones(d, dtype=torch.float64, device=DEV) if w is None else w.double() + offset


def _forward(x, w, offset, eps, positions, rope):
    n = x.double()
    if eps is not None:
        n = n / torch.sqrt(n.pow(2).mean(-1, keepdim=True) + eps) * _factor(w, offset, x.shape[-1])
    return _turned(n, positions, rope) if rope is not None else (n, n.abs())


def _backward(x, w, offset, eps, positions, rope, dy):
    """(dx, what its tolerance is relative to, dw, the same)"""
    g, size = _turned(dy.double(), positions, rope, -1.0) if rope is not None else (dy.double(), dy.double().abs())
    if eps is None:
        return g, size, None, None
    x, f = x.double(), _factor(w, offset, x.shape[-1])
    r = 1 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    n, h = x * r, g * f
    dx = r * (h - n * (h * n).mean(-1, keepdim=True))
    big = size * f.abs()
    return dx, r * (big + n.abs() * (big * n.abs()).mean(-1, keepdim=True)), (g * n).sum((0, 1)), (size * n.abs()).sum((0, 1))


def _close(out, want, dtype, slack):
    return bool(((out.double() - want).abs() <= HALF_STEP[dtype] * want.abs() + slack).all())


def _positions(g, axes, n, far):
    p = torch.randint(-far, far, (axes, n), generator=g, device=DEV, dtype=torch.int32)
    p[0, 0] = 0
    p[-1, -1] = far - 1
    return p


SHAPES = [  # tokens, heads, kv_heads, head_dim, rot_dim, sections, order, spectrum
    (1, 1, 1, 128, 128, (24, 20, 20), "interleaved", "shared"), (3, 5, 2, 128, 64, (16, 16), "sections", "own"),
    (64, 8, 1, 128, 128, (16, 24, 24), "sections", "shared"), (257, 3, 3, 64, 64, (11, 7, 7, 7), "interleaved", "own"),
    (33, 2, 1, 256, 256, (128,), "sections", "shared"), (17, 4, 0, 80, 32, (1, 2, 13), "sections", "own"),
    (9, 0, 2, 96, 24, (4, 4, 4), "interleaved", "shared"), (5, 3, 1, 8, 2, (1,), "sections", "own"),
    (70, 2, 2, 128, 126, (60, 3), "sections", "shared"), (2049, 8, 2, 128, 128, (22, 21, 21), "interleaved", "shared"),
    (11, 3, 1, 72, 72, (30, 3, 3), "sections", "own"), (6, 2, 3, 200, 100, (20, 10, 10, 10), "interleaved", "shared")]


def _inputs(shape, dtype, seed):
    n, h, kv, d, rot, sections, order, spectrum = shape
    g = _gen(seed)
    rope = cf.rope_axes_make(d, rot, "half" if seed % 2 else "interleaved", base=5e5, scaling="wavelength", factor=8.0, trained_len=8192, magnitude=1.25,
                             sections=sections, order=order, spectrum=spectrum)
    x = (_normal(g, n, h + 2 * kv + 1, d) * torch.exp(_normal(g, d))).to(TYPES[dtype])      # the heads lie inside a wider row
    w = [(0.3 * _normal(g, d) + 1.0).to(TYPES["bf16" if seed % 3 else "f32"]) for _ in range(2)]
    pos = _positions(g, len(sections), n, 2 ** 31 - 1 if n % 2 else 100000)
    return g, rope, x, x[:, 1:1 + h], x[:, 1 + h:1 + h + kv], w, pos


@pytest.mark.parametrize("seed", [1, 2, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_gradient(shape, dtype, seed):
    n, h, kv, d, rot, _, _, _ = shape
    g, rope, x, q, k, w, pos = _inputs(shape, dtype, seed)
    offset, eps = (1.0, 1e-6) if seed == 2 else (0.0, 1e-5)
    norm = cf.head_norm(eps, offset, "bf16" if w[0].dtype == torch.bfloat16 else "f32")
    y = torch.full((n, h + kv, d), NAN, dtype=TYPES[dtype], device=DEV)
    yq, yk = y[:, :h], y[:, h:]
    rows = cf.head_rows(n, h, kv, d, dtype, q=_pair(x), k=_pair(x), oq=_pair(y), ok=_pair(y))
    keep = x.clone()
    cf.norm_rope(rope, norm, rows, q, k, w[0], w[1], pos, pos.stride(0), yq, yk)
    torch.cuda.synchronize()
    assert torch.equal(x, keep)
    for part, out, wt in ((q, yq, w[0]), (k, yk, w[1])):
        want, size = _forward(part, wt, offset, eps, pos, rope)
        assert _close(out, want, dtype, 2.0 ** -18 * size)
    # gradient
    dy = _normal(g, n, h + kv, d).to(TYPES[dtype])
    dx = torch.full_like(x, NAN)
    dw = torch.full((2, d), NAN, device=DEV)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    cf.norm_rope_grad(rope, norm, rows, q, k, w[0], w[1], pos, pos.stride(0), dy[:, :h], dy[:, h:], dx[:, 1:1 + h], dx[:, 1 + h:1 + h + kv], dw[0], dw[1], scratch)
    torch.cuda.synchronize()
    for part, grad, go, wt, dwt in ((q, dx[:, 1:1 + h], dy[:, :h], w[0], dw[0]), (k, dx[:, 1 + h:1 + h + kv], dy[:, h:], w[1], dw[1])):
        want, slack, want_w, slack_w = _backward(part, wt, offset, eps, pos, rope, go)
        assert _close(grad, want, dtype, 2.0 ** -16 * slack)
        assert bool(((dwt.double() - want_w).abs() <= 2.0 ** -15 * slack_w).all())
    assert bool(dx[:, :1].isnan().all()) and bool(dx[:, 1 + h + kv:].isnan().all())          # what is no head of Q or K stays as it was
    # the same call, the same bits; in place over dy
    again, dw2 = dy.clone(), torch.empty_like(dw)
    rows2 = cf.head_rows(n, h, kv, d, dtype, q=_pair(dy), k=_pair(dy), oq=_pair(dy), ok=_pair(dy))
    packed = torch.cat([q, k], 1).contiguous()
    cf.norm_rope_grad(rope, norm, rows2, packed[:, :h], packed[:, h:], w[0], w[1], pos, pos.stride(0), again[:, :h], again[:, h:], again[:, :h], again[:, h:],
                      dw2[0], dw2[1], scratch)
    # in place over x
    over = torch.cat([q, k], 1).contiguous()
    cf.norm_rope_grad(rope, norm, rows2, over[:, :h], over[:, h:], w[0], w[1], pos, pos.stride(0), dy[:, :h], dy[:, h:], over[:, :h], over[:, h:], None, dw2[1], scratch)
    # in place forward
    cf.norm_rope(rope, norm, rows2, packed[:, :h], packed[:, h:], w[0], w[1], pos, pos.stride(0), packed[:, :h], packed[:, h:])
    torch.cuda.synchronize()
    assert torch.equal(again, dx[:, 1:1 + h + kv]) and torch.equal(over, again) and torch.equal(dw2, dw) and torch.equal(packed, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n, d, rot", [(65, 128, 128), (7, 96, 64), (3, 72, 70)])
def test_rotation_alone_on_one_axis_is_the_rotation(n, d, rot, layout, dtype):
    g = _gen(n)
    h, kv = 3, 2
    one, axes = cf.rope_make(d, rot, layout, base=1e6, magnitude=0.5), cf.rope_axes_make(d, rot, layout, base=1e6, magnitude=0.5)
    x, pos = _normal(g, n, h + kv, d).to(TYPES[dtype]), _positions(g, 1, n, 1 << 30)
    out, want = torch.empty(2, n, h + kv, d, dtype=TYPES[dtype], device=DEV)
    rows = cf.head_rows(n, h, kv, d, dtype, *[_pair(x)] * 4)
    for back in (False, True):
        cf.rope(one, cf.rope_rows(n, h + kv, dtype), x, pos, want, back)
        if back:
            cf.norm_rope_grad(axes, None, rows, None, None, None, None, pos, 0, x[:, :h], x[:, h:], out[:, :h], out[:, h:])
        else:
            cf.norm_rope(axes, None, rows, x[:, :h], x[:, h:], None, None, pos, 0, out[:, :h], out[:, h:])
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_alone_one_position_and_no_weights(dtype):
    """Without rope; without weights; and one row of positions for all axes."""
    g = _gen(3)
    n, h, kv, d = 130, 4, 1, 128
    x, w = _normal(g, n, h + kv, d).to(TYPES[dtype]), _normal(g, d).to(TYPES[dtype])
    rows, norm = cf.head_rows(n, h, kv, d, dtype, *[_pair(x)] * 4), cf.head_norm(1e-6, 0.0, dtype)
    out = torch.empty_like(x)
    cf.norm_rope(None, norm, rows, x[:, :h], x[:, h:], w, None, None, 0, out[:, :h], out[:, h:])
    torch.cuda.synchronize()
    for a, b, wt in ((0, h, w), (h, h + kv, None)):
        want, size = _forward(x[:, a:b], wt, 0.0, 1e-6, None, None)
        assert _close(out[:, a:b], want, dtype, 2.0 ** -18 * size)
    three = cf.rope_axes_make(d, d, sections=(20, 22, 22))
    pos, out2 = _positions(g, 1, n, 5000), torch.empty_like(x)
    cf.norm_rope(three, norm, rows, x[:, :h], x[:, h:], w, w, pos, 0, out[:, :h], out[:, h:])
    cf.norm_rope(three, norm, rows, x[:, :h], x[:, h:], w, w, pos.expand(3, n).contiguous(), n, out2[:, :h], out2[:, h:])
    torch.cuda.synchronize()
    assert torch.equal(out, out2)


def test_gradient_against_differences():
    """<dx, v> and <dw, u> against central differences, in 64 bits, of the definition: of order 2^-24 of the sums (the third derivative over
    h^2 / 6, h = 2^-12), and the kernel's own tolerance."""
    g = _gen(9)
    n, h, d = 21, 3, 128
    rope = cf.rope_axes_make(d, 96, "interleaved", sections=(20, 14, 14), order="interleaved", magnitude=1.5)
    x, w, dy, v, u = _normal(g, n, h, d), _normal(g, d), _normal(g, n, h, d), _normal(g, n, h, d), _normal(g, d)
    pos = _positions(g, 3, n, 4000)
    rows, norm = cf.head_rows(n, h, 0, d, "f32"), cf.head_norm(1e-2, 1.0, "f32")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    cf.norm_rope_grad(rope, norm, rows, x, None, w, None, pos, n, dy, None, dx, None, dw, None, scratch)
    torch.cuda.synchronize()
    loss = lambda xx, ww: float((_forward(xx, ww, 1.0, 1e-2, pos, rope)[0] * dy.double()).sum())
    t = 2.0 ** -12
    xd, wd = x.double(), w.double()
    by_x = (loss(xd + t * v.double(), wd) - loss(xd - t * v.double(), wd)) / (2 * t)
    by_w = (loss(xd, wd + t * u.double()) - loss(xd, wd - t * u.double())) / (2 * t)
    _, slack, _, slack_w = _backward(x, w, 1.0, 1e-2, pos, rope, dy)
    far = 2.0 ** -15
    assert abs(by_x - float((dx.double() * v.double()).sum())) <= far * float((slack * v.double().abs()).sum())
    assert abs(by_w - float((dw.double() * u.double()).sum())) <= far * float((slack_w * u.double().abs()).sum())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_extreme_rows(dtype):
    """Rows of zeros, of the smallest and the largest magnitudes, and not finite ones, which reach no other row."""
    g = _gen(4)
    n, h, d = 40, 2, 128
    x = _normal(g, n, h, d)
    x[3] = 0.0
    x[5] *= 1e30                                                     # (squares beyond fp32's range)
    x[7] *= 1e-30
    x = x.to(TYPES[dtype])
    clean = x.clone()
    x[11, 0, 17], x[13, 1, 100], x[15, 1] = NAN, float("inf"), -float("inf")
    w, pos, rope = _normal(g, d).to(TYPES[dtype]), _positions(g, 1, n, 1000), cf.rope_axes_make(d, 64)
    dy = _normal(g, n, h, d).to(TYPES[dtype])
    rows, norm = cf.head_rows(n, h, 0, d, dtype), cf.head_norm(1e-6, 0.0, dtype)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    got = []
    for t in (clean, x):
        out, dx, dw = torch.empty_like(t), torch.empty_like(t), torch.empty(d, device=DEV)
        cf.norm_rope(rope, norm, rows, t, None, w, None, pos, 0, out, None)
        cf.norm_rope_grad(rope, norm, rows, t, None, w, None, pos, 0, dy, None, dx, None, dw, None, scratch)
        torch.cuda.synchronize()
        got.append((out, dx, dw))
    want, size = _forward(clean, w, 0.0, 1e-6, pos, rope)
    dx, slack, dw, slack_w = _backward(clean, w, 0.0, 1e-6, pos, rope, dy)
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -148           # (steps of what is too small to be normal)
    assert _close(got[0][0], want, dtype, 2.0 ** -18 * size + tiny)
    assert _close(got[0][1], dx, dtype, 2.0 ** -16 * slack + tiny)
    assert bool(((got[0][2].double() - dw).abs() <= 2.0 ** -15 * slack_w).all())
    odd = torch.zeros(n, h, dtype=torch.bool, device=DEV)
    odd[11, 0] = odd[13, 1] = odd[15, 1] = True
    for a, b in zip(got[0][:2], got[1][:2]):
        assert torch.equal(a[~odd], b[~odd])
    assert bool(got[1][0][11, 0].isnan().all()) and bool(got[1][0][13, 1].isnan().any()) and bool(got[1][2].isnan().all())


def test_no_rows():
    d = 128
    dw = torch.full((2, d), NAN, device=DEV)
    rows, norm = cf.head_rows(0, 4, 1, d), cf.head_norm(1e-6)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    cf.norm_rope(None, norm, rows, None, None, None, None, None, 0, None, None)
    cf.norm_rope_grad(None, norm, rows, None, None, None, None, None, 0, None, None, None, None, dw[0], dw[1], scratch)
    torch.cuda.synchronize()
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n, h, kv, d, rot, page", [(1, 8, 1, 128, 128, 16), (67, 4, 4, 128, 64, 64), (300, 5, 2, 96, 96, 32), (20, 2, 1, 256, 128, 16),
                                                    (2050, 8, 1, 128, 128, 64), (19, 0, 3, 64, 64, 16), (5, 2, 2, 16, 16, 16)])
def test_cache_write(n, h, kv, d, rot, page, dtype):
    """bf16: the bits of norm_rope's results; e4m3: within half a step of the normed keys.  V, and with neither norm nor several axes everything, as the
    cache's other writer has it."""
    g = _gen(n + page)
    half = rot // 2
    rope = cf.rope_axes_make(d, rot, "half" if n % 2 else "interleaved", sections=(half - 2 * (half // 3), half // 3, half // 3), order="interleaved")
    norm = cf.head_norm(1e-6, 1.0, "f32")
    x, pos = _normal(g, n, h + 2 * kv, d).to(torch.bfloat16), _positions(g, 3, n, 100000)
    w = [0.2 * _normal(g, d) for _ in range(2)]
    pages = -(-n // page) + 2
    slots = torch.randperm(pages * page, device=DEV, generator=g)[:n]
    if n > 4:
        slots[2], slots[3] = -1, pages * page                        # padding
    stored = (slots >= 0) & (slots < pages * page)
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    rows = cf.cache_rows(n, h, q=_pair(x), k=_pair(x), v=_pair(x))
    desc = cf.cache_desc(dtype, pages, page, kv, d)

    def pools():
        t = torch.bfloat16 if dtype == "bf16" else torch.uint8
        p = [torch.full((pages, kv, page, d), 113, dtype=torch.uint8, device=DEV).to(t) for _ in range(2)]
        e = [torch.full((pages, kv, page), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
        return p, e, cf.make_cache(p[0], p[1], e[0], e[1])

    def back(cache):
        out = torch.zeros(2, n, kv, d, dtype=torch.bfloat16, device=DEV)
        cf.cache_read(desc, cache, cf.cache_rows(n), slots, out[0], out[1])
        torch.cuda.synchronize()
        return out[0][stored], out[1][stored]

    q_out, want_q = torch.full((2, n, max(h, 1), d), NAN, dtype=torch.bfloat16, device=DEV)
    want_k = torch.empty(n, kv, d, dtype=torch.bfloat16, device=DEV)
    p, e, cache = pools()
    cf.cache_write_norm(desc, cache, rows, rope, norm, q if h else None, k, v, w[0], w[1], pos, n, slots, q_out if h else None)
    got_k, got_v = back(cache)
    cf.norm_rope(rope, norm, cf.head_rows(n, h, kv, d, q=_pair(x), k=_pair(x)), q, k, w[0], w[1], pos, n, want_q, want_k)
    torch.cuda.synchronize()
    assert h == 0 or torch.equal(q_out, want_q)
    if dtype == "bf16":
        assert torch.equal(got_k, want_k[stored]) and torch.equal(got_v, v[stored])
    else:
        y, size = _forward(k, w[1], 1.0, 1e-6, pos, rope)
        y, size = y[stored], size[stored]
        # the largest magnitude is at most 448 * 2^e and more than 224 * 2^e (but for 2^-18 of it): steps below 2^-6 * 2^e are 2^-9 * 2^e
        step = 2.0 ** -9 * y.abs().amax(-1, keepdim=True) / 223.0
        assert bool(((got_k.double() - y).abs() <= 2.0 ** -4 * y.abs() * 1.0001 + step / 2 + 2.0 ** -17 * size).all())
    # rows of other slots stay as they were
    other = torch.ones(pages * page, dtype=torch.bool, device=DEV)
    other[slots[stored]] = False
    for t in p:
        assert bool((t.transpose(1, 2).reshape(pages * page, kv, d)[other] == 113).all())
    # neither norm nor axes: the other writer's bits
    plain, one = cf.rope_make(d, rot, "half", base=5e5), cf.rope_axes_make(d, rot, "half", base=5e5)
    (pa, ea, a), (pb, eb, b) = pools(), pools()
    qa, qb = torch.zeros(2, n, max(h, 1), d, dtype=torch.bfloat16, device=DEV)
    cf.cache_write(desc, a, rows, plain, q if h else None, k, v, pos[0], slots, qa if h else None)
    cf.cache_write_norm(desc, b, rows, one, None, q if h else None, k, v, None, None, pos, 0, slots, qb if h else None)
    torch.cuda.synchronize()
    assert torch.equal(qa, qb) and all(torch.equal(s, t) for s, t in zip(pa + ea, pb + eb))
    if dtype == "e4m3":                                              # V is written as there
        assert torch.equal(got_v, back(a)[1])


def test_replayed_and_on_another_stream():
    """A captured forward and gradient replays with other contents; calls on another stream than the tensors' own."""
    g = _gen(8)
    n, h, kv, d = 300, 4, 2, 128
    rope, norm = cf.rope_axes_make(d, d, sections=(24, 20, 20), order="interleaved"), cf.head_norm(1e-6)
    x, dy = _normal(g, n, h + kv, d).bfloat16(), _normal(g, n, h + kv, d).bfloat16()
    w, pos = _normal(g, 2, d).bfloat16(), _positions(g, 3, n, 5000)
    rows = cf.head_rows(n, h, kv, d, "bf16", *[_pair(x)] * 4)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(2, d, device=DEV)

    def step(y, dx, dw, scratch, s):
        cf.norm_rope(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, y[:, :h], y[:, h:], s)
        cf.norm_rope_grad(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, dy[:, :h], dy[:, h:], dx[:, :h], dx[:, h:], dw[0], dw[1], scratch, s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(y, dx, dw, scratch, torch.cuda.current_stream())
    scratch2, other = torch.empty_like(scratch), torch.cuda.Stream()
    for i in range(3):
        x.copy_(_normal(g, n, h + kv, d))
        dy.copy_(_normal(g, n, h + kv, d))
        w.copy_(_normal(g, 2, d))
        pos.copy_(_positions(g, 3, n, 1000 * (i + 1)))
        want = torch.empty_like(x), torch.empty_like(x), torch.empty_like(dw)
        other.wait_stream(torch.cuda.current_stream())
        step(*want, scratch2, other)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads_outermost_and_offsets_beyond_32_bits(dtype):
    g = _gen(11)
    n, h, kv, d = 70, 3, 2, 128
    rope, norm = cf.rope_axes_make(d, d, sections=(24, 20, 20), order="interleaved"), cf.head_norm(1e-6, 0.0, dtype)
    x, dy = _normal(g, n, h + kv, d).to(TYPES[dtype]), _normal(g, n, h + kv, d).to(TYPES[dtype])
    w, pos = _normal(g, 2, d).to(TYPES[dtype]), _positions(g, 3, n, 5000)
    rows = cf.head_rows(n, h, kv, d, dtype, *[_pair(x)] * 4)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    want, grad, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(2, d, device=DEV)
    cf.norm_rope(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, want[:, :h], want[:, h:])
    cf.norm_rope_grad(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, dy[:, :h], dy[:, h:], grad[:, :h], grad[:, h:], dw[0], dw[1], scratch)
    # tokens 2^26 elements apart, and heads outermost
    far = 1 << 26
    big = torch.zeros((n - 1) * far + (h + kv) * d, dtype=TYPES[dtype], device=DEV)
    view = big.as_strided((n, h + kv, d), (far, d, 1))
    view.copy_(x)
    rows2, dw2 = cf.head_rows(n, h, kv, d, dtype, q=_pair(view), k=_pair(view), oq=(d, n * d), ok=(d, n * d)), torch.empty(2, d, device=DEV)
    outer, gouter = torch.empty(h + kv, n, d, dtype=TYPES[dtype], device=DEV), dy.transpose(0, 1).contiguous()
    cf.norm_rope(rope, norm, rows2, view[:, :h], view[:, h:], w[0], w[1], pos, n, outer[:h], outer[h:])
    torch.cuda.synchronize()
    assert torch.equal(outer.transpose(0, 1), want)
    cf.norm_rope_grad(rope, norm, rows2, view[:, :h], view[:, h:], w[0], w[1], pos, n, gouter[:h], gouter[h:], view[:, :h], view[:, h:], dw2[0], dw2[1], scratch)
    torch.cuda.synchronize()
    assert torch.equal(view, grad) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, h, kv", [(40000, 2, 1), (1, 300, 100), (3, 1, 65), (9000, 1, 0), (70000, 0, 1)])
def test_many_tokens_and_many_heads(n, h, kv, dtype):
    """Rounds of tokens, and a token's heads shared out to workgroups.  (Chains of the weights' sums: 40000 tokens in 1024 workgroups of 8 and more, so
    fewer than 400 additions each.)"""
    g = _gen(n + h)
    d = 128
    rope, norm = cf.rope_axes_make(d, d, sections=(32, 32)), cf.head_norm(1e-6, 0.0, dtype)
    x, dy = _normal(g, n, h + kv, d).to(TYPES[dtype]), _normal(g, n, h + kv, d).to(TYPES[dtype])
    w, pos = _normal(g, 2, d).to(TYPES[dtype]), _positions(g, 2, n, 100000)
    rows = cf.head_rows(n, h, kv, d, dtype, *[_pair(x)] * 4)
    scratch = torch.empty(cf.norm_rope_scratch_bytes(rows), dtype=torch.uint8, device=DEV)
    out, grad, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(2, d, device=DEV)
    cf.norm_rope(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, out[:, :h], out[:, h:])
    cf.norm_rope_grad(rope, norm, rows, x[:, :h], x[:, h:], w[0], w[1], pos, n, dy[:, :h], dy[:, h:], grad[:, :h], grad[:, h:], dw[0], dw[1], scratch)
    torch.cuda.synchronize()
    for part, wt, dwt in ((slice(0, h), w[0], dw[0]), (slice(h, h + kv), w[1], dw[1])):
        want, size = _forward(x[:, part], wt, 0.0, 1e-6, pos, rope)
        assert _close(out[:, part], want, dtype, 2.0 ** -18 * size)
        want, slack, want_w, slack_w = _backward(x[:, part], wt, 0.0, 1e-6, pos, rope, dy[:, part])
        assert _close(grad[:, part], want, dtype, 2.0 ** -16 * slack)
        assert bool(((dwt.double() - want_w).abs() <= 2.0 ** -15 * slack_w).all())
