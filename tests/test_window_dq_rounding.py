"""How often dQ of windowed attention is rounded on its way to bf16.

The gradient's operands are Q, K, V, dout, `out` and lse as they are given, so that in 64 bits P = exp(scale q k - lse), delta = sum of dout * out and
dQ = scale (P (dP - delta)) K are exact, and what a result is off by is its own rounding and what dS lost before its product.  An element x = m 2^e,
1 <= m < 2, rounded to bf16 is off by up to 2^(e-8), evenly spread: a mean square of 4^(e-8) / 3.  Sums of that over N >= 4e4 elements vary by
sqrt(0.8 / N) < 0.5 % of themselves; fp32 sums and scores (2^-17 of what they add up) and dS as two bf16 numbers (2^-16) add less than a
thousandth to it, and 15 % are left for elements that are not spread evenly.  dS rounded once adds, for every element of dQ, the sum over keys of
scale^2 k^2 4^(e-8) / 3 with e of each element of dS: about as much again.  The CPU test plants that in the oracle and shows that the limit tells both apart."""
import math
import os

import pytest
import torch

D = 128
SCALE = 1 / math.sqrt(D)
LIMIT = 1.15
CASES = [(4, 4, [700, 500], 128, 4), (8, 1, [900], 256, 16), (2, 1, [64, 300, 33], 40, 0)]        # heads, key heads, lengths, window, first tokens


def problem(case):
    """Q, K, V in one tensor, dout and the starts of the sequences, on the CPU."""
    h, kv, lens, _, _ = case
    g = torch.Generator()
    g.manual_seed(31)
    x = torch.randn(sum(lens), h + 2 * kv, D, generator=g).to(torch.bfloat16)
    return x, torch.randn(sum(lens), h, D, generator=g).to(torch.bfloat16), [sum(lens[:i]) for i in range(len(lens) + 1)]


def hidden(n, window, sinks):
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    return (j > i) | ((j <= i - window) & (j >= sinks))


def forward(case, x, at):
    """out in bf16 and lse in fp32, rounded once."""
    h, kv, _, window, sinks = case
    out, lse = torch.empty(x.shape[0], h, D, dtype=torch.bfloat16), torch.empty(h, x.shape[0])
    for a, b in zip(at, at[1:]):
        for i in range(h):
            q, k, v = x[a:b, i].double(), x[a:b, h + i // (h // kv)].double(), x[a:b, h + kv + i // (h // kv)].double()
            s = (q @ k.t() * SCALE).masked_fill(hidden(b - a, window, sinks), -math.inf)
            lse[i, a:b], out[a:b, i] = torch.logsumexp(s, 1).float(), (torch.softmax(s, 1) @ v).to(torch.bfloat16)
    return out, lse


def mean_square_of_rounding(x):
    """... to bf16, of each element."""
    _, e = torch.frexp(x)                                            # (x = m 2^e with m from 1/2 on)
    return torch.where(x == 0, torch.zeros_like(x), torch.ldexp(torch.ones_like(x), 2 * (e - 9)) / 3)


def exact(case, x, dout, at, out, lse, dS=lambda t: t):
    """dQ in 64 bits, of operands as they are, with dS as `dS` rounds it; and the mean square that rounding dS once adds to it, summed over all elements."""
    h, kv, _, window, sinks = case
    dq, added = torch.empty(x.shape[0], h, D, dtype=torch.float64), 0.0
    for a, b in zip(at, at[1:]):
        for i in range(h):
            q, k, v = x[a:b, i].double(), x[a:b, h + i // (h // kv)].double(), x[a:b, h + kv + i // (h // kv)].double()
            g = dout[a:b, i].double()
            p = torch.exp((q @ k.t() * SCALE).masked_fill(hidden(b - a, window, sinks), -math.inf) - lse[i, a:b, None].double())
            ds = p * (g @ v.t() - (g * out[a:b, i].double()).sum(1)[:, None])
            dq[a:b, i] = SCALE * dS(ds) @ k
            added += SCALE ** 2 * float((mean_square_of_rounding(ds) @ (k ** 2)).sum())
    return dq, added


def excess(dq, want):
    """Of the sum of squared errors over what one rounding makes."""
    return float(((dq.double() - want) ** 2).sum() / mean_square_of_rounding(want).sum())


@pytest.mark.parametrize("case", CASES)
def test_the_limit_tells_one_rounding_from_two(case):
    x, dout, at = problem(case)
    out, lse = forward(case, x, at)
    want, added = exact(case, x, dout, at, out, lse)

    def once(t):
        return t.to(torch.bfloat16).double()

    halves, _ = exact(case, x, dout, at, out, lse, lambda t: once(t) + once(t - once(t)))
    rounded, _ = exact(case, x, dout, at, out, lse, once)
    assert want.numel() >= 40000 and excess(once(want), want) <= LIMIT and excess(once(halves), want) <= LIMIT
    two = 1 + added / float(mean_square_of_rounding(want).sum())
    assert two > LIMIT ** 2 and two / LIMIT <= excess(once(rounded), want) <= two * LIMIT


@pytest.mark.gpu
@pytest.mark.parametrize("launch", [None, "4x100000", "8x1", "4x3"])       # waves of a workgroup and tiles of a split
@pytest.mark.parametrize("case", CASES)
def test_dq_has_one_rounding(case, launch, monkeypatch):
    from paper_2604_24013_amd import binding as cf
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    if launch:
        monkeypatch.setenv("COMMFUSE_CAUSAL", launch)
    h, kv, lens, window, sinks = case
    x, dout, at = problem(case)
    dev = "cuda:0"
    xd, gd, starts = x.to(dev), dout.to(dev), torch.tensor(at, dtype=torch.int32, device=dev)
    T, s, w = x.shape[0], x.stride()[:2], cf.window(window, sinks)
    out, lse, delta = torch.empty(T, h, D, dtype=torch.bfloat16, device=dev), torch.empty(h, T, device=dev), torch.empty(h, T, device=dev)
    q, k, v, dx = xd[:, :h], xd[:, h:h + kv], xd[:, h + kv:], torch.empty_like(xd)
    ws = torch.empty(128 << 20, dtype=torch.uint8, device=dev)
    desc = cf.prompt_desc(T, len(lens), h, kv, SCALE, q=s, k=s, v=s)
    cf.set_workspace(ws)
    try:
        cf.attn_prompt_window(desc, w, q, k, v, starts, out, lse)
        cf.attn_prompt_window_grad(desc, w, q, k, v, out, lse, gd, starts, delta, dx[:, :h], dx[:, h:h + kv], dx[:, h + kv:])
        torch.cuda.synchronize()
    finally:
        cf.set_workspace(None)
    want, _ = exact(case, x, dout, at, out.cpu(), lse.cpu())
    assert excess(dx[:, :h].cpu(), want) <= LIMIT
