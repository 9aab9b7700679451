"""Entries of the page table between the first tokens and the window, whatever they hold, leave no trace in a result.  Needs an MI355X: ``-m gpu``."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_paged import DEV
from tests.test_gpu_attn_window_paged import Windowed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    ws = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(ws)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)


CASES = [(8, 1, 16, [1, 1], [1003, 5000], 64, 4), (8, 1, 16, [1, 4], [5000, 3000], 700, 40), (4, 4, 32, [1, 1], [2000, 4096], 100, 0), (16, 1, 16, [2], [9001], 1500, 1)]
MANY = [(8, 1, 16, [40, 64], [5000, 3000], 700, 40)]


def _results(b, what, value):
    """Outputs but for feature 5, and lse; V of a key in every row's window has `value` there, and the entries that no row sees, and that share no tile of 64
    keys with one that is seen, are `what`."""
    b.table.copy_(b.whole)
    for s, (m, n) in enumerate(zip(b.new, b.ctx)):
        key = n - max(b.new)                                             # the first new token's own, or one that it sees
        b.pool[1][int(b.whole[s, key // b.page]), :, key % b.page, 5] = value
        first, last = -(-b.sinks // 64) * 64, (n - m - b.window + 1) // 64 * 64
        for i in range(-(-first // b.page), last // b.page):
            b.table[s, i] = {"there": b.whole[s, i], "none": -1, "another": b.whole[1 - s if len(b.new) > 1 else s, 0]}[what]
    out, lse = b.run()
    assert bool(torch.isfinite(lse).all()) and bool(torch.isfinite(out[..., :5].float()).all()) and bool(torch.isfinite(out[..., 6:].float()).all())
    return out[..., 5].float(), torch.cat([out[..., :5], out[..., 6:]], -1), lse


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES + MANY)
def test_results_that_are_not_finite_do_not_look_at_them(case, dtype):
    """One feature of V is not finite, so that every row has a feature that is not.  The other 127 have the same bits whether what lies between first
    tokens and window is there, names no page (an entry that went back) or another sequence's."""
    heads, kv, page, new, ctx, window, sinks = case
    b = Windowed(17, heads, kv, page, dtype, new, ctx, window, sinks)
    value = math.inf if dtype == "bf16" else 127
    results = [_results(b, what, value) for what in ("there", "none", "another")]
    for five, out, lse in results:
        assert not bool(torch.isfinite(five).any()) and torch.equal(out, results[0][1]) and torch.equal(lse, results[0][2])


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", CASES)
def test_what_every_row_sees_is_no_reason_for_a_second_walk(case, dtype):
    """A second walk, for values that some rows do not see, has other roundings (of probabilities under another maximum).  A feature of V that is not finite
    where all rows see it leaves the bits of the other features as they are with a finite one."""
    heads, kv, page, new, ctx, window, sinks = case
    b = Windowed(18, heads, kv, page, dtype, new, ctx, window, sinks)
    finite, odd = _results(b, "none", 0), _results(b, "none", math.inf if dtype == "bf16" else 127)
    assert bool(torch.isfinite(finite[0]).all()) and not bool(torch.isfinite(odd[0]).any())
    assert torch.equal(finite[1], odd[1]) and torch.equal(finite[2], odd[2])
