"""Batches of chunks and decoded tokens over the paged cache with a sliding window: walks are cut where few of a batch's sequences bring rows enough, and
left whole where their blocks fill the chip.  Tolerances as for the same attention without a window.  Needs an MI355X: ``-m gpu``."""
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_attn_paged import DEV, check
from tests.test_gpu_attn_window_paged import Windowed

pytestmark = pytest.mark.gpu
WORKSPACE = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    global WORKSPACE
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    cf.load()
    WORKSPACE = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(WORKSPACE)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)
    WORKSPACE = None


# heads, key heads, page, new, ctx, window, first tokens, whether walks are left whole: where the blocks that have rows fill three quarters of the 256 compute
# units (two workgroups each where a sequence and key head have less than 256 rows: blocks of 128 rows instead of 256).  The last batch's are left whole by
# the size of pieces: 383 walks of 10 tiles are 15 a compute unit, and where two workgroups share one no piece is below 1.2 times that.
BATCHES = [
    (8, 1, 32, [1024] + [1] * 8, [9000] * 9, 4096, 4, False),
    (8, 1, 16, [512] + [1] * 5 + [0, 3], [6000, 9000, 1, 700, 2000, 2001, 0, 3], 2000, 0, False),
    (12, 4, 64, [700, 1, 1], [3000, 2999, 5000], 1000, 3, False),
    (8, 1, 32, [1024] * 6, [1600] * 6, 600, 4, True),                        # 192 blocks
    (8, 1, 32, [1024] * 5 + [992], [1600] * 6, 600, 4, False),               # 191
    (12, 3, 32, [1024] * 4, [1600] * 4, 600, 0, True),                       # 64 of each of 3 key heads
    (12, 3, 32, [1024] * 3 + [960], [1600] * 4, 600, 0, False),
    (8, 1, 16, [16] * 384, [800] * 384, 500, 4, True),                       # 384 of 512
    (8, 1, 16, [16] * 383 + [0] * 5, [800] * 388, 500, 4, True)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", BATCHES)
def test_walks_are_cut_by_the_blocks_that_have_rows(case, dtype):
    heads, kv, page, new, ctx, window, sinks, whole = case
    b = Windowed(7 + sum(new), heads, kv, page, dtype, new, ctx, window, sinks, behind=3)
    desc = cf.paged_desc(len(new), heads, b.total, max(new), max(ctx), b.table.shape[1], 0.1)
    assert 0 < cf.attn_paged_window_workspace_bytes(b.cache()[0], desc, cf.window(window, sinks)) <= WORKSPACE.numel()
    ref = b.definition()
    out, lse = b.run()
    check(out, lse, ref)
    again = b.run()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    cf.set_workspace(None)                                                   # not cut
    try:
        one = b.run()
    finally:
        cf.set_workspace(WORKSPACE)
    check(*one, ref)
    assert (torch.equal(one[0], out) and torch.equal(one[1], lse)) == whole


def test_replays_from_chunks_that_fill_the_chip_to_one_among_decoded_tokens():
    """One captured call, whose tables say with each replay whether walks are cut."""
    places, rows = 8, 8 * 1024
    b = Windowed(3, 8, 1, 32, "e4m3", [1024] * places, [1600] * places, 600, 4)
    b.table.copy_(b.whole)                                                   # (other lengths see other pages)
    out, lse = torch.zeros(rows, 8, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(8, rows, device=DEV)
    side = torch.cuda.Stream()
    cf.set_workspace(WORKSPACE, 0, side)
    try:
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.run(max_q=1024, max_kv=1600, stream=side, out=out, lse=lse)
        for new, ctx in (([1024] * 8, [1600] * 8), ([1024] + [1] * 7, [1600] * 8), ([1, 0, 900, 2, 1, 1, 0, 5], [1, 0, 1500, 70, 900, 1600, 9, 1200]),
                         ([1024] * 6 + [0, 1], [1300] * 8)):
            b.new, b.ctx = new, ctx
            b.starts.copy_(torch.tensor([sum(new[:i]) for i in range(places + 1)], dtype=torch.int32))
            b.lens.copy_(torch.tensor(ctx, dtype=torch.int32))
            out.fill_(-7), lse.fill_(-7)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            check(out, lse, b.definition())
            eager = b.run(max_q=1024, max_kv=1600)
            assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)
    finally:
        cf.set_workspace(None, 0, side)
