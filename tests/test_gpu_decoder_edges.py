"""Causal attention over packed prompts, its gradient and the paged cache where workspaces, numbers of sequences and values that are not
finite take paths of their own.  Needs an MI355X: ``-m gpu``.  Limits are those of the files that test each operator alone."""
import math
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests import test_gpu_attn_grad as grad
from tests import test_gpu_attn_prompt as prompt
from tests.test_gpu_attn_paged import Batch
from tests.test_gpu_attn_paged import check as check_paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
SCALE = 1 / math.sqrt(D)
WORKSPACE = None


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    global WORKSPACE
    cf.load()
    WORKSPACE = torch.empty(256 << 20, dtype=torch.uint8, device=DEV)
    cf.set_workspace(WORKSPACE)
    yield
    torch.cuda.synchronize()
    cf.set_workspace(None)
    WORKSPACE = None


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("n, new", [(64, 1), (65, 1), (200, 1), (65, 3), (66, 30)])
def test_large_batches_in_the_workspace_that_they_ask_for(n, new, dtype):
    """One long context among short ones, in exactly the bytes asked for, with a guard behind."""
    ctx = [new + (i * 7) % 40 for i in range(n)]
    ctx[n // 2] += 6000
    b = Batch(300 + n, 8, 1, 16, dtype, [new] * n, ctx)
    ask = cf.attn_paged_workspace_bytes(b.cache()[0], cf.paged_desc(n, 8, b.total, new, max(ctx), b.table.shape[1], SCALE))
    assert ask > 64 << 10
    buf = torch.full((ask + (1 << 20),), 85, dtype=torch.uint8, device=DEV)
    cf.set_workspace(buf[:ask])
    try:
        check_paged(*b.run(), b.definition())
        assert bool((buf[ask:] == 85).all())
        assert bool((buf[64 << 10:ask] != 85).any())                          # keys were split
    finally:
        torch.cuda.synchronize()
        cf.set_workspace(WORKSPACE)
