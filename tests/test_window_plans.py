"""Which batches over the paged cache have their walks cut when a window hides part of them, without a GPU: no kernel runs."""
import pytest

from paper_2604_24013_amd import binding as cf
from tests.dry import Dry

A, B, C, D, E, F, G, H, I, J = (0x10000 * i for i in range(1, 11))      # fake, aligned, never dereferenced


@pytest.fixture(scope="module")
def dry(tmp_path_factory):
    return Dry(str(tmp_path_factory.mktemp("dry")))


def _calls(dry, pool, desc, window, room):
    """Kernels and workgroups of the call with a window, and of the one without."""
    cache = cf.make_cache(A, B, C, D)
    args = E, F, G, H, I, None

    def run():
        cf.set_workspace(J, room)
        try:
            cf.attn_paged_window(pool, cache, desc, window, *args)
            cf.attn_paged(pool, cache, desc, *args)
        finally:
            cf.set_workspace(None)

    (name, wgs, _), (other, plain, _) = [c for c in dry.calls(run) if "attn" in c[0]]
    return wgs, plain, name, other


MIXED = [  # new tokens, cached tokens, heads, key heads, window, first tokens, rows that there may be
    ([1024] + [1] * 8, 9000, 8, 1, 4096, 0, None), ([1024] + [1] * 5, 32768, 8, 1, 4096, 4, None), ([512] + [1] * 15, 30000, 8, 1, 8192, 0, None),
    ([1500] + [1] * 3, 9000, 16, 2, 4096, 4, None), ([1500] + [1] * 3, 9000, 12, 4, 4096, 4, None), ([1024] + [1] * 8, 9000, 8, 1, 4096, 4, 8192),
    ([700, 0, 0, 0, 0, 0, 0, 1], 20000, 8, 1, 2000, 1, 6000), ([40] + [1] * 30, 20000, 8, 1, 2000, 0, None)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("case", MIXED)
def test_a_chunk_among_decoded_tokens_is_cut_as_without_a_window(dry, case, dtype):
    """`max_q` rows for every sequence are many more blocks than have rows: they do not keep the walks of those that have whole."""
    new, ctx, heads, kv, window, sinks, total = case
    pool, w = cf.cache_desc(dtype, 4096, 16, kv), cf.window(window, sinks)
    desc = cf.paged_desc(len(new), heads, total or sum(new), max(new), ctx, -(-ctx // 16), 0.1)
    plain = cf.attn_paged_workspace_bytes(pool, desc)
    assert plain > 0 and cf.attn_paged_window_workspace_bytes(pool, desc, w) == plain
    with_window, without, name, other = _calls(dry, pool, desc, w, plain)
    assert "attn_blocks" in name and "attn_blocks" in other and with_window == without
    whole = _calls(dry, pool, desc, w, 65792)                            # (room for nothing that is parked)
    assert with_window > whole[0]


def test_walks_too_short_to_be_cut_ask_for_nothing():
    pool = cf.cache_desc("bf16", 4096, 16, 1)
    desc = cf.paged_desc(9, 8, 1032, 1024, 9000, 563, 0.1)
    assert cf.attn_paged_workspace_bytes(pool, desc) > cf.attn_paged_window_workspace_bytes(pool, desc, cf.window(40, 4)) == 0


@pytest.mark.parametrize("tokens, heads, kv", [(131072, 8, 1), (32768, 32, 4)])
def test_walks_of_first_keys_ask_for_room_of_their_own(tokens, heads, kv):
    """In the gradient a sequence's first keys are seen to its end.  Their walks are cut where blocks of keys are too many for the call without a window, and
    for the one without first tokens, to be cut at all: up to 2048 blocks of 128 keys."""
    desc = cf.prompt_desc(tokens, 1, heads, kv, 0.1)
    assert cf.attn_prompt_workspace_bytes(desc) == cf.attn_prompt_window_workspace_bytes(desc, cf.window(1024, 0)) == 0
    assert cf.attn_prompt_window_workspace_bytes(desc, cf.window(1024, 4)) > 0


def test_beyond_2048_blocks_of_keys_nothing_is_cut():
    for tokens, cut in ((2048 * 128, True), (2048 * 128 + 1, False)):
        assert (cf.attn_prompt_window_workspace_bytes(cf.prompt_desc(tokens, 1, 8, 1, 0.1), cf.window(1024, 4)) > 0) == cut
