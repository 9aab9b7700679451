"""How many bytes of workspace the causal attention asks for, without a GPU: the sizes with which walks over the keys are split."""
import pytest

from paper_2604_24013_amd import binding as cf


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import os
    if not os.path.exists(cf.LIB_PATH):
        from paper_2604_24013_amd import build
        build.build()
    cf.load()


def paged(n, max_q, max_kv=65536, heads=8, kv=1, dtype="bf16", page=16):
    return cf.attn_paged_workspace_bytes(cf.cache_desc(dtype, 9, page, kv), cf.paged_desc(n, heads, n * max_q, max_q, max_kv, -(-max_kv // page), 0.1))


@pytest.mark.parametrize("max_q", [1, 4, 5])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_batches_of_more_than_64_sequences_ask_for_a_workspace(max_q, dtype):
    """A split's share: rows of 132 floats (16 or 32 of them) of the few-rows kernel, 128 rows' of the other."""
    for n in (1, 64, 65, 100, 255, 256, 511, 512):
        assert paged(n, max_q, dtype=dtype) >= 65536 + n * 16 * 132 * 4, n
    assert paged(513, max_q, dtype=dtype) == 0                                # more blocks than are looked at


def test_what_is_asked_for_does_not_fall_as_contexts_grow():
    for n in (1, 63, 64, 65, 66, 200, 512):
        sizes = [paged(n, 1, 1 << b) for b in range(4, 20)]
        assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[-1] > 0


def test_walks_that_32_bits_do_not_count_are_not_split():
    """The kernels add up the tiles of all walks (of 32 or 64 keys) in 32 bits.  Beyond that a batch is not split: 512 sequences that share pages
    may see 2^31 tokens each."""
    for max_q, tile in ((1, 32), (5, 64)):
        for n in (2, 64, 512):
            tokens = min((2 ** 31 - 1) // n * tile, 2 ** 31 - 2 ** 14) // 1024 * 1024
            assert paged(n, max_q, tokens, page=1024) > 0
            if (2 ** 31 - 1) // n * tile < 2 ** 31 - 2 ** 14:
                assert paged(n, max_q, tokens + 1024 * tile, page=1024) == 0


@pytest.mark.parametrize("which", ["in_dtype", "out_dtype"])
def test_e4m3_is_for_cache_pages_only(which):
    """The projections refuse it."""
    desc = cf.layer_desc(2, 0, 16, 256, 256, **{which: "e4m3"})
    for call in (lambda: cf.ag_step(desc, 0, 0x10000, 0x20000, 0x30000), lambda: cf.rs_step(desc, 0, 0x10000, 0x20000, 0x30000, 0x40000)):
        with pytest.raises(cf.CommFuseError) as refused:
            call()
        assert refused.value.status == cf.CF_ERR_UNSUPPORTED
