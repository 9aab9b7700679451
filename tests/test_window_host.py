"""Attention with a sliding window without a GPU: what is refused, which kernels a call comes to, and the workspaces.  No kernel runs."""
import ctypes

import pytest

from paper_2604_24013_amd import binding as cf
from tests.dry import Dry

A, B, C, D, E, F, G, H, I, J, K, L = (0x10000 * i for i in range(1, 13))      # fake, aligned, never dereferenced


@pytest.fixture(scope="module")
def dry(tmp_path_factory):
    return Dry(str(tmp_path_factory.mktemp("dry")))


def status(f, *args):
    try:
        f(*args)
    except cf.CommFuseError as e:
        return e.status
    return cf.CF_OK


def _paged(dry_or_none, n, ctx, new, heads, kv, window, dtype="bf16", lse=None):
    desc = cf.paged_desc(n, heads, n * new, new, ctx, -(-ctx // 16), 0.1)
    args = cf.cache_desc(dtype, 4096, 16, kv), cf.make_cache(A, B, C, D), desc, window, E, F, G, H, I, lse
    if dry_or_none is None:
        return status(cf.attn_paged_window, *args)
    return dry_or_none.calls(lambda: cf.attn_paged_window(*args))


def test_struct_layout_matches_the_header():
    assert ctypes.sizeof(cf.Window) == 8 and cf.Window.sinks.offset == 4


@pytest.mark.parametrize("window, sinks, want", [(0, 0, cf.CF_ERR_INVALID_ARG), (-5, 0, cf.CF_ERR_INVALID_ARG), (4, -1, cf.CF_ERR_INVALID_ARG)])
def test_windows_are_refused(window, sinks, want):
    w, desc = cf.window(window, sinks), cf.prompt_desc(100, 1, 8, 1, 0.1)
    assert status(cf.attn_prompt_window, desc, w, A, B, C, D, E) == want
    assert status(cf.attn_prompt_window_grad, desc, w, A, B, C, D, E, F, G, H, I, J, K) == want
    assert _paged(None, 2, 500, 1, 8, 1, w) == want
    assert cf.attn_prompt_window_workspace_bytes(desc, w) == 0


def test_calls_are_refused_as_without_a_window():
    lib, desc, w = cf.load(), cf.prompt_desc(100, 1, 8, 1, 0.1), cf.window(10, 2)
    assert lib.commfuse_attn_prompt_window(desc, None, A, B, C, D, E, None, None) == cf.CF_ERR_NULL_PTR
    assert lib.commfuse_attn_prompt_window(None, w, A, B, C, D, E, None, None) == cf.CF_ERR_NULL_PTR
    assert lib.commfuse_attn_prompt_window_grad(desc, None, A, B, C, D, E, F, G, H, I, J, K, None) == cf.CF_ERR_NULL_PTR
    assert lib.commfuse_attn_prompt_window_workspace_bytes(desc, None) == 0 and lib.commfuse_attn_prompt_window_workspace_bytes(None, w) == 0
    full = [A, B, C, D, E]
    for i in range(5):
        args = list(full)
        args[i] = None
        assert status(cf.attn_prompt_window, desc, w, *args) == cf.CF_ERR_NULL_PTR
        args[i] = A + 2
        assert status(cf.attn_prompt_window, desc, w, *args) == cf.CF_ERR_MISALIGNED
    assert status(cf.attn_prompt_window, desc, w, A, B, C, D, A) == cf.CF_ERR_INVALID_ARG            # out over Q
    assert status(cf.attn_prompt_window, cf.prompt_desc(100, 1, 8, 1, 0.1, head_dim=64), w, *full) == cf.CF_ERR_UNSUPPORTED
    assert status(cf.attn_prompt_window, cf.prompt_desc(100, 1, 8, 3, 0.1), w, *full) == cf.CF_ERR_INVALID_ARG
    assert status(cf.attn_prompt_window, cf.prompt_desc(0, 1, 8, 1, 0.1), w, *full) == cf.CF_OK
    assert status(cf.attn_prompt_window_grad, desc, w, A, B, C, D, E, F, G, H, I, J, J) == cf.CF_ERR_INVALID_ARG
    assert status(cf.attn_paged_window, cf.cache_desc("bf16", 8, 16, 1, 64), cf.make_cache(A, B), cf.paged_desc(1, 8, 1, 1, 64, 4, 0.1), w, C, D, E, F, G) == cf.CF_ERR_UNSUPPORTED


def test_a_window_that_hides_nothing_takes_the_causal_kernels(dry):
    desc = cf.prompt_desc(1000, 2, 8, 1, 0.1)
    causal = dry.calls(lambda: cf.attn_prompt(desc, A, B, C, D, E))
    for w in ((1000, 0), (990, 10), (1, 999), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert dry.calls(lambda: cf.attn_prompt_window(desc, cf.window(*w), A, B, C, D, E)) == causal
    for w in ((999, 0), (990, 9), (1, 998)):
        assert dry.calls(lambda: cf.attn_prompt_window(desc, cf.window(*w), A, B, C, D, E)) != causal
    desc2 = cf.paged_desc(4, 8, 4, 1, 500, 32, 0.1)
    pool = cf.cache_desc("bf16", 64, 16, 1), cf.make_cache(A, B)
    causal = dry.calls(lambda: cf.attn_paged(*pool, desc2, C, D, E, F, G))
    assert dry.calls(lambda: cf.attn_paged_window(*pool, desc2, cf.window(496, 4), C, D, E, F, G)) == causal
    assert dry.calls(lambda: cf.attn_paged_window(*pool, desc2, cf.window(496, 3), C, D, E, F, G)) != causal
    grads = [dry.calls(lambda: f(desc, *w, A, B, C, D, E, F, G, H, I, J, K)) for f, w in
             ((cf.attn_prompt_grad, ()), (cf.attn_prompt_window_grad, (cf.window(1000, 0),)), (cf.attn_prompt_window_grad, (cf.window(999, 0),)))]
    assert grads[0] == grads[1] != grads[2]


def test_few_rows_and_many(dry):
    w = cf.window(100, 4)
    for new, heads, few in ((1, 8, True), (4, 8, True), (5, 8, False), (1, 32, True), (32, 1, True), (33, 1, False)):
        (name, _, _), = _paged(dry, 3, 5000, new, heads, 1, w)
        assert ("attn_few" in name) == few and "true" in name


def test_workspaces_hold_what_the_plan_parks():
    """A window needs no more room than the same call without one, and none where its walks are too short to be split."""
    for tokens, heads, kv in ((4096, 8, 1), (8192, 4, 4), (700, 2, 1)):
        desc = cf.prompt_desc(tokens, 1, heads, kv, 0.1)
        assert 0 <= cf.attn_prompt_window_workspace_bytes(desc, cf.window(256, 0)) <= cf.attn_prompt_workspace_bytes(desc)
        assert cf.attn_prompt_window_workspace_bytes(desc, cf.window(tokens, 0)) == cf.attn_prompt_workspace_bytes(desc)
    pool, desc = cf.cache_desc("e4m3", 5000, 64, 1), cf.paged_desc(4, 8, 4, 1, 100000, 2000, 0.1)
    assert cf.attn_paged_window_workspace_bytes(pool, desc, cf.window(128, 4)) == 0
    assert 0 < cf.attn_paged_window_workspace_bytes(pool, desc, cf.window(4096, 4)) <= cf.attn_paged_workspace_bytes(pool, desc)
