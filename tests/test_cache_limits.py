"""Sizes that a call of include/rac_cache.h does not take, as the header states
them, refused before any launch."""
from __future__ import annotations

import ctypes

import pytest

import paper_2608_04991_amd as rac
from paper_2608_04991_amd import cache
from tests.test_cache_abi import P, lib  # noqa: F401

UNSUPPORTED = 6  # RAC_ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,q_heads", [(1 << 20, 64), (1 << 16, 1024), ((1 << 20) - 1, 65)])
def test_rows_and_heads_beyond_the_counts(lib, rows, q_heads):  # noqa: F811
    cfg = rac.CacheConfig(1, q_heads, 16, 16, 100, 8, 10)
    ok, many = (rac.TreeConfig(q_heads, n, n, 5) for n in ((1 << 26) // q_heads - 1, rows))
    assert rac.rac_tree_attention_workspace(cfg, ok) > 0
    assert rac.rac_tree_attention_workspace(cfg, many) == 0
    t = cache._TreeTensors(q=P, k=None, v=None, q_start=P, draft_start=None, mask=None, out=P, lse=None,
                           q_stride=16 * q_heads, kv_stride=0, out_stride=16 * q_heads, draft_rows=0, mask_words=0)
    assert lib.rac_tree_attention(cfg._ref, many._ref, 0, P, P, P, ctypes.byref(t), P, 1 << 40, 0) == UNSUPPORTED


def test_copies_of_more_than_2_to_the_24_pieces(lib):  # noqa: F811
    small = rac.CacheConfig(1, 1, 16, 8, 1 << 24, 1, 1)        # a piece each
    large = rac.CacheConfig(64, 8, 128, 64, 1 << 20, 1, 1)     # 1024 pieces each
    for cfg, n in ((small, 1 << 24), (large, 1 << 14)):
        assert lib.rac_cache_copy(cfg._ref, P, P, P, P, n, 0) == UNSUPPORTED
