"""Attention weights in a cache of as many sequences as there may be."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say
from tests.test_gpu_tree_attention import Batch
from tests.test_gpu_weights import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [R.BF16, R.FP8])
@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("rows", [1, 20, 70], ids=["alone", "shared", "many"])
def test_4096_sequences(kind, dim, rows):
    """Most of them without rows; the beginnings of all take 32 KiB of LDS beside the tiles."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()
    say(f"[gpu] weights of 4096 sequences, {dim} channels, up to {rows} rows, type {kind}")
    shapes = [(5 * s % 37, rows if s % 1365 == 0 else 0, rows if s % 1365 == 0 else 0) for s in range(4096)]
    b = Batch(shapes, 2, 2, dim, 8, kind, mask="tree", seed=rows, layers=1, layer=0)
    check(b)
    check(b, True)
