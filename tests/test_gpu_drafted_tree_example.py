"""examples/drafted_tree.py runs: predictor, codec and cache together."""
from __future__ import annotations

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rounds_of_drafted_trees():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("drafted_tree", os.path.join(ROOT, "examples", "drafted_tree.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    share, nmse = M.main(hidden=1024, model=128, groups=3, beams=2, branch=3, depth=2, rounds=3, window=8)
    # 4 bits, a scale and a coefficient pair for every 128 channels; the residual's quantization noise
    assert 0.25 < share < 0.35 and nmse < 0.02
