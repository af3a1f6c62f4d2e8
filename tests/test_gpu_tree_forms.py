"""Every form of the tree attention's kernels, by the shapes that take them
(tests/test_cache_dispatch.py checks that none is missing), against the binary64
form: few and many rows of each padded head width, sequences cut into parts and
joined by either join, and more sequences than a wavefront has lanes."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say
from tests.test_gpu_tree_attention import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def many(count, rows, longest):
    return [(i * 977 % longest, rows, rows) for i in range(count)] + [(longest, rows, rows)]


# name: shapes, query heads, key-value heads, channels
FORMS = {
    "64 x 1 token, 8 heads": ([(4001, 1, 1), (33, 1, 1)], 8, 8, 64),
    "64, 80 sequences": (many(79, 4, 1100), 16, 8, 64),
    "64, 32 rows": ([(900, 8, 8), (0, 5, 5), (2000, 1, 1)], 16, 4, 64),
    "64, 64 rows": ([(700, 16, 16), (64, 12, 12), (1300, 3, 3)], 8, 2, 64),
    "64, 200 rows": ([(800, 50, 50), (1, 40, 40)], 8, 2, 64),
    "128 x 1 token, 5 heads": ([(5000, 1, 1), (2, 1, 1), (640, 1, 1)], 20, 4, 128),
    "128, 80 sequences": (many(79, 4, 900), 8, 4, 128),
    "96, 28 rows": ([(1500, 4, 4), (95, 3, 3)], 14, 2, 96),
    "128, 60 rows": ([(1000, 15, 15), (257, 9, 9)], 8, 2, 128),
    "112, 200 rows": ([(600, 50, 50), (31, 20, 20)], 4, 1, 112),
    "128, 600 rows": ([(300, 150, 150), (0, 130, 130)], 4, 1, 128),
    "256 x 1 token": ([(3000, 1, 1), (17, 1, 1)], 4, 2, 256),
    "256, 80 sequences": (many(79, 4, 700), 4, 2, 256),
    "192, 90 rows": ([(500, 30, 30), (0, 17, 17)], 3, 1, 192),
}


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("name", FORMS)
def test_every_form(name, kind):
    shapes, q_heads, kv_heads, dim = FORMS[name]
    say(f"[gpu] tree attention {name}, type {kind}")
    for mask, window in (("tree", 0), ("none", 333)):
        b = Batch(shapes, q_heads, kv_heads, dim, 16, kind, mask=mask, window=window, seed=len(name), layers=1, layer=0)
        out, lse, _ = b.run(garbage=255)
        say(f"[gpu]   mask {mask} window {window}: worst {b.check(out, lse):.2f} of the bound")


def test_values_that_some_rows_must_not_see_in_every_form():
    # an infinity among the drafted values: who does not see it keeps its bits
    for name, (shapes, q_heads, kv_heads, dim) in FORMS.items():
        say(f"[gpu] unseen infinity, {name}")
        b = Batch(shapes, q_heads, kv_heads, dim, 16, mask="tree", branch=1, seed=3, layers=1, layer=0)
        at = [(s, n - 1) for s, (_, _, n) in enumerate(shapes) if n > 1]  # (seen by the last row only)
        for s, j in at:
            b.v[int(b.d_start[s]) + j] = 1.0
        clean, clean_lse, _ = b.run()
        b.check(clean, clean_lse)
        for s, j in at:
            b.v[int(b.d_start[s]) + j] = float("inf")
        out, lse, _ = b.run()
        hit = torch.zeros(out.shape[0], dtype=torch.bool)
        for s, j in at:
            hit[int(b.q_start[s + 1]) - 1] = True
        assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit]), name
        # (the others' weights are summed in another order: two fp32 sums of the bound's 2^-18)
        assert ((lse - clean_lse).abs() <= 2.0 ** -17 + 2.0 ** -21 * clean_lse.abs()).all(), name
        assert (out[hit] == float("inf")).all(), name
