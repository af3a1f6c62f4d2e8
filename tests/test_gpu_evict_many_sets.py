"""Eviction with as many sets as a deep model has layers and heads, and with last tokens
that take many steps to shift, against the contract's words."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests.gpu_util import say
from tests.test_gpu_evict import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


@pytest.mark.parametrize("page", [8, 64])
def test_a_set_for_every_head_of_many_layers(page):
    """384 sets over shared pages: those at the front change in no set, others in some, most in
    all; then with sequences whose first pages are gone."""
    layers, heads = 48, 8
    for gaps in ((), ((0, 0), (1, 1))):
        say(f"[gpu] evict {layers * heads} sets, pages of {page}, gaps {gaps}")
        c = Cache([200, 200, 200, 150], page, layers, heads, 16, rac.RAC_CACHE_FP8, 2, share=((1, 0), (2, 0)), gaps=gaps,
                  spare=60, seed=page)
        c.weight[1] = torch.arange(c.weight.shape[2]).float()        # (every set lets the first ones go)
        c.weight[2, :, :] = -torch.arange(c.weight.shape[2]).float()  # (and the last ones)
        c.weight[2, 383, 65:90] = -1000.0                            # (but for one set)
        c.upload()
        c.evict([-1, 130, 140, 149], 4, 6)
        c.evict([60, 100, 139, 20], 0, 30)


@pytest.mark.parametrize("dim,kind", [(256, rac.RAC_CACHE_BF16), (80, rac.RAC_CACHE_FP16), (16, rac.RAC_CACHE_FP8)])
@pytest.mark.parametrize("sets", [1, 2])
def test_long_last_tokens_that_shift_by_few(dim, kind, sets):
    """Fewer tokens go than the last ones are: every step reads what the one before it is about
    to write, or what lies beside it."""
    for by in (1, 15, 16, 17, 300):
        say(f"[gpu] evict {by} tokens ahead of 1300 last ones, {dim} channels, sets {sets}")
        lengths = [1500, 1304 + by, 40, 1300]
        Cache(lengths, 32, 1, 2, dim, kind, sets, share=((3, 0),), spare=60, seed=by).evict(
            [n - min(by, n) for n in lengths], 3, 1300)
