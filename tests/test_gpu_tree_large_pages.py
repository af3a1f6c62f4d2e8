"""Pages of 64 GiB (many layers and heads): the second page of a pool is read
from where it lies."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

LAYERS, HEADS, PAGE, DIM = 1024, 512, 128, 256


@pytest.fixture(scope="module")
def pool():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()
    cfg = rac.CacheConfig(LAYERS, HEADS, DIM, PAGE, 2, 1, 1, R.BF16)
    need = rac.rac_cache_pool_bytes(cfg)
    assert need == 2 << 36
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip("128 GiB of device memory are not free")
    pool = torch.empty(2, LAYERS, 2, HEADS, PAGE, DIM, dtype=torch.bfloat16, device="cuda")
    yield cfg, pool
    del pool
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows", [1, 80])
@pytest.mark.parametrize("layer", [0, LAYERS - 1])
def test_the_second_of_two_pages_of_64_gib(pool, rows, layer):
    cfg, pool = pool
    say(f"[gpu] pages of 64 GiB, layer {layer}, {rows} rows")
    gen = torch.Generator(device="cuda").manual_seed(rows + layer)
    pool[0, layer].fill_(float("nan"))
    pool[1, layer].copy_(torch.randn(2, HEADS, PAGE, DIM, device="cuda", generator=gen))
    q = torch.randn(rows, HEADS, DIM, device="cuda", generator=gen).bfloat16()
    outs = []
    # (and the same in a cache of one layer)
    for c, held, at in ((cfg, pool, layer), (rac.CacheConfig(1, HEADS, DIM, PAGE, 2, 1, 1, R.BF16),
                                             pool[:, layer:layer + 1].contiguous(), 0)):
        tree = rac.TreeConfig(HEADS, rows, rows, 0)
        ws = torch.empty(rac.rac_tree_attention_workspace(c, tree), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
        rac.rac_tree_attention(c, tree, at, held, i32(1).view(1, 1), i32(100), q, i32(0, rows), None, None, out, ws)
        torch.cuda.synchronize()
        outs.append(out.cpu())
    assert torch.isfinite(outs[0]).all() and torch.equal(*outs)
