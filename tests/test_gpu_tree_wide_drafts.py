"""Drafted keys and values whose rows lie far apart, so that a sequence's span
4 GiB and more: the same bits as from rows that lie together."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

STRIDE, DRAFTS = 1 << 25, 70  # the widest there is; 70 rows of 64 MiB


@pytest.fixture(scope="module")
def far():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()
    return torch.empty(DRAFTS * STRIDE, dtype=torch.int16, device="cuda").view(DRAFTS, STRIDE)


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("rows,dim", [(1, 64), (70, 64), (1, 128), (70, 128)])
def test_drafts_that_span_more_than_4_gib(far, kind, rows, dim):
    say(f"[gpu] {rows} rows over {DRAFTS} drafts {2 * STRIDE >> 20} MiB apart, {dim} channels, type {kind}")
    gen = torch.Generator(device="cuda").manual_seed(dim + rows)
    act, heads = R.ACT[kind], 2
    k, v = (torch.randn(DRAFTS, heads, dim, device="cuda", generator=gen).to(act) for _ in range(2))
    q = torch.randn(rows, heads, dim, device="cuda", generator=gen).to(act)
    wide_k = far[:, :heads * dim].view(act).unflatten(1, (heads, dim))
    wide_v = far[:, heads * dim:2 * heads * dim].view(act).unflatten(1, (heads, dim))
    wide_k.copy_(k)
    wide_v.copy_(v)
    assert wide_k.stride() == (STRIDE, dim, 1)
    cfg = rac.CacheConfig(1, heads, dim, 16, 4, 1, 4, kind)
    tree = rac.TreeConfig(heads, rows, rows, DRAFTS)
    pool = torch.zeros(rac.rac_cache_pool_bytes(cfg), dtype=torch.uint8, device="cuda")
    table, lengths, _ = rac.rac_cache_new(cfg)
    start = lambda n: torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ws = torch.empty(rac.rac_tree_attention_workspace(cfg, tree), dtype=torch.uint8, device="cuda")
    got = []
    for a, b in ((k, v), (wide_k, wide_v)):
        out = torch.empty(rows, heads, dim, dtype=act, device="cuda")
        rac.rac_tree_attention(cfg, tree, 0, pool, table, lengths, q, start(rows), a, b, out, ws,
                               draft_start=start(DRAFTS))
        torch.cuda.synchronize()
        got.append(out.cpu())
    assert torch.isfinite(got[0]).all() and torch.equal(*got)
