"""Checks, without a GPU, of the weights of cached tokens and of eviction: sizes, and
refusals, which come before any launch."""
from __future__ import annotations

import copy
import ctypes
import dataclasses
import pickle

import pytest

import paper_2608_04991_amd as rac
from paper_2608_04991_amd import cache
from tests.test_cache_abi import CFG, P, TREE, _Fake as F, lib  # noqa: F401

EVICT = rac.EvictConfig(8, 4, 16)
POSITIONS = CFG.max_pages * CFG.page_tokens


def weigh(lib, cfg=CFG, tree=TREE, layer=0, sets=8, pool=P, table=P, lengths=P, weight=P, draft=P, ws=P, cap=1 << 40, **change):  # noqa: F811
    t = dict(q=P, k=P, v=None, q_start=P, draft_start=None, mask=P, out=None, lse=P, q_stride=512, kv_stride=256, out_stride=0,
             draft_rows=20, mask_words=1)
    t.update(change)
    return lib.rac_tree_weights(cfg._ref, tree._ref, layer, sets, pool, table, lengths, ctypes.byref(cache._TreeTensors(**t)),
                                weight, draft, ws, cap, None)


def test_weights_refusals(lib):  # noqa: F811
    assert rac.rac_tree_weights_workspace(CFG, TREE) > 0
    for bad in (dict(layer=-1), dict(layer=2), dict(sets=0), dict(sets=2), dict(sets=4), dict(pool=None), dict(table=None),
                dict(lengths=None), dict(ws=None), dict(weight=None), dict(lse=None), dict(q=None), dict(q_start=None),
                dict(q_stride=504), dict(q_stride=516), dict(kv_stride=248), dict(kv_stride=260), dict(kv_stride=(1 << 25) + 8),
                dict(draft_rows=-1), dict(mask_words=-1), dict(mask=None), dict(mask_words=0),
                dict(tree=dataclasses.replace(TREE, q_heads=6)), dict(tree=dataclasses.replace(TREE, scale=-1.0)),
                dict(cfg=dataclasses.replace(CFG, head_dim=72))):
        assert weigh(lib, **bad) == 1, bad
    for bad in (dict(pool=P + 8), dict(table=P + 2), dict(lengths=P + 1), dict(ws=P + 128), dict(weight=P + 2), dict(draft=P + 2),
                dict(lse=P + 2), dict(q=P + 8), dict(k=P + 8), dict(q_start=P + 2), dict(draft_start=P + 2), dict(mask=P + 4)):
        assert weigh(lib, **bad) == 2, bad
    assert weigh(lib, cap=rac.rac_tree_weights_workspace(CFG, TREE) - 1) == 3
    wide = dataclasses.replace(CFG, page_tokens=256, max_pages=1 << 22, seqs=64)
    assert weigh(lib, cfg=wide, sets=1) == 6 and rac.rac_cache_evict_workspace(wide, rac.EvictConfig()) == 0
    many = dataclasses.replace(TREE, rows=1 << 20, q_heads=64)
    assert weigh(lib, tree=many, q_stride=64 * 64) == 6 and rac.rac_tree_weights_workspace(CFG, many) == 0
    assert weigh(lib, tree=dataclasses.replace(TREE, rows=0), q=None, weight=None) == 0


def evict(lib, cfg=CFG, e=EVICT, pool=P, table=P, lengths=P, refs=P, weight=P, keep=P, evicted=P, source=P, ws=P, cap=1 << 40):  # noqa: F811
    return lib.rac_cache_evict(cfg._ref, e._ref, pool, table, lengths, refs, weight, keep, evicted, source, ws, cap, None)


def test_evict_refusals(lib):  # noqa: F811
    need = rac.rac_cache_evict_workspace(CFG, EVICT)
    assert need >= 8 * 8 * POSITIONS * 4
    for bad in (dict(sets=0), dict(sets=2), dict(first=-1), dict(recent=-1), dict(first=(1 << 30) + 1), dict(recent=(1 << 30) + 1)):
        e = dataclasses.replace(EVICT, **bad)
        assert evict(lib, e=e) == 1 and rac.rac_cache_evict_workspace(CFG, e) == 0
    for name in ("pool", "table", "lengths", "refs", "weight", "keep", "evicted", "ws"):
        assert evict(lib, **{name: None}) == 1, name
    for name in ("pool", "table", "lengths", "refs", "weight", "keep", "evicted", "source"):
        assert evict(lib, **{name: P + (8 if name == "pool" else 2)}) == 2, name
    assert evict(lib, ws=P + 128) == 2 and evict(lib, cap=need - 1) == 3
    assert evict(lib, cfg=dataclasses.replace(CFG, pages=0)) == 1


def test_weights_commit_refusals(lib):  # noqa: F811
    def call(sets=8, lengths=P, committed=P, start=P, path=P, max_path=5, draft=P, rows=20, weight=P, cfg=CFG):
        return lib.rac_cache_weights_commit(cfg._ref, sets, lengths, committed, start, path, max_path, draft, rows, weight, None)

    for bad in (dict(sets=3), dict(lengths=None), dict(committed=None), dict(start=None), dict(max_path=-1), dict(rows=-1),
                dict(weight=None), dict(cfg=dataclasses.replace(CFG, seqs=0))):
        assert call(**bad) == 1, bad
    for bad in (dict(lengths=P + 2), dict(committed=P + 2), dict(start=P + 2), dict(path=P + 2), dict(draft=P + 2), dict(weight=P + 2)):
        assert call(**bad) == 2, bad


def test_binding_checks_tensors_before_the_call(lib, monkeypatch):  # noqa: F811
    called = []
    names = ("rac_tree_weights", "rac_cache_weights_commit", "rac_cache_evict")
    fake = type("L", (), {n: (lambda *a: called.append(a) or 0) for n in names})()
    for n in ("rac_cache_pool_bytes", "rac_tree_weights_workspace", "rac_cache_evict_workspace"):
        setattr(fake, n, getattr(lib, n))
    monkeypatch.setattr(rac, "library", lambda: fake)
    pool, table, lengths = F((rac.rac_cache_pool_bytes(CFG) // 2,)), F((8, 10), 4), F((8,), 4)
    weight = F((8, 8, POSITIONS), 4)
    weigh = lambda **bad: rac.rac_tree_weights(CFG, TREE, 0, **{**dict(
        pool=pool, table=table, lengths=lengths, q=F((20, 8, 64)), q_start=F((9,), 4), k=F((20, 4, 64)), lse=F((20, 8), 4),
        weight=weight, workspace=F((1 << 30,), 1), draft_weight=F((8, 20), 4), mask=F((20, 1), 8), stream=0), **bad})
    weigh()
    weigh(weight=F((8, 1, POSITIONS), 4), draft_weight=F((1, 20), 4))
    assert [a[4] for a in called] == [8, 1]
    for bad in (dict(weight=P), dict(weight=F((8, 2, POSITIONS), 4)), dict(weight=F((7, 8, POSITIONS), 4)),
                dict(weight=F((8, 8, POSITIONS + 1), 4)), dict(weight=F((8, 8, POSITIONS), 2)), dict(weight=F((8, 8, POSITIONS), 4, cuda=False)),
                dict(draft_weight=F((1, 20), 4)), dict(draft_weight=F((8, 19), 4)), dict(draft_weight=P), dict(k=P), dict(mask=P),
                dict(lse=F((19, 8), 4)), dict(q=F((19, 8, 64))), dict(workspace=F((5,), 1)), dict(table=F((8, 9), 4))):
        with pytest.raises(ValueError):
            weigh(**bad)
    commit = lambda **bad: rac.rac_cache_weights_commit(CFG, **{**dict(
        lengths=lengths, committed=F((8,), 4), draft_start=F((9,), 4), draft_weight=F((8, 20), 4), weight=weight,
        path=F((8, 5), 4), stream=0), **bad})
    commit()
    assert called[-1][7] == 5 and called[-1][9] == 20
    commit(path=None)
    assert called[-1][7] == 20
    for bad in (dict(path=P), dict(path=F((8, 4), 4), max_path=5), dict(draft_weight=F((7, 20), 4)), dict(committed=F((7,), 4)),
                dict(draft_start=F((8,), 4)), dict(draft_rows=19)):
        with pytest.raises(ValueError):
            commit(**bad)
    cut = lambda **bad: rac.rac_cache_evict(CFG, EVICT, **{**dict(
        pool=pool, table=table, lengths=lengths, refs=F((100,), 4), weight=weight, keep=F((8,), 4), evicted=F((8,), 4),
        workspace=F((1 << 30,), 1), source=F((8, 8, POSITIONS), 4), stream=0), **bad})
    cut()
    for bad in (dict(weight=F((8, 1, POSITIONS), 4)), dict(refs=F((99,), 4)), dict(keep=F((7,), 4)), dict(evicted=F((8,), 8)),
                dict(source=F((8, 1, POSITIONS), 4)), dict(workspace=F((64,), 1)), dict(pool=F((100,)))):
        with pytest.raises(ValueError):
            cut(**bad)
    assert len(called) == 5


def test_configurations_can_be_copied_and_pickled_after_use(lib):  # noqa: F811
    rac.rac_cache_evict_workspace(CFG, EVICT)
    rac.rac_tree_weights_workspace(CFG, TREE)
    for c in (EVICT, TREE):
        assert copy.deepcopy(c) == c and pickle.loads(pickle.dumps(c)) == c
