"""What the binding of the paged cache does with its arguments, without a GPU: a
library that records the calls, and tensors without memory."""
from __future__ import annotations

import copy
import dataclasses
import pickle

import pytest

import paper_2608_04991_amd as rac
from tests.test_cache_abi import CFG, P, TREE, _Fake as F, lib  # noqa: F401

PRED = rac.PredictorConfig(512, 128, 2, 256, 16, 8)
PRED_CACHE, PRED_TREE = rac.CacheConfig(1, 2, 64, 16, 20, 4, 5), rac.TreeConfig(2, 6, 3, 3, 16)


@pytest.fixture
def calls(lib, monkeypatch):  # noqa: F811
    """The arguments of every call that reaches the library."""
    called = []
    fake = type("L", (), {})()
    for name in ("rac_tree_attention", "rac_cache_commit", "rac_predictor_tree_step"):
        setattr(fake, name, lambda *a, name=name: called.append((name, a)) or 0)
    for name in ("rac_cache_pool_bytes", "rac_tree_attention_workspace", "rac_cache_commit_workspace",
                 "rac_predictor_tree_workspace"):
        setattr(fake, name, getattr(lib, name))
    monkeypatch.setattr(rac, "library", lambda: fake)
    return called


def attend(**change):
    a = dict(pool=P, table=P, lengths=P, q=F((20, 8, 64)), q_start=P, k=F((20, 4, 64)), v=F((20, 4, 64)),
             out=F((20, 8, 64)), workspace=P, mask=None)
    a.update(change)
    mask = a.pop("mask")
    rac.rac_tree_attention(CFG, TREE, 0, *a.values(), mask=mask, stream=0)


def step(**change):
    a = dict(weights=P, pool=P, table=P, lengths=P, q_start=P, draft_start=P, slot=P, pos=P, h_prev=P,
             draft_k=F((9, 2, 64)), draft_v=F((9, 2, 64)), ref_out=P, workspace=P, mask=None)
    a.update(change)
    mask = a.pop("mask")
    rac.rac_predictor_tree_step(PRED, PRED_CACHE, PRED_TREE, *a.values(), mask=mask, stream=0)


def test_drafted_keys_and_values_are_counted(calls):
    attend()
    attend(q=P, out=P)
    attend(k=None, v=None)
    step()
    tensors = [a[6]._obj for name, a in calls[:3]]
    assert [t.draft_rows for t in tensors] == [20, 20, 0] and calls[3][1][16] == 9


@pytest.mark.parametrize("names", [("k",), ("v",), ("k", "v")])
def test_addresses_of_drafts_are_refused(calls, names):
    # (their rows are unknown: the drafted tokens would be left out)
    with pytest.raises(ValueError, match="address"):
        attend(**{n: P for n in names})
    with pytest.raises(ValueError, match="address"):
        step(**{"draft_" + n: P for n in names})
    assert not calls


def test_an_address_of_a_mask_is_refused(calls):
    # (it was taken as the number of a row's words)
    attend(mask=F((20, 2), 8))
    assert calls[0][1][6]._obj.mask_words == 2
    for call in (attend, step):
        with pytest.raises(ValueError, match="address"):
            call(mask=P)
    assert len(calls) == 1


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x))],
                         ids=["copy", "deepcopy", "pickle"])
def test_configurations_are_copied_after_their_use(lib, again):  # noqa: F811
    cfg, tree = rac.CacheConfig(2, 4, 64, 16, 100, 8, 10, 2, 0.5, 0.25), rac.TreeConfig(8, 20, 5, 5, 7, 0.5)
    sizes = lambda c, t: (rac.rac_cache_pool_bytes(c), rac.rac_cache_commit_workspace(c),
                          rac.rac_tree_attention_workspace(c, t))
    want = sizes(cfg, tree)
    c, t = again(cfg), again(tree)
    assert c == cfg and t == tree and c._ref._obj is not cfg._ref._obj and t._ref._obj is not tree._ref._obj
    assert sizes(c, t) == want and bytes(c._c()) == bytes(cfg._c()) and bytes(t._c()) == bytes(tree._c())


def test_rows_of_a_path(calls):
    kv = F((2, 20, 4, 64))
    commit = lambda path, **kw: rac.rac_cache_commit(CFG, P, P, P, P, kv, kv, P, P, P, path=path, stream=0, **kw)
    commit(F((8, 5), 4))
    commit(F((8, 5), 4), max_path=5)
    commit(F((40,), 4), max_path=5)
    commit(P, max_path=3)
    commit(None)
    commit(None, max_path=7)
    one = lambda path, **kw: rac.rac_cache_commit(dataclasses.replace(CFG, seqs=1), P, P, P, P, kv, kv, P, P, P, path=path,
                                                  stream=0, **kw)
    one(F((5,), 4))
    one(F((1, 5), 4), max_path=3)  # (the first entries of one row)
    assert [a[12] for _, a in calls] == [5, 5, 5, 3, 20, 7, 5, 3]
    for path, kw in ((F((8, 5), 4), dict(max_path=3)), (F((8, 5), 4), dict(max_path=6)), (F((40,), 4), {}),
                     (F((40,), 4), dict(max_path=6)), (P, {})):
        with pytest.raises(ValueError):
            commit(path, **kw)
    assert len(calls) == 8
