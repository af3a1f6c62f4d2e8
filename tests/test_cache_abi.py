"""Checks of include/rac_cache.h that need no GPU: every declared function is
exported, sizes, and refusals, which come before any launch."""
from __future__ import annotations

import ctypes
import dataclasses
import os
import re

import pytest

import paper_2608_04991_amd as rac
from paper_2608_04991_amd import cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # a stand-in for device pointers that nothing reads
CFG = rac.CacheConfig(2, 4, 64, 16, 100, 8, 10)
TREE = rac.TreeConfig(8, 20, 5, 5)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rac.library_path()):
        pytest.fail("librac.so is not built; run __graft_entry__.build()")
    return rac.library()


def test_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rac_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(rac_[a-z_]+)\s*\(", text))
    assert {"rac_tree_attention", "rac_cache_fork", "rac_cache_commit", "rac_cache_copy"} <= names
    for n in names:
        assert hasattr(lib, n) and hasattr(rac, n), n


def test_pool_bytes():
    assert rac.rac_cache_pool_bytes(CFG) == 100 * 2 * 2 * 4 * 16 * 64 * 2
    assert rac.rac_cache_pool_bytes(dataclasses.replace(CFG, type=rac.RAC_CACHE_FP8)) == 100 * 2 * 2 * 4 * 16 * 64
    big = rac.CacheConfig(64, 8, 128, 64, 1 << 20, 8, 10)
    assert rac.rac_cache_pool_bytes(big) == (1 << 20) * 64 * 2 * 8 * 64 * 128 * 2


@pytest.mark.parametrize("bad", [
    dict(layers=0), dict(layers=1025), dict(kv_heads=0), dict(head_dim=8), dict(head_dim=72), dict(head_dim=272),
    dict(page_tokens=4), dict(page_tokens=24), dict(page_tokens=512), dict(pages=0), dict(pages=(1 << 24) + 1),
    dict(seqs=0), dict(seqs=4097), dict(max_pages=0), dict(max_pages=1 << 27), dict(type=3), dict(type=-1),
    dict(type=2, k_scale=0.0), dict(type=2, v_scale=-1.0), dict(type=2, k_scale=float("nan")),
    dict(type=2, v_scale=float("inf"))], ids=str)
def test_bad_configurations_are_refused(lib, bad):
    c = dataclasses.replace(CFG, **bad)
    assert rac.rac_cache_pool_bytes(c) == 0 and rac.rac_cache_commit_workspace(c) == 0
    assert rac.rac_tree_attention_workspace(c, TREE) == 0
    for call in (lambda: rac.rac_cache_fork(c, P, P, P, P, stream=0),
                 lambda: rac.rac_cache_copy(c, P, P, P, P, 1, stream=0)):
        with pytest.raises(rac.RacError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("bad", [
    dict(q_heads=0), dict(q_heads=6), dict(q_heads=4 * 65), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(max_rows=-1),
    dict(max_draft=-1), dict(window=-1), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan"))], ids=str)
def test_bad_trees_are_refused(lib, bad):
    assert rac.rac_tree_attention_workspace(CFG, TREE) > 0
    assert rac.rac_tree_attention_workspace(CFG, dataclasses.replace(TREE, **bad)) == 0


def test_attention_refusals(lib):
    need = rac.rac_tree_attention_workspace(CFG, TREE)
    ok = dict(q=P, k=P, v=P, q_start=P, draft_start=None, mask=P, out=P, lse=P, q_stride=512, kv_stride=256,
              out_stride=512, draft_rows=20, mask_words=1)

    def call(layer=0, pool=P, table=P, lengths=P, ws=P, cap=need, tree=TREE, **change):
        t = cache._TreeTensors(**{**ok, **change})
        return lib.rac_tree_attention(ctypes.byref(CFG._c()), ctypes.byref(tree._c()), layer, pool, table, lengths,
                                      ctypes.byref(t), ws, cap, 0)

    for bad in (dict(layer=-1), dict(layer=2), dict(pool=None), dict(table=None), dict(lengths=None), dict(ws=None),
                dict(q=None), dict(q_start=None), dict(out=None), dict(k=None), dict(v=None), dict(q_stride=504),
                dict(q_stride=516), dict(out_stride=511), dict(kv_stride=248), dict(kv_stride=260), dict(draft_rows=-1),
                dict(mask_words=0), dict(mask=None), dict(mask_words=-1)):
        assert call(**bad) == 1, bad
    for bad in (dict(pool=P + 8), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8), dict(table=P + 2),
                dict(lengths=P + 1), dict(q_start=P + 2), dict(draft_start=P + 2), dict(lse=P + 2), dict(mask=P + 4),
                dict(ws=P + 128)):
        assert call(**bad) == 2, bad
    assert call(cap=need - 1) == 3
    # no rows: nothing to do
    assert call(tree=dataclasses.replace(TREE, rows=0), q=None, out=None) == 0


def test_fork_and_copy_refusals(lib):
    c = ctypes.byref(CFG._c())
    fork = lambda *a: lib.rac_cache_fork(c, *a, 0)
    assert fork(None, None, None, P, P, P) == 1 and fork(P, None, None, None, P, P) == 1
    assert fork(P, None, None, P, None, P) == 1 and fork(P, None, None, P, P, None) == 1
    for i in range(6):
        a = [P] * 6
        a[i] += 2
        assert fork(*a) == 2
    copy = lambda a, s, b, d, n: lib.rac_cache_copy(c, a, s, b, d, n, 0)
    assert copy(P, P, P, P, -1) == 1 and copy(P, P, P, P, 101) == 1 and copy(None, P, P, P, 1) == 1
    assert copy(P, None, P, P, 1) == 1 and copy(P, P, None, P, 1) == 1 and copy(P, P, P, None, 1) == 1
    assert copy(P + 8, P, P, P, 1) == 2 and copy(P, P + 2, P, P, 1) == 2 and copy(P, P, P + 4, P, 1) == 2
    assert copy(P, P, P, P + 1, 1) == 2 and copy(None, None, None, None, 0) == 0


def test_commit_refusals(lib):
    need = rac.rac_cache_commit_workspace(CFG)
    names = ("pool", "table", "lengths", "refs", "k", "v", "kv_stride", "layer_stride", "draft_rows", "draft_start",
             "path", "max_path", "committed", "workspace", "workspace_bytes")
    ok = dict(zip(names, (P, P, P, P, P, P, 256, 256 * 20, 20, P, P, 5, P, P, need)))
    call = lambda **bad: lib.rac_cache_commit(ctypes.byref(CFG._c()), *{**ok, **bad}.values(), 0)
    for bad in (dict(pool=None), dict(table=None), dict(lengths=None), dict(refs=None), dict(k=None), dict(v=None),
                dict(kv_stride=248), dict(kv_stride=257), dict(layer_stride=-8), dict(layer_stride=4), dict(draft_rows=-1),
                dict(draft_start=None), dict(max_path=-1), dict(committed=None), dict(workspace=None)):
        assert call(**bad) == 1, bad
    for name, off in (("pool", 8), ("k", 8), ("v", 4), ("workspace", 64), ("table", 2), ("lengths", 2), ("refs", 1),
                      ("draft_start", 2), ("path", 2), ("committed", 2)):
        assert call(**{name: P + off}) == 2, name
    assert call(workspace_bytes=need - 1) == 3


def test_predictor_tree_refusals(lib):
    pred = rac.PredictorConfig(512, 128, 2, 256, 16, 8)
    cfg, tree = rac.CacheConfig(1, 2, 64, 16, 20, 4, 5), rac.TreeConfig(2, 6, 3, 3, 16)
    need = rac.rac_predictor_tree_workspace(pred, cfg, tree)
    assert need > rac.rac_predictor_workspace_bytes(pred)
    for c, t in ((dataclasses.replace(cfg, layers=2), tree), (dataclasses.replace(cfg, kv_heads=1), tree),
                 (dataclasses.replace(cfg, head_dim=128), tree), (dataclasses.replace(cfg, type=rac.RAC_CACHE_FP16), tree),
                 (cfg, dataclasses.replace(tree, q_heads=4)), (cfg, dataclasses.replace(tree, window=0)),
                 (cfg, dataclasses.replace(tree, rows=9)), (cfg, dataclasses.replace(tree, scale=0.5))):
        assert rac.rac_predictor_tree_workspace(pred, c, t) == 0
    names = ("weights", "pool", "table", "lengths", "q_start", "draft_start", "slot", "pos", "mask", "mask_words", "h_prev",
             "draft_k", "draft_v", "draft_rows", "ref_out", "workspace", "workspace_bytes")
    ok = dict(zip(names, (P, P, P, P, P, P, P, P, P, 1, P, P, P, 9, P, P, need)))

    def call(tree=tree, **bad):
        return lib.rac_predictor_tree_step(ctypes.byref(pred._c()), cfg._ref, tree._ref, *{**ok, **bad}.values(), 0)

    for name in names:
        if name not in ("mask_words", "draft_rows", "workspace_bytes"):
            assert call(**{name: None}) == 1, name
            assert call(**{name: P + 2 if name in ("table", "lengths", "q_start", "draft_start", "slot", "pos", "mask")
                           else P + 8}) == 2, name
    assert call(draft_rows=-1) == 1 and call(mask_words=0) == 1 and call(workspace_bytes=need - 1) == 3
    assert call(tree=dataclasses.replace(tree, rows=0), weights=None) == 0


class _Fake:
    """A tensor's shape without memory."""

    def __init__(self, shape, elem=2, stride=None, cuda=True):
        self.shape, self._elem, self.is_cuda = tuple(shape), elem, cuda
        st, n = [], 1
        for d in reversed(shape):
            st.insert(0, n)
            n *= d
        self._stride, self._n = tuple(stride or st), n

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._stride

    def numel(self):
        return self._n

    def element_size(self):
        return self._elem

    def data_ptr(self):
        return P


def test_binding_checks_tensors_before_the_call(lib, monkeypatch):
    called = []
    fake = type("L", (), {n: (lambda *a: called.append(a) or 0) for n in ("rac_tree_attention", "rac_cache_commit")})()
    fake.rac_cache_pool_bytes = lib.rac_cache_pool_bytes
    fake.rac_tree_attention_workspace = lib.rac_tree_attention_workspace
    fake.rac_cache_commit_workspace = lib.rac_cache_commit_workspace
    monkeypatch.setattr(rac, "library", lambda: fake)
    F = _Fake
    pool = F((rac.rac_cache_pool_bytes(CFG) // 2,))
    ok = dict(pool=pool, table=F((8, 10), 4), lengths=F((8,), 4), q=F((20, 8, 64)), q_start=F((9,), 4), k=F((20, 4, 64)),
              v=F((20, 4, 64)), out=F((20, 8, 64)), workspace=F((1 << 28,), 1), mask=F((20, 1), 8), lse=F((20, 8), 4))

    def attend(**bad):
        a = {**ok, **bad}
        m, l = a.pop("mask"), a.pop("lse")
        rac.rac_tree_attention(CFG, TREE, 0, *a.values(), mask=m, lse=l, stream=0)

    attend()
    assert len(called) == 1
    for bad in (dict(pool=F((100,))), dict(table=F((8, 9), 4)), dict(table=F((8, 10), 8)), dict(lengths=F((7,), 4)),
                dict(q=F((19, 8, 64))), dict(q=F((20, 8, 64), 4)), dict(q=F((20, 7, 64))), dict(q=F((20, 8, 64), cuda=False)),
                dict(q=F((20, 8, 64), stride=(512, 128, 1))), dict(out=F((20, 512))), dict(q_start=F((8,), 4)),
                dict(v=F((19, 4, 64))), dict(v=F((20, 4, 64), stride=(512, 64, 1))), dict(mask=F((19, 1), 8)),
                dict(mask=F((20, 1), 4)), dict(lse=F((20, 7), 4)), dict(workspace=F((8,), 1))):
        with pytest.raises(ValueError):
            attend(**bad)
    assert len(called) == 1
    commit = dict(pool=pool, table=F((8, 10), 4), lengths=F((8,), 4), refs=F((100,), 4), k=F((2, 20, 4, 64)),
                  v=F((2, 20, 4, 64)), draft_start=F((9,), 4), committed=F((8,), 4), workspace=F((1 << 20,), 1))
    run = lambda **bad: rac.rac_cache_commit(CFG, *{**commit, **bad}.values(), path=F((8, 5), 4), stream=0)
    run()
    assert len(called) == 2
    for bad in (dict(k=F((1, 20, 4, 64))), dict(v=F((2, 19, 4, 64))), dict(k=F((2, 20, 4, 64), 4)), dict(refs=F((99,), 4)),
                dict(v=F((2, 20, 4, 64), stride=(20 * 512, 512, 64, 1))), dict(committed=F((7,), 4))):
        with pytest.raises(ValueError):
            run(**bad)
    assert len(called) == 2
