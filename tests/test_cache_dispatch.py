"""The kernels that the cache and the tree attention launch, as the library
itself decides them, recorded without a GPU (tests/hip_recorder.cpp)."""
from __future__ import annotations

import json
import os
import re
import subprocess
import sys

import pytest

import paper_2608_04991_amd as rac

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHILD = r"""
import ctypes, json, sys
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
rec.recorded.restype = rec.registered.restype = ctypes.c_char_p
import paper_2608_04991_amd as rac
from paper_2608_04991_amd import cache
P = 1 << 20  # a stand-in for every device pointer (aligned; nothing reads it)
out = []
for kind, cfg, tree in json.load(sys.stdin):
    rec.forget()
    if kind == "all":
        rac.library()
        out.append(rec.registered().decode())
        continue
    c = rac.CacheConfig(*cfg)
    if kind == "attention":
        t = rac.TreeConfig(*tree)
        x = cache._TreeTensors(P, P, P, P, P, None, P, P, t.q_heads * c.head_dim, c.kv_heads * c.head_dim,
                               t.q_heads * c.head_dim, 64, 0)
        n = rac.rac_tree_attention_workspace(c, t)
        assert rac.library().rac_tree_attention(c._ref, t._ref, 0, P, P, P, ctypes.byref(x), P, n, 0) == 0
    elif kind == "fork":
        rac.rac_cache_fork(c, P, P, P, P, stream=0)
    elif kind == "copy":
        rac.rac_cache_copy(c, P, P, P, P, tree, stream=0)
    elif kind == "commit":
        row = c.kv_heads * c.head_dim
        n = rac.rac_cache_commit_workspace(c)
        assert rac.library().rac_cache_commit(c._ref, P, P, P, P, P, P, row, row * tree, tree, P, P, tree, P, P, n, 0) == 0
    elif kind == "predictor":
        p, t = rac.PredictorConfig(64 * c.kv_heads * 4, 64 * c.kv_heads, c.kv_heads, 256, 8, 16), rac.TreeConfig(*tree)
        n = rac.rac_predictor_tree_workspace(p, c, t)
        assert rac.library().rac_predictor_tree_step(ctypes.byref(p._c()), c._ref, t._ref, P, P, P, P, P, P, P, P, None, 0, P,
                                                     P, P, 9, P, P, n, 0) == 0
    out.append(rec.recorded().decode())
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    if not os.path.exists(rac.library_path()):
        pytest.fail("librac.so is not built; run __graft_entry__.build()")
    so = str(tmp_path_factory.mktemp("recorder") / "hip_recorder.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", so, os.path.join(ROOT, "tests", "hip_recorder.cpp")], check=True)

    def launches(calls):
        """(kernel, grid, threads) of each call's launches."""
        r = subprocess.run([sys.executable, "-c", _CHILD, so], cwd=ROOT, input=json.dumps(calls), text=True,
                           stdout=subprocess.PIPE, check=True, timeout=300)
        logs = [[l.split("\t") for l in log.splitlines()] for log in json.loads(r.stdout)]
        mangled = sorted({l[0] for log in logs for l in log})
        plain = subprocess.run(["c++filt"], input="\n".join(mangled), text=True, capture_output=True, check=True).stdout
        name = {m: re.sub(r"\(anonymous namespace\)::|^void ", "", p).split("(")[0]
                for m, p in zip(mangled, plain.splitlines())}
        return [[(name[l[0]], int(l[1]), int(l[3])) for l in log] for log in logs]

    return launches


def test_every_kernel_is_run_by_a_gpu_test(record):
    pytest.importorskip("torch")
    from tests import test_gpu_tree_forms as F
    calls = [("all", None, None)]
    for shapes, q_heads, kv_heads, dim in F.FORMS.values():
        for kind in (0, 1, 2):
            for window in (0, 333):
                b = F.Batch(shapes, q_heads, kv_heads, dim, 16, kind, window=window, layers=1, layer=0)
                c, t = b.cfg, b.tree
                calls.append(("attention", [c.layers, c.kv_heads, c.head_dim, c.page_tokens, c.pages, c.seqs, c.max_pages,
                                            c.type], [t.q_heads, t.rows, t.max_rows, t.max_draft, t.window]))
    # (tests/test_gpu_cache.py has these)
    calls += [("fork", [1, 1, 16, 8, 100, s, 3], None) for s in (4, 4096)]
    calls += [("copy", [1, 1, 16, 8, 100, 1, 1], 5)] + [("commit", [1, 1, 16, 8, 100, 4, 3, k], 9) for k in (0, 2)]
    calls.append(("predictor", [1, 2, 64, 8, 36, 3, 12], [2, 5, 3, 3, 8]))  # (tests/test_gpu_predictor_tree.py)
    every, *got = record(calls)
    kernels = {k for k, _, _ in every if k.startswith(("tree_", "cache_"))}
    assert len(kernels) > 40
    assert kernels - {k for ls in got for k, _, _ in ls} == set()


def test_forms_by_rows_of_a_key_value_head(record):
    cases = [(64, 1, 16, "tree_few_kernel<0, 64, 1>"), (64, 2, 16, "tree_few_kernel<0, 64, 2>"),
             (64, 4, 16, "tree_many_kernel<0, 64, 1, 4>"), (64, 100, 16, "tree_many_kernel<0, 64, 2, 4>"),
             (80, 1, 7, "tree_few_kernel<0, 128, 1>"), (128, 3, 7, "tree_many_kernel<0, 128, 1, 4>"),
             (128, 63, 8, "tree_many_kernel<0, 128, 2, 4>"), (128, 64, 8, "tree_many_kernel<0, 128, 2, 8>"),
             (144, 1, 1, "tree_many_kernel<0, 256, 1, 4>")]
    got = record([("attention", [1, 2, dim, 16, 1000, 3, 100], [2 * group, 3 * rows, rows, rows, 0])
                  for dim, rows, group, _ in cases])
    assert [ls[0][0] for ls in got] == [c[3] for c in cases]


def test_launches_of_a_call(record):
    """One launch where no sequence can be long, two (with the join) where one
    can, three beyond 64 sequences."""
    cfg = lambda seqs, width: [1, 8, 64, 16, 1000, seqs, width]
    got = record([("attention", cfg(8, 5), [8, 96, 12, 12, 64]), ("attention", cfg(8, 500), [8, 96, 12, 12, 0]),
                  ("attention", cfg(65, 500), [8, 96, 12, 12, 0])])
    assert [len(ls) for ls in got] == [1, 2, 3]
    assert got[2][0][0] == "tree_plan_kernel" and got[1][1][0].startswith("tree_join_kernel<0, 64, ")
