"""The kernels that rotary positions, log probabilities, weights and eviction launch, as
the library itself decides them, recorded without a GPU (tests/hip_recorder.cpp): the
tests on the GPU run every one, and calls launch no more than their contract says."""
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
from paper_2608_04991_amd import cache, tokens
P = 1 << 20  # a stand-in for every device pointer (aligned; nothing reads it)
L, out = rac.library(), []
for kind, cfg, more in json.load(sys.stdin):
    rec.forget()
    if kind == "all":
        out.append(rec.registered().decode())
        continue
    if kind == "rotary":
        c = rac.RotaryConfig(*cfg)
        t = tokens._RotaryTensors(P, P, P, P, c.q_heads * c.head_dim, c.k_heads * c.head_dim, c.q_heads * c.head_dim,
                                  c.k_heads * c.head_dim)
        st = L.rac_rotary(c._ref, P, P, ctypes.byref(t), None)
    elif kind == "logprobs":
        c = rac.LogprobConfig(*cfg)
        t = tokens._LogprobTensors(P, c.vocab, P, P if more[0] else None, P, P, P if more[1] else None, P, P)
        st = L.rac_logprobs(c._ref, ctypes.byref(t), P, 1 << 40, None)
    elif kind == "backward":
        c = rac.LogprobConfig(*cfg)
        g = tokens._LogprobGradients(P, c.vocab, P, P, P, P, P if more[0] else None, P + (0 if more[1] else 4), c.vocab)
        st = L.rac_logprobs_backward(c._ref, ctypes.byref(g), None)
    elif kind == "weights":
        c, t = rac.CacheConfig(*cfg), rac.TreeConfig(*more)
        x = cache._TreeTensors(P, P, None, P, P, None, None, P, t.q_heads * c.head_dim, c.kv_heads * c.head_dim, 0, 64, 0)
        st = L.rac_tree_weights(c._ref, t._ref, 0, 1, P, P, P, ctypes.byref(x), P, P, P, 1 << 40, None)
    elif kind == "append":
        c = rac.CacheConfig(*cfg)
        st = L.rac_cache_weights_commit(c._ref, 1, P, P, P, P, 5, P, 20, P, None)
    else:
        c, e = rac.CacheConfig(*cfg), rac.EvictConfig(*more)
        st = L.rac_cache_evict(c._ref, e._ref, P, P, P, P, P, P, P, P, P, 1 << 50, None)
    assert st == 0, (kind, cfg, more, st)
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
        """(kernel, workgroups, threads) of each call's launches."""
        r = subprocess.run([sys.executable, "-c", _CHILD, so], cwd=ROOT, input=json.dumps(calls), text=True,
                           stdout=subprocess.PIPE, check=True, timeout=300)
        logs = [[l.split("\t") for l in log.splitlines()] for log in json.loads(r.stdout)]
        mangled = sorted({l[0] for log in logs for l in log})
        plain = subprocess.run(["c++filt"], input="\n".join(mangled), text=True, capture_output=True, check=True).stdout
        name = {m: re.sub(r"\(anonymous namespace\)::|^void ", "", p).split("(")[0]
                for m, p in zip(mangled, plain.splitlines())}
        return [[(name[l[0]], int(l[1]) * int(l[2]), int(l[3])) for l in log] for log in logs]

    return launches


def calls_of_the_gpu_tests():
    calls = []
    for type in (0, 1, 2):
        for layout in (0, 1):
            calls.append(("rotary", [17, 8, 8, 64, 32, type, layout], None))
        for rows, vocab in ((5, 8), (64, 1025), (600, 517), (3, 131071), (513, 8191), (520, 33001), (2, 2400001)):
            for top in (0, 5):
                for entropy in (0, 1):
                    calls.append(("logprobs", [rows, vocab, rows, top, type], [0, entropy]))
        calls.append(("logprobs", [40, 70001, 100, 3, type], [1, 1]))
        for entropy in (0, 1):
            for alike in (0, 1):
                calls.append(("backward", [9, 3001, 9, 0, type], [entropy, alike]))
        for dim in (64, 128, 256):
            for shape in ((8, 20, 2), (8, 30, 6), (2, 300, 130)):
                calls.append(("weights", [2, 2, dim, 16, 100, 13, 20, type], [shape[0], shape[1], shape[2], shape[2]]))
    calls.append(("append", [2, 3, 16, 8, 200, 5, 20], None))
    for cfg in ([2, 3, 32, 16, 100, 14, 20], [1, 1, 16, 8, 900, 1100, 10], [1, 2, 16, 64, 2000, 3, 1200], [1, 2, 16, 16, 5000, 4, 4200]):
        for sets in (1, cfg[0] * cfg[1]):
            calls.append(("evict", cfg, [sets, 2, 9]))
    return calls


def test_every_kernel_is_run_by_a_gpu_test(record):
    every, *got = record([("all", None, None)] + calls_of_the_gpu_tests())
    kernels = {k for k, _, _ in every if k.startswith(("rotary_", "logprob_", "weights_", "evict_"))}
    assert len(kernels) > 30
    assert kernels - {k for ls in got for k, _, _ in ls} == set()


def test_launches_of_a_call(record):
    calls = calls_of_the_gpu_tests()
    most = {"rotary": 1, "logprobs": 3, "backward": 1, "weights": 2, "append": 1, "evict": 10}
    for (kind, _, more), ls in zip(calls, record(calls)):
        assert 1 <= len(ls) <= most[kind] - (kind == "logprobs" and not more[0])


def test_grids_stay_within_a_dispatch(record):
    """The largest calls: fewer than 2^32 threads."""
    big = [("rotary", [1 << 24, 64, 8, 256, 256, 2], None), ("rotary", [1 << 24, 1, 0, 16, 16, 0], None),
           ("logprobs", [1 << 24, 1 << 24, 1 << 24, 0, 2], [1, 1]), ("backward", [1 << 24, 1 << 24, 1 << 24, 0, 2], [1, 1]),
           ("evict", [1024, 1024, 16, 8, 1 << 24, 4096, 1], [1, 0, 0]), ("evict", [64, 64, 16, 8, 1 << 24, 1024, 1], [4096, 0, 0])]
    for (kind, cfg, _), ls in zip(big, record(big)):
        assert ls and all(0 < grid * threads < 1 << 32 for _, grid, threads in ls), (kind, cfg, ls)
