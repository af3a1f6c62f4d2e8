"""Checks of include/rac_tokens.h that need no GPU: every declared function is
exported, the frequencies, sizes, and refusals, which come before any launch."""
from __future__ import annotations

import copy
import ctypes
import dataclasses
import math
import os
import pickle
import re

import pytest

import paper_2608_04991_amd as rac
from paper_2608_04991_amd import tokens
from tests.test_cache_abi import P, ROOT, _Fake as F, lib  # noqa: F401

ROTARY = rac.RotaryConfig(20, 8, 2, 64, 48)
LOGPROB = rac.LogprobConfig(20, 1000, 20, 5)


def test_exports_every_declared_symbol(lib):  # noqa: F811
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rac_tokens.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(rac_[a-z_]+)\s*\(", text))
    assert names == {"rac_rotary_frequencies", "rac_rotary", "rac_logprobs_workspace", "rac_logprobs", "rac_logprobs_backward"}
    for n in names:
        assert hasattr(lib, n) and hasattr(rac, n), n


def test_frequencies(lib):  # noqa: F811
    plain = rac.rac_rotary_frequencies(64, 10000.0)
    assert len(plain) == 32
    for i, f in enumerate(plain):
        assert f == pytest.approx(10000.0 ** (-2 * i / 64) / (2 * math.pi), rel=1e-14)
    # (8192 positions: pair 0 turns 1304 times, the last 0.13 times)
    scaled = rac.rac_rotary_frequencies(64, 10000.0, 4.0, 8192, 1.0, 32.0)
    for f, g in zip(plain, scaled):
        keep = min(1.0, max(0.0, (8192 * f - 1.0) / 31.0))
        assert g == pytest.approx(f * (keep + (1 - keep) / 4.0), rel=1e-14)
    assert scaled[0] == plain[0] and scaled[-1] == plain[-1] / 4.0
    assert rac.rac_rotary_frequencies(64, 10000.0, 4.0) == pytest.approx([f / 4.0 for f in plain], rel=1e-15)
    for bad in (dict(rotary_dim=8), dict(rotary_dim=40), dict(rotary_dim=272), dict(base=1.0), dict(base=math.inf),
                dict(base=math.nan), dict(factor=0.0), dict(factor=-1.0), dict(factor=math.nan), dict(trained=-1),
                dict(slow=-1.0), dict(slow=32.0), dict(fast=math.inf)):
        with pytest.raises(rac.RacError) as e:
            rac.rac_rotary_frequencies(**{**dict(rotary_dim=64, base=10000.0), **bad})
        assert e.value.status == 1


def rotary(lib, cfg=ROTARY, pos=P, freq=P, **change):  # noqa: F811
    t = dict(q=P, k=P, q_out=P, k_out=P, q_stride=512, k_stride=128, q_out_stride=512, k_out_stride=128)
    t.update(change)
    return lib.rac_rotary(cfg._ref, pos, freq, ctypes.byref(tokens._RotaryTensors(**t)), None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=(1 << 24) + 1), dict(q_heads=0), dict(q_heads=4097), dict(k_heads=-1), dict(k_heads=4097),
    dict(head_dim=8), dict(head_dim=40), dict(head_dim=272), dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=80),
    dict(type=3), dict(type=-1), dict(layout=2), dict(transpose=2), dict(amplitude=math.nan), dict(amplitude=math.inf)], ids=str)
def test_bad_rotary_configurations_are_refused(lib, bad):  # noqa: F811
    assert rotary(lib, dataclasses.replace(ROTARY, **bad)) == 1


def test_rotary_refusals(lib):  # noqa: F811
    for bad in (dict(pos=None), dict(freq=None), dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None),
                dict(q_stride=504), dict(q_stride=516), dict(k_stride=120), dict(q_out_stride=511), dict(k_out_stride=132),
                dict(q_stride=1 << 37), dict(q_out_stride=1024), dict(k_stride=256)):
        assert rotary(lib, **bad) == 1, bad
    for bad in (dict(pos=P + 2), dict(freq=P + 4), dict(q=P + 8), dict(k=P + 2), dict(q_out=P + 8), dict(k_out=P + 4)):
        assert rotary(lib, **bad) == 2, bad
    assert rotary(lib, dataclasses.replace(ROTARY, rows=0), pos=None, q=None) == 0
    assert lib.rac_rotary(None, P, P, None, None) == 1 and lib.rac_rotary(ROTARY._ref, P, P, None, None) == 1


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(tokens=-1), dict(tokens=(1 << 24) + 1),
    dict(top=-1), dict(top=65), dict(type=3), dict(type=-1), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
    dict(scale=1e-13), dict(scale=1e13)], ids=str)
def test_bad_logprob_configurations_are_refused(lib, bad):  # noqa: F811
    cfg = dataclasses.replace(LOGPROB, **bad)
    assert rac.rac_logprobs_workspace(cfg) == 0
    assert logprobs(lib, cfg, token_rows=P) == 1
    assert backward(lib, dataclasses.replace(cfg, tokens=cfg.rows)) == 1 or "tokens" in bad or "top" in bad


def logprobs(lib, cfg=LOGPROB, ws=P, cap=1 << 30, **change):  # noqa: F811
    t = dict(logits=P, stride=1000, tokens=P, token_rows=None, logprob=P, lse=P, entropy=P, top_ids=P, top_logprobs=P)
    t.update(change)
    return lib.rac_logprobs(cfg._ref, ctypes.byref(tokens._LogprobTensors(**t)), ws, cap, None)


def backward(lib, cfg=LOGPROB, **change):  # noqa: F811
    g = dict(logits=P, stride=1000, tokens=P, lse=P, entropy=P, grad_logprob=P, grad_entropy=P, grad_logits=P, grad_stride=1000)
    g.update(change)
    return lib.rac_logprobs_backward(cfg._ref, ctypes.byref(tokens._LogprobGradients(**g)), None)


def test_logprob_refusals(lib):  # noqa: F811
    for bad in (dict(logits=None), dict(stride=999), dict(stride=1 << 41), dict(tokens=None), dict(logprob=None), dict(lse=None),
                dict(top_ids=None), dict(top_logprobs=None), dict(ws=None), dict(cfg=dataclasses.replace(LOGPROB, tokens=19))):
        assert logprobs(lib, **bad) == 1, bad
    for bad in (dict(logits=P + 1), dict(tokens=P + 2), dict(token_rows=P + 2), dict(logprob=P + 2), dict(lse=P + 1),
                dict(entropy=P + 2), dict(top_ids=P + 2), dict(top_logprobs=P + 2), dict(ws=P + 128)):
        assert logprobs(lib, **bad) == 2, bad
    assert logprobs(lib, cfg=dataclasses.replace(LOGPROB, type=rac.RAC_TYPE_FP32), logits=P + 2) == 2
    assert logprobs(lib, cap=rac.rac_logprobs_workspace(LOGPROB) - 1) == 3
    none = dataclasses.replace(LOGPROB, rows=0, tokens=0)
    assert logprobs(lib, none, ws=None, logits=None, lse=None, tokens=None) == 0
    for bad in (dict(logits=None), dict(stride=999), dict(tokens=None), dict(lse=None), dict(entropy=None), dict(grad_logits=None),
                dict(grad_stride=999), dict(grad_logprob=None, grad_entropy=None), dict(grad_stride=1008),
                dict(cfg=dataclasses.replace(LOGPROB, tokens=19)), dict(cfg=dataclasses.replace(LOGPROB, tokens=0))):
        assert backward(lib, **bad) == 1, bad
    for bad in (dict(logits=P + 1), dict(grad_logits=P + 1), dict(tokens=P + 2), dict(lse=P + 2), dict(entropy=P + 1),
                dict(grad_logprob=P + 2), dict(grad_entropy=P + 2)):
        assert backward(lib, **bad) == 2, bad
    assert backward(lib, none, logits=None) == 0


def test_binding_checks_tensors_before_the_call(lib, monkeypatch):  # noqa: F811
    called = []
    fake = type("L", (), {n: (lambda *a: called.append(a) or 0) for n in ("rac_rotary", "rac_logprobs", "rac_logprobs_backward")})()
    fake.rac_logprobs_workspace = lib.rac_logprobs_workspace
    monkeypatch.setattr(rac, "library", lambda: fake)
    turn = lambda **bad: rac.rac_rotary(ROTARY, **{**dict(pos=F((20,), 4), freq=F((24,), 8), q=F((20, 8, 64)), k=F((20, 2, 64)),
                                                          stream=0), **bad})
    turn()
    turn(q=F((30, 8, 64), stride=(700, 64, 1)), q_out=F((20, 8, 64)))
    assert len(called) == 2 and called[1][4]._obj.q_stride == 700 and called[1][4]._obj.q_out_stride == 512
    for bad in (dict(pos=F((19,), 4)), dict(pos=F((20,), 8)), dict(freq=F((24,), 4)), dict(freq=F((23,), 8)),
                dict(q=F((19, 8, 64))), dict(q=F((20, 8, 64), 4)), dict(q=F((20, 7, 64))), dict(q=F((20, 512))),
                dict(k=F((20, 2, 64), cuda=False)), dict(k_out=F((20, 2, 64), stride=(128, 1, 2))), dict(q_out=F((20, 8, 32)))):
        with pytest.raises(ValueError):
            turn(**bad)
    score = lambda **bad: rac.rac_logprobs(LOGPROB, **{**dict(
        logits=F((20, 1000)), tokens=F((20,), 4), logprob=F((20,), 4), lse=F((20,), 4), workspace=F((1 << 20,), 1),
        top_ids=F((20, 5), 4), top_logprobs=F((20, 5), 4), stream=0), **bad})
    score()
    for bad in (dict(logits=F((20, 999))), dict(logits=F((19, 1000))), dict(logits=F((20, 1000), 4)), dict(tokens=F((19,), 4)),
                dict(tokens=F((20,), 8)), dict(token_rows=F((19,), 4)), dict(lse=F((19,), 4)), dict(entropy=F((19,), 4)),
                dict(top_ids=F((20, 4), 4)), dict(top_logprobs=F((20, 4), 4)), dict(workspace=F((1,), 1)),
                dict(logits=F((20, 1000), stride=(1000, 2)))):
        with pytest.raises(ValueError):
            score(**bad)
    grad = lambda **bad: rac.rac_logprobs_backward(LOGPROB, **{**dict(
        logits=F((20, 1000)), tokens=F((20,), 4), lse=F((20,), 4), grad_logits=F((20, 1000), stride=(1008, 1)),
        grad_logprob=F((20,), 4), stream=0), **bad})
    grad()
    assert called[-1][2]._obj.grad_stride == 1008
    for bad in (dict(grad_logits=F((20, 1000), 4)), dict(grad_logprob=F((19,), 4)), dict(entropy=F((3,), 4)), dict(lse=F((20,), 2))):
        with pytest.raises(ValueError):
            grad(**bad)
    assert len(called) == 4


def test_configurations_can_be_copied_and_pickled_after_use(lib):  # noqa: F811
    for c in (ROTARY, LOGPROB):
        c._ref
        assert copy.deepcopy(c) == c and pickle.loads(pickle.dumps(c)) == c and hash(c) == hash(copy.copy(c))
