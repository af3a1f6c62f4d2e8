"""Rotary positions, log probabilities and gradients between guards: whatever positions,
tokens and row numbers hold, nothing is written outside the outputs, at any alignment and
around the sizes at which rows are held, cut into parts or read as a stream."""
from __future__ import annotations

import random

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests.gpu_util import say
from tests.test_gpu_cache_guards import Guarded, nonsense
from tests.test_gpu_logprobs import TYPES, Call, check_gradients, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def columns(g, x, off, apart):
    """The rows of x, `apart` elements between them, from the off-th of these on, between guards."""
    rows, width = x.shape
    whole = torch.full((rows, width + apart), 3.0, dtype=x.dtype, device="cuda")
    whole[:, off:off + width] = x
    return g.read_only(whole)[:, off:off + width]


class Between(Call):
    """A call whose every buffer lies between guards."""

    def __init__(self, g, logits, tokens, scale, top, token_rows=None):
        kind = {v: k for k, v in TYPES.items()}[logits.dtype]
        rows, vocab = logits.shape
        self.cfg = rac.LogprobConfig(rows, vocab, tokens.numel(), top, kind, scale)
        self.logits, self.tokens = logits, g.read_only(tokens)
        self.token_rows = None if token_rows is None else g.read_only(token_rows)
        new = lambda *s, dtype=torch.float32: g(torch.full(s, 77, dtype=dtype))
        self.logprob, self.lse, self.entropy = new(tokens.numel()), new(rows), new(rows)
        self.ids, self.tops = (new(rows, top, dtype=torch.int32), new(rows, top)) if top else (None, None)
        self.ws = g(torch.full((rac.rac_logprobs_workspace(self.cfg),), 0xAB, dtype=torch.uint8))
        self.run()
        g.check()


# Blocks of 16 bytes of a row, around those that 256 threads hold (nine each), 512 threads, and
# two parts of these.
HELD = [9 * 256 + i for i in (-2, -1, 0, 1)] + [9 * 512 + i for i in (-2, -1, 0, 1)] + [2 * 9 * 512 + i for i in (-1, 0)]


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
def test_log_probabilities_where_rows_are_held_and_cut(dtype):
    n = 16 // torch.empty(0, dtype=dtype).element_size()
    for blocks in HELD:
        for more in (0, 1, n - 1):
            vocab = blocks * n + more
            say(f"[gpu] log probabilities between guards, {vocab} words of {dtype}")
            rng, g = random.Random(vocab), Guarded()
            off = rng.randrange(0, n)
            x = columns(g, normal(3, vocab, dtype, vocab), off, n + rng.randrange(0, n))
            tokens = torch.tensor([rng.randrange(vocab), vocab - 1, rng.choice([-1, vocab, (1 << 31) - 1, -(1 << 31)])],
                                  dtype=torch.int32)
            Between(g, x, tokens, 0.9, rng.choice([1, 5, 64])).check()


@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (2, 3, 64), (9, 1025, 0), (700, 517, 7), (5, 2400001, 3), (5, 2400001, 0),
                                            (1300, 9001, 0), (33, 50001, 64)])
def test_broken_tokens_and_rows(rows, vocab, top):
    for seed, dtype in enumerate(TYPES.values()):
        say(f"[gpu] broken tokens, {rows} x {vocab} {dtype}")
        rng, g = random.Random(seed), Guarded()
        x = columns(g, normal(rows, vocab, dtype, seed), seed, 5)
        tokens = nonsense(rng, torch.randint(0, vocab, (rows,), dtype=torch.int32), vocab)
        Between(g, x, tokens, 1.1, top).check()
        count = 2 * rows + 3
        tokens = nonsense(rng, torch.randint(0, vocab, (count,), dtype=torch.int32), vocab)
        of = nonsense(rng, torch.randint(0, rows, (count,), dtype=torch.int32), rows)
        Between(g, x, tokens, 0.0, top, of).check()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (600, 517), (5, 8191), (5, 8192), (5, 8193), (3, 50001)])
def test_gradients_between_guards(dtype, rows, vocab):
    say(f"[gpu] gradients between guards, {rows} x {vocab} {dtype}")
    for off, out_off, apart, out_apart in ((0, 0, 0, 0), (1, 1, 5, 5), (0, 3, 3, 8), (2, 1, 9, 1)):
        rng, g = random.Random(off + vocab), Guarded()
        x = columns(g, normal(rows, vocab, dtype, vocab), off, apart)
        tokens = nonsense(rng, torch.randint(0, vocab, (rows,), dtype=torch.int32), vocab)
        c = Between(g, x, tokens, 0.7, 0)
        gl, ge = g.read_only(torch.randn(rows)), g.read_only(torch.randn(rows))
        frame = g(torch.full((rows, vocab + out_apart), 7.0, dtype=dtype))
        out = frame[:, out_off:out_off + vocab]
        for a, b in ((gl, None), (None, ge), (gl, ge)):
            rac.rac_logprobs_backward(c.cfg, x, c.tokens, c.lse, out, grad_logprob=a, grad_entropy=b, entropy=c.entropy)
            g.check()
            check_gradients(c, x, out, a, b)
        rest = torch.ones(vocab + out_apart, dtype=torch.bool, device="cuda")
        rest[out_off:out_off + vocab] = False
        assert (frame[:, rest] == 7).all()


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,q_heads,k_heads,dim,turned", [(1, 1, 0, 16, 16), (70, 1, 1, 112, 16), (33, 7, 1, 80, 80),
                                                             (19, 3, 2, 64, 32), (5, 60, 4, 256, 128)])
def test_broken_positions(type, rows, q_heads, k_heads, dim, turned):
    say(f"[gpu] broken positions, {rows} rows, heads {q_heads}+{k_heads} x {dim}, {turned} turned, type {type}")
    freq = torch.tensor(rac.rac_rotary_frequencies(turned, 10000.0), dtype=torch.float64)
    for seed, layout in enumerate((rac.RAC_ROTARY_INTERLEAVED, rac.RAC_ROTARY_HALF)):
        rng, g = random.Random(seed), Guarded()
        cfg = rac.RotaryConfig(rows, q_heads, k_heads, dim, turned, type, layout)
        pos = g.read_only(nonsense(rng, torch.arange(rows, dtype=torch.int32), 1 << 20))
        f = g.read_only(freq)
        heads = lambda n, make: make(torch.randn(rows, n + seed, dim).to(TYPES[type]))  # (rows apart, or not)
        q, k = heads(q_heads, g.read_only), heads(k_heads, g.read_only) if k_heads else None
        frames = [heads(q_heads, g), heads(k_heads, g) if k_heads else None]
        was = [None if t is None else t.clone() for t in frames]
        part = lambda t, n: None if t is None else t[:, :n]
        rac.rac_rotary(cfg, pos, f, part(q, q_heads), part(k, k_heads), q_out=part(frames[0], q_heads),
                       k_out=part(frames[1], k_heads))
        g.check()
        for t, old, n in zip(frames, was, (q_heads, k_heads)):
            if t is not None:  # (rows of padding, and what lies between the rows)
                assert torch.equal(t[pos < 0], old[pos < 0]) and torch.equal(t[:, n:], old[:, n:])
                assert torch.isfinite(t).all()
