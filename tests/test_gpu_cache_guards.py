"""Device arrays that hold nonsense: whatever they say, nothing is written outside
the buffers.  Every buffer lies between two guards."""
from __future__ import annotations

import random

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say
from tests.test_gpu_tree_attention import Batch

pytestmark = pytest.mark.gpu

GUARD, SIGN = 1 << 20, 0x5A


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


class Guarded:
    """Copies of tensors between guards."""

    def __init__(self):
        self.held = []

    def __call__(self, t):
        t = t.cuda().contiguous()
        n = t.numel() * t.element_size()
        buffer = torch.full((GUARD + n + GUARD,), SIGN, dtype=torch.uint8, device="cuda")
        inner = buffer[GUARD:GUARD + n].view(t.dtype).view(t.shape) if n else t
        inner.copy_(t)
        self.held.append((buffer, n, inner, None))
        return inner

    def read_only(self, t):
        inner = self(t)
        self.held[-1] = (*self.held[-1][:3], inner.clone())
        return inner

    def check(self):
        torch.cuda.synchronize()
        for i, (buffer, n, inner, was) in enumerate(self.held):
            assert (buffer[:GUARD] == SIGN).all() and (buffer[GUARD + n:] == SIGN).all(), f"buffer {i}"
            if was is not None:
                same = (inner.contiguous().view(torch.uint8) == was.view(torch.uint8)).all() if n else True
                assert same, f"buffer {i} is read only"


def nonsense(rng, like, most):
    """A third of the entries of an int32 tensor replaced."""
    out = like.clone().ravel()
    for i in range(out.numel()):
        if rng.random() < 0.33:
            out[i] = rng.choice([-1, -2, -77, -(1 << 31), 0, most - 1, most, most + 1, 2 * most, 1 << 20, 1 << 28,
                                 (1 << 31) - 1, rng.randrange(0, most + 1)])
    return out.view(like.shape)


SHAPES = {
    "few rows": ([(0, 1, 1), (1, 1, 1), (65, 2, 2), (130, 3, 3), (257, 1, 1), (300, 0, 0)], 4, 2, 64),
    "many rows": ([(0, 33, 33), (700, 40, 40), (31, 9, 9)], 8, 2, 128),
    "wide heads": ([(100, 1, 1), (9, 30, 30), (64, 2, 2)], 4, 2, 192),
    "parts": ([(4001, 1, 1), (33, 1, 1), (2000, 2, 2)], 8, 8, 64),
    "70 sequences": ([(17 * i % 900, 2, 2) for i in range(70)], 4, 2, 80),
}


@pytest.mark.parametrize("kind", [R.BF16, R.FP8])
@pytest.mark.parametrize("name", SHAPES)
def test_attention_between_guards(name, kind):
    say(f"[gpu] attention with broken arrays, {name}, type {kind}")
    shapes, q_heads, kv_heads, dim = SHAPES[name]
    for seed in range(6):
        rng = random.Random(seed)
        b = Batch(shapes, q_heads, kv_heads, dim, 16, kind, mask="tree" if seed % 2 else "none", seed=seed,
                  window=(0, 0, 5, 100)[seed % 4])
        g = Guarded()
        rows, S = b.tree.rows, len(shapes)
        lengths, table = nonsense(rng, b.lengths, 16 * b.cfg.max_pages), nonsense(rng, b.table, b.cfg.pages)
        q_start, d_start = nonsense(rng, b.q_start, rows), nonsense(rng, b.d_start, b.k.shape[0])
        if seed == 5:  # everything overlaps
            q_start = torch.tensor([(s % 2) * rows for s in range(S + 1)], dtype=torch.int32)
            d_start, lengths = q_start.clone(), torch.full_like(lengths, 1 << 30)
        out = g(torch.full((rows, q_heads, dim), 7.0).to(R.ACT[kind]))
        lse = g(torch.zeros(rows, q_heads))
        ws = g(torch.zeros(rac.rac_tree_attention_workspace(b.cfg, b.tree), dtype=torch.uint8))
        rac.rac_tree_attention(
            b.cfg, b.tree, b.layer, g.read_only(b.pool.view(torch.uint8)), g.read_only(table), g.read_only(lengths),
            g.read_only(b.q), g.read_only(q_start), g.read_only(b.k), g.read_only(b.v), out, ws,
            draft_start=g.read_only(d_start), mask=None if b.words is None else g.read_only(b.words), lse=lse)
        g.check()


@pytest.mark.parametrize("kind", [R.BF16, R.FP8])
@pytest.mark.parametrize("seqs,pages,width,page", [(6, 60, 9, 8), (1100, 300, 5, 16), (3, 5000, 40, 64)])
def test_cache_calls_between_guards(kind, seqs, pages, width, page):
    say(f"[gpu] cache calls with broken arrays, {seqs} sequences, {pages} pages of {page}, type {kind}")
    cfg = rac.CacheConfig(2, 3, 32, page, pages, seqs, width, kind)
    for seed in range(6):
        rng = random.Random(seed)
        g = Guarded()
        ids = list(range(pages))
        rng.shuffle(ids)
        held = [[ids.pop() if ids and rng.random() < 0.4 else -1 for _ in range(width)] for _ in range(seqs)]
        counts = torch.zeros(pages, dtype=torch.int32)
        for row in held:
            for p in row:
                if p >= 0:
                    counts[p] += 1
        table = g(nonsense(rng, torch.tensor(held, dtype=torch.int32), pages))
        lengths = g(nonsense(rng, torch.tensor([rng.randrange(0, width * page + 1) for _ in range(seqs)], dtype=torch.int32),
                             width * page))
        refs = g(nonsense(rng, counts, 3) if seed % 2 else counts)
        pool = g(torch.zeros(rac.rac_cache_pool_bytes(cfg), dtype=torch.uint8))
        rows, most = 4 * seqs, 6
        k, v = (g.read_only(torch.randn(2, rows, 3, 32).bfloat16()) for _ in range(2))
        start = g.read_only(nonsense(rng, torch.arange(0, rows + 1, 4, dtype=torch.int32), rows))
        path = g.read_only(nonsense(rng, torch.tensor([[0, 1, 2, 3, -1, -1]] * seqs, dtype=torch.int32), 4))
        out = g(torch.zeros(seqs, dtype=torch.int32))
        ws = g(torch.zeros(rac.rac_cache_commit_workspace(cfg), dtype=torch.uint8))
        one = lambda n, top: g.read_only(nonsense(rng, torch.arange(n, dtype=torch.int32), top))
        rac.rac_cache_commit(cfg, pool, table, lengths, refs, k, v, start, out, ws, path=path, max_path=most)
        g.check()
        rac.rac_cache_fork(cfg, one(seqs, seqs), table, lengths, refs, one(seqs, width * page), one(seqs, width * page))
        g.check()
        rac.rac_cache_commit(cfg, pool, table, lengths, refs, k, v, start, out, ws, max_path=rng.choice([0, 3, 50]))
        g.check()
        n = min(pages, 40)
        rac.rac_cache_copy(cfg, pool, one(n, pages), pool, one(n, pages))
        g.check()
        assert (out >= 0).all() and (out <= rows).all()


def test_a_page_outside_the_pool_is_not_copied():
    cfg = rac.CacheConfig(2, 3, 32, 8, 60, 6, 9)
    g = Guarded()
    pool = g(torch.randint(0, 256, (rac.rac_cache_pool_bytes(cfg),), dtype=torch.uint8))
    want = pool.clone().view(60, -1)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    rac.rac_cache_copy(cfg, pool, i32(0, 1 << 20, -1, 7, 60), pool, i32(60, 3, 4, -1, 5))
    rac.rac_cache_copy(cfg, pool, i32(2, 60), pool, i32(59, 0))
    g.check()
    want[59] = want[2]
    assert torch.equal(pool.view(60, -1), want)
