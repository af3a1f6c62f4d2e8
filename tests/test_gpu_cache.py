"""Forking, committing and copying pages against the contract's words
(tests/cache_reference.py): every table entry, count and stored bit is equal."""
from __future__ import annotations

import random

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Pair:
    """A cache on the GPU and its model."""

    def __init__(self, cfg, seed=0):
        self.cfg, self.rng = cfg, random.Random(seed)
        self.gen = torch.Generator().manual_seed(seed)
        self.model = R.Model(cfg.pages, cfg.page_tokens, cfg.seqs, cfg.max_pages)
        self.table, self.lengths, self.refs = rac.rac_cache_new(cfg)
        shape = (cfg.pages, cfg.layers, 2, cfg.kv_heads, cfg.page_tokens, cfg.head_dim)
        self.want = R.bits(torch.randn(*shape, generator=self.gen).to(R.STORED[cfg.type]))
        self.pool = self.want.cuda()
        self.ws = torch.empty(rac.rac_cache_commit_workspace(cfg), dtype=torch.uint8, device="cuda")

    def fork(self, parents, keep_from=None, keep_to=None):
        self.model.fork(parents, keep_from, keep_to)
        rac.rac_cache_fork(self.cfg, i32(parents), self.table, self.lengths, self.refs,
                           None if keep_from is None else i32(keep_from), None if keep_to is None else i32(keep_to))
        self.check()

    def commit(self, drafted, path=None, max_path=None, size=1.0, special=None):
        """drafted: rows of each sequence; path: lists, or None for all rows."""
        c = self.cfg
        rows = sum(drafted)
        start = [sum(drafted[:s]) for s in range(c.seqs + 1)]
        k, v = ((size * torch.randn(c.layers, rows, c.kv_heads, c.head_dim, generator=self.gen)).to(R.ACT[c.type])
                for _ in range(2))
        if special is not None:
            k[..., ::2] = special
        most = max_path if max_path is not None else (max(map(len, path), default=0) if path is not None else rows)
        if path is None:
            steps = [list(range(min(n, most))) for n in drafted]
        else:
            steps = [p[:R.accepted_tokens(p[:most], n)] for p, n in zip(path, drafted)]
        committed, copies, writes = self.model.commit([len(p) for p in steps])
        for a, b, n in copies:
            self.want[b, :, :, :, :n] = self.want[a, :, :, :, :n]
        held = [R.bits(R.stored(x, c.type, sc)) for x, sc in ((k, c.k_scale), (v, c.v_scale))]
        for s, i, page, place in writes:
            for side in (0, 1):
                self.want[page, :, side, :, place] = held[side][:, start[s] + steps[s][i]]
        out = torch.full((c.seqs,), -3, dtype=torch.int32, device="cuda")
        device_path = None
        if path is not None:
            device_path = i32([(p + [-1] * most)[:most] for p in path]).reshape(c.seqs, most)
        rac.rac_cache_commit(c, self.pool, self.table, self.lengths, self.refs, k.cuda(), v.cuda(), i32(start), out,
                             self.ws, path=device_path, max_path=most)
        torch.cuda.synchronize()
        assert out.tolist() == committed
        self.check()
        return committed

    def check(self):
        torch.cuda.synchronize()
        assert self.table.tolist() == self.model.table
        assert self.lengths.tolist() == self.model.lengths
        assert self.refs.tolist() == self.model.refs()
        got = self.pool.cpu()
        if self.cfg.type == R.FP8:  # a NaN's sign means nothing
            got[got == 255] = 127
            self.want[self.want == 255] = 127
        assert torch.equal(got, self.want), (got != self.want).nonzero()[:5].tolist()


def config(seqs=6, pages=60, width=9, layers=2, heads=3, dim=32, page=8, kind=R.BF16):
    return rac.CacheConfig(layers, heads, dim, page, pages, seqs, width, kind, 0.5 if kind == R.FP8 else 1.0,
                           0.125 if kind == R.FP8 else 1.0)


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("page,dim,heads,layers", [(8, 32, 3, 2), (16, 64, 8, 1), (64, 80, 1, 3), (256, 16, 2, 1)])
def test_drafting_rounds(kind, page, dim, heads, layers):
    say(f"[gpu] cache rounds type {kind} page {page} heads {heads} x {dim} layers {layers}")
    p = Pair(config(page=page, dim=dim, heads=heads, layers=layers, kind=kind), seed=page)
    p.commit([page + 3, 2 * page, 1, 0, page - 1, page + 1])
    p.fork([0, 0, 0, 1, 4, 4])                     # shared last pages, whole ones, and slots replaced
    p.commit([2, 3, 1, 5, 0, 4], path=[[1], [0, 2], [0], [1, 3, 4], [], [0, 1, 2, 3]])
    p.commit([3] * 6, path=[[0, 2], [0], [-1, 0], [5], [2, 1, 0], [0, 1, 9]])
    p.fork([3, 2, 1, 0, 5, 4])                     # a reordering
    p.commit([1] * 6)
    p.fork([0, -1, 2, 2, 99, 5], keep_to=[page, 5, 3, 1 << 30, 7, 0])
    p.commit([2, page + 2, 1, 1, 3, 1])
    p.fork(list(range(6)), keep_from=[1, page, 2, 0, 1 << 30, -4])
    p.commit([1] * 6)
    p.fork([-1] * 6)
    assert not p.refs.any()


def test_random_lives():
    say("[gpu] random lives of a cache")
    for seed in range(6):
        p = Pair(config(seqs=9, pages=40, width=6, layers=1, heads=1, dim=16), seed=seed)
        rng = p.rng
        for _ in range(12):
            if rng.random() < 0.5:
                parents = [rng.randrange(-2, 10) if rng.random() < 0.5 else d for d in range(9)]
                to = [rng.randrange(0, 48) for _ in range(9)] if rng.random() < 0.5 else None
                frm = [rng.choice([0, 0, rng.randrange(0, 20)]) for _ in range(9)] if rng.random() < 0.3 else None
                p.fork(parents, frm, to)
            else:
                drafted = [rng.choice([0, 1, 2, 7, 8, 9, 20]) for _ in range(9)]
                path = [sorted(rng.sample(range(n), rng.randrange(0, n + 1))) for n in drafted] if rng.random() < 0.6 else None
                p.commit(drafted, path)


def test_a_full_pool_and_a_full_table_leave_sequences_alone():
    p = Pair(config(seqs=4, pages=5, width=3, layers=1, heads=1, dim=16))
    assert p.commit([8, 17, 1, 9]) == [8, 17, 1, 0]      # the fourth finds no second page
    assert p.commit([17, 8, 8, 0]) == [0, 0, 0, 0]       # beyond the pool; beyond the table; beyond the pool
    assert p.commit([0, 7, 7, 0]) == [0, 7, 7, 0]        # places in pages that are there
    p.fork([0, -1, 0, 3])
    assert p.commit([1, 1, 1, 0]) == [1, 1, 1, 0]


def test_the_last_page_is_copied_only_while_it_is_shared():
    p = Pair(config(seqs=3, pages=8, width=3))
    p.commit([5, 0, 0])
    p.fork([0, 0, -1])
    p.commit([1, 0, 0])   # copies
    p.commit([0, 1, 0])   # alone by now
    assert p.model.refs().count(1) == 2


def test_many_sequences_and_pages():
    say("[gpu] cache of 1500 sequences")
    cfg = rac.CacheConfig(1, 1, 16, 8, 9000, 1500, 4, R.BF16)
    p = Pair(cfg, seed=2)
    p.commit([s % 19 for s in range(1500)])
    p.fork([(s * 7) % 1500 for s in range(1500)], keep_to=[(s * 5) % 30 for s in range(1500)])
    p.commit([(s * 3) % 5 for s in range(1500)])
    p.fork([s // 2 for s in range(1500)])
    p.commit([1 if s % 2 else 0 for s in range(1500)])


def test_wide_tables_and_4096_sequences():
    cfg = rac.CacheConfig(1, 1, 16, 8, 5000, 4096, 3, R.BF16)
    p = Pair(cfg)
    p.commit([1 if s < 2500 else 0 for s in range(4096)])
    p.fork([(s + 1000) % 4096 for s in range(4096)])
    p.commit([1 if s % 3 == 0 else 0 for s in range(4096)])
    cfg = rac.CacheConfig(1, 1, 16, 8, 3000, 3, 1200, R.BF16)
    p = Pair(cfg)
    p.commit([9000, 0, 4001], max_path=9000)
    p.fork([2, 0, 0], keep_from=[100, 5000, 0], keep_to=[4000, 9000, 8888])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -1e30, 5e3, 1e-30, -0.0])
def test_special_values_are_kept_or_clamped(value):
    for kind in (R.BF16, R.FP8):
        p = Pair(config(kind=kind))
        p.commit([9, 1, 0, 0, 3, 8], special=value)


@pytest.mark.parametrize("size", [0.01, 1.0, 300.0])
def test_fp8_rounding(size):
    p = Pair(config(kind=R.FP8, pages=200, width=20), seed=4)
    p.commit([60, 1, 33, 0, 3, 100], size=size)


def test_strided_drafts():
    cfg = config(layers=3)
    outs = []
    for strided in (False, True):
        table, lengths, refs = rac.rac_cache_new(cfg)
        gen = torch.Generator().manual_seed(1)
        pool = torch.zeros(rac.rac_cache_pool_bytes(cfg) // 2, dtype=torch.int16, device="cuda")
        kv = torch.randn(3, 20, 2, 3, 32, generator=gen).bfloat16().cuda()
        k, v = kv[:, :, 0], kv[:, :, 1]
        if not strided:
            k, v = k.contiguous(), v.contiguous()
        ws = torch.empty(rac.rac_cache_commit_workspace(cfg), dtype=torch.uint8, device="cuda")
        out = i32([0] * 6)
        rac.rac_cache_commit(cfg, pool, table, lengths, refs, k, v, i32([0, 3, 3, 9, 20, 20, 20]), out, ws)
        torch.cuda.synchronize()
        assert out.tolist() == [3, 0, 6, 11, 0, 0]
        outs.append(pool.cpu())
    assert torch.equal(*outs)


def test_broken_device_arrays_stay_inside_the_buffers():
    p = Pair(config())
    p.commit([9, 8, 1, 0, 3, 4])
    p.table[0, 0], p.table[1, 0] = 1 << 28, -77
    p.lengths[2], p.lengths[3] = 1 << 30, -5
    k = torch.zeros(2, 12, 3, 32, dtype=torch.bfloat16, device="cuda")
    out = i32([0] * 6)
    rac.rac_cache_commit(p.cfg, p.pool, p.table, p.lengths, p.refs, k, k, i32([0, 2, -5, 1 << 30, 3, 12, 4]), out, p.ws)
    rac.rac_cache_fork(p.cfg, i32([5, 0, 1 << 30, -9, 2, 2]), p.table, p.lengths, p.refs, i32([-5] * 6), i32([1 << 30] * 6))
    rac.rac_cache_copy(p.cfg, p.pool, i32([0, 1 << 20, -1]), p.pool, i32([60, 3, 4]))
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", [R.BF16, R.FP8])
@pytest.mark.parametrize("n,page,dim,layers", [(1, 8, 16, 1), (5, 16, 64, 1), (17, 32, 80, 3), (40, 256, 128, 2), (0, 8, 16, 1)])
def test_copies_of_pages(kind, n, page, dim, layers):
    say(f"[gpu] copy of {n} pages of {page} x {dim} x {layers}")
    cfg = rac.CacheConfig(layers, 2, dim, page, n + 3, 1, 1, kind)
    rng = random.Random(n)
    src, dst = rng.sample(range(n + 3), n), rng.sample(range(n + 3), n)
    gen = torch.Generator(device="cuda").manual_seed(n)
    shape = (n + 3, layers, 2, 2, page, dim)
    a, b = (torch.randint(0, 256, (*shape, 1 if kind == R.FP8 else 2), generator=gen, dtype=torch.uint8, device="cuda")
            for _ in range(2))
    want = b.clone()
    want[dst] = a[src]
    rac.rac_cache_copy(cfg, a, i32(src), b, i32(dst), n)
    torch.cuda.synchronize()
    assert torch.equal(b, want)
    if n >= 5:  # within one pool, and a pair that names no page
        want = b.clone()
        want[[0, 1]] = b[[2, 3]]
        rac.rac_cache_copy(cfg, b, i32([2, 99999, 3]), b, i32([0, 4, 1]))
        torch.cuda.synchronize()
        assert torch.equal(b, want)


def test_a_round_as_a_graph():
    """Fork and commit recorded once and replayed on changing device arrays."""
    cfg = config(seqs=4, pages=40, width=6)
    calls = {}
    k = torch.randn(2, 8, 3, 32, dtype=torch.float32).bfloat16().cuda()
    v = torch.randn(2, 8, 3, 32, dtype=torch.float32).bfloat16().cuda()
    start, parents, path = i32([0, 2, 4, 6, 8]), i32([0, 0, 0, 0]), i32([[0, 1]] * 4)
    states = []
    for name in ("eager", "graph"):
        pool = torch.zeros(rac.rac_cache_pool_bytes(cfg) // 2, dtype=torch.int16, device="cuda")
        states.append((pool, *rac.rac_cache_new(cfg), torch.zeros(4, dtype=torch.int32, device="cuda"),
                       torch.empty(rac.rac_cache_commit_workspace(cfg), dtype=torch.uint8, device="cuda")))

    def step(state):
        pool, table, lengths, refs, out, ws = state
        rac.rac_cache_fork(cfg, parents, table, lengths, refs)
        rac.rac_cache_commit(cfg, pool, table, lengths, refs, k, v, start, out, ws, path=path)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        step(states[1])
    for i in range(5):
        parents.copy_(i32([i % 2, i % 2, (i + 1) % 4, 3 if i < 3 else -1]))
        path.copy_(i32([[0, 1], [1, -1], [0, -1], [-1, 0]]))
        torch.cuda.synchronize()
        step(states[0])
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(states[0][:5], states[1][:5]):
            assert torch.equal(a, b), i
