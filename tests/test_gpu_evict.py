"""Eviction against the contract's words (tests/eviction_reference.py): every table
entry, count, sum, source and stored byte is equal."""
from __future__ import annotations

import math
import random

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import eviction_reference as E
from tests.gpu_util import say
from tests.test_gpu_cache_guards import Guarded, nonsense

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Cache:
    """A cache of random bytes and sums.  lengths of sequences with pages of their own;
    share: (sequence, parent) that hold the parent's pages instead; gaps: (sequence, page)
    without a page; spare: free pages."""

    def __init__(self, lengths, page=16, layers=2, heads=3, dim=32, kind=0, sets=1, share=(), gaps=(), spare=20, width=None,
                 seed=0, ties=0):
        rng, gen = random.Random(seed), torch.Generator().manual_seed(seed)
        width = width or max(-(-n // page) for n in lengths) + 1
        own = [0 if s in dict(share) else -(-n // page) for s, n in enumerate(lengths)]
        pages = sum(own) + spare
        self.cfg = rac.CacheConfig(layers, heads, dim, page, pages, len(lengths), width, kind)
        self.sets = layers * heads if sets != 1 else 1
        ids = list(range(pages))
        rng.shuffle(ids)
        table = [[ids.pop() for _ in range(k)] + [-1] * (width - k) for k in own]
        lengths = list(lengths)
        for s, parent in share:
            table[s] = table[parent][:-(-lengths[s] // page)]
            table[s] += [-1] * (width - len(table[s]))
        for s, j in gaps:
            table[s][j] = -1 - rng.randrange(3)
        refs = [0] * pages
        for row in table:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        self.model = E.Bounded(pages, page, table, lengths, refs)
        self.weight = torch.rand(len(lengths), self.sets, width * page, generator=gen)
        if ties:
            self.weight = (self.weight * ties).floor()
        size = 1 if kind == rac.RAC_CACHE_FP8 else 2
        self.want = torch.randint(0, 256, (pages, layers, 2, heads, page, dim * size), dtype=torch.uint8, generator=gen)
        self.upload()

    def upload(self):
        self.pool, self.table, self.lengths = self.want.cuda(), i32(self.model.table), i32(self.model.lengths)
        self.refs, self.gpu_weight = i32(self.model.refs), self.weight.cuda()

    def expect(self, keep, first, recent):
        """What an eviction leaves, on the CPU."""
        source = torch.full(self.weight.shape, -9, dtype=torch.int32)
        pool = self.want.clone()
        evicted, moves = self.model.evict(self.weight, keep, first, recent, source)
        H = self.cfg.kv_heads
        P = self.cfg.page_tokens
        for s, g, i, to, page, place in moves:
            heads = [(g // H, g % H)] if self.sets > 1 else [(l, h) for l in range(self.cfg.layers) for h in range(H)]
            for l, h in heads:
                pool[to, l, :, h, i % P] = self.want[page, l, :, h, place % P]
        self.want = pool
        return evicted, source

    def call(self, keep, first, recent, stream=None, garbage=0xA5, source=True):
        evict = rac.EvictConfig(self.sets, first, recent)
        ws = torch.full((rac.rac_cache_evict_workspace(self.cfg, evict),), garbage, dtype=torch.uint8, device="cuda")
        evicted = torch.full((self.cfg.seqs,), -7, dtype=torch.int32, device="cuda")
        src = torch.full(self.weight.shape, -9, dtype=torch.int32, device="cuda") if source else None
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        rac.rac_cache_evict(self.cfg, evict, self.pool, self.table, self.lengths, self.refs, self.gpu_weight, i32(keep), evicted,
                            ws, source=src, stream=stream)
        torch.cuda.synchronize()
        return evicted, src

    def equal(self):
        assert self.table.tolist() == self.model.table
        assert self.lengths.tolist() == self.model.lengths and self.refs.tolist() == self.model.refs
        got = self.gpu_weight.cpu()
        assert torch.equal(got.view(torch.int32), self.weight.view(torch.int32))
        assert torch.equal(self.pool.cpu(), self.want)

    def evict(self, keep, first=0, recent=0, **how):
        want, source = self.expect(keep, first, recent)
        got, src = self.call(keep, first, recent, **how)
        assert got.tolist() == want
        if src is not None:
            assert torch.equal(src.cpu(), source)
        self.equal()
        return want


LENGTHS = [0, 1, 7, 8, 9, 15, 16, 17, 63, 64, 65, 130, 257, 300]


@pytest.mark.parametrize("sets", [1, 2], ids=["one set", "a set a head"])
@pytest.mark.parametrize("page,layers,heads,dim,kind", [(8, 1, 1, 16, 0), (16, 2, 3, 32, 1), (32, 1, 2, 80, 2), (64, 3, 1, 256, 0),
                                                        (256, 1, 5, 16, 2)])
def test_ragged_lengths(page, layers, heads, dim, kind, sets):
    say(f"[gpu] evict pages of {page}, {layers} layers, {heads} heads x {dim}, type {kind}, sets {sets}")
    for first, recent, keep in ((0, 0, [n // 2 for n in LENGTHS]), (4, 8, [max(0, n - 3) for n in LENGTHS]),
                                (2, 100, [n * 3 // 4 for n in LENGTHS]), (1 << 30, 1, [n // 3 for n in LENGTHS]),
                                (3, 1 << 30, [n - 1 for n in LENGTHS]), (1, 2, [0, 0, 3, 8, 10, -1, 1, 16, 64, 2, 64, 5, 256, 301]),
                                (0, 0, [0] * len(LENGTHS)), (5, 5, [1] * len(LENGTHS))):
        Cache(LENGTHS, page, layers, heads, dim, kind, sets, seed=first % 97 + recent % 89).evict(keep, first, recent)


@pytest.mark.parametrize("sets", [1, 2])
def test_ties_and_odd_weights(sets):
    for ties in (1, 2, 5):
        c = Cache([300, 200, 77, 4500], sets=sets, ties=ties, layers=1, heads=2, dim=16, seed=ties)
        c.weight[0, :, ::7] = -0.0
        c.weight[0, :, 3::11] = -1.0
        c.weight[1, :, ::3] = math.nan
        c.weight[1, :, 1::5] = -math.inf
        c.weight[2, :, ::5] = math.inf
        c.weight[2, :, 4::5] = 1e-40
        c.weight[3] = 0.0
        c.upload()
        c.evict([150, 50, 30, 4000], 3, 9)
        c.evict([149, 10, 20, 37], 3, 9)


@pytest.mark.parametrize("sets", [1, 2])
def test_long_sequences(sets):
    for lengths, keep in (([40001, 3000, 9], [20000, 100, 9]), ([70000], [69990])):
        for first, recent in ((4, 64), (0, 2000)):
            say(f"[gpu] evict {lengths} to {keep}, first {first}, recent {recent}, sets {sets}")
            Cache(lengths, 64, 1, 2, 16, 2, sets, seed=recent).evict(keep, first, recent)


@pytest.mark.parametrize("sets", [1, 2])
@pytest.mark.parametrize("ties", [0, 2, 100])
def test_parts_of_sequences(ties, sets):
    """Long caches, whose sequences several workgroups share, or none: cuts, borders and rows of weights that are alike
    in any part; short sequences in long caches; places without a page."""
    for width in (1000, 1500, 2100, 4200):  # positions: to 20000, 28000, and past the length from which parts are made
        cases = (([19999, 8192, 8193, 1], [9000, 8191, 1, 0]), ([width * 16 - 40, 16384, 100, 0], [16384, 16000, 37, -1]),
                 ([width * 16 - 16, 12000, 12000, 12000], [width * 16 - 17, 12000, 11999, 3]))
        for i, (lengths, keep) in enumerate(cases):
            if max(lengths) > width * 16:
                continue
            first, recent = ((0, 0), (5, 3000), (8200, 77))[i]
            say(f"[gpu] evict {lengths} to {keep} in {width} pages, first {first}, recent {recent}, ties {ties}, sets {sets}")
            gaps = ((0, 0), (0, 600), (1, 3), (1, 700)) if i < 2 and lengths[1] > 11300 else ()
            Cache(lengths, 16, 1, 2, 16, 2, sets, width=width, seed=i, ties=ties, gaps=gaps).evict(keep, first, recent)


@pytest.mark.parametrize("sets", [1, 2])
@pytest.mark.parametrize("page", [8, 16, 64])
def test_shared_pages_are_replaced(page, sets):
    """Forks of one sequence: what the others hold stays, byte for byte."""
    for keep, first, recent in (([-1, 100, 60, 150], 4, 10), ([100, 100, 100, 100], 90, 10), ([150, 140, 130, 0], 0, 0),
                                ([-1, 199, -1, 199], 0, 3)):
        c = Cache([200, 200, 180, 200], page, sets=sets, share=((1, 0), (2, 0), (3, 0)), spare=80, seed=page)
        c.evict(keep, first, recent)
        c.evict([k // 2 for k in keep], first, recent)


def test_too_few_pages():
    """Sequences in order: one that cannot have its pages keeps its state, those behind it that can are cut."""
    for spare in (0, 1, 5, 12, 13, 30):
        c = Cache([200, 200, 200, 60, 60, 60], 16, share=((1, 0), (2, 0), (4, 3), (5, 3)), spare=spare, seed=spare)
        got = c.evict([-1, 150, 100, -1, 30, 50], 0, 8)
        assert spare > 0 or set(got) == {0, -1}


@pytest.mark.parametrize("sets", [1, 2])
def test_positions_without_a_page(sets):
    """A window let pages at the front go (and a broken table some elsewhere): places are what is left."""
    for gaps in (((0, 0), (0, 1), (1, 0)), ((0, 2), (0, 5), (1, 12)), ((0, 12), (1, 0), (1, 3), (2, 0))):
        for first, recent, keep in ((4, 10, [90, 100, 40]), (0, 0, [30, 150, 1]), (200, 1, [100, 30, 8]), (0, 70, [80, 99, 16])):
            c = Cache([200, 197, 50], 16, gaps=gaps, sets=sets, seed=recent)
            c.evict(keep, first, recent)
            c.evict([k // 2 for k in keep], first, recent)
    # shared, with gaps
    c = Cache([200, 200, 170], 8, gaps=((0, 0), (1, 0), (1, 1)), share=((1, 0), (2, 0)), sets=sets, spare=60)
    c.evict([100, 90, 80], 3, 20)


def test_many_sequences():
    lengths = [(37 * s) % 70 for s in range(1100)]
    c = Cache(lengths, 8, 1, 1, 16, 0, spare=900, share=[(s, s - 1) for s in range(1, 1100, 3) if lengths[s] <= lengths[s - 1]])
    c.evict([(13 * s) % 60 - 3 for s in range(1100)], 1, 5)


def test_rounds_of_appends_and_evictions():
    """With the cache's own calls between: what is appended, forked and cut again."""
    c = Cache([100, 64, 33, 7], 16, 2, 3, 32, 0, 2, spare=60, seed=5)
    rng = random.Random(1)
    ws = torch.empty(rac.rac_cache_commit_workspace(c.cfg), dtype=torch.uint8, device="cuda")
    for turn in range(4):
        k = torch.randn(2, 20, 3, 32, device="cuda").bfloat16()
        committed = torch.zeros(4, dtype=torch.int32, device="cuda")
        draft = torch.rand(6, 20, device="cuda")
        rac.rac_cache_commit(c.cfg, c.pool, c.table, c.lengths, c.refs, k, k, i32([0, 5, 10, 15, 20]), committed, ws)
        rac.rac_cache_weights_commit(c.cfg, c.lengths, committed, i32([0, 5, 10, 15, 20]), draft, c.gpu_weight)
        if turn == 2:
            rac.rac_cache_fork(c.cfg, i32([0, 0, 2, 2]), c.table, c.lengths, c.refs)
            c.gpu_weight[1], c.gpu_weight[3] = c.gpu_weight[0], c.gpu_weight[2]
        c.model = E.Bounded(c.cfg.pages, 16, c.table.tolist(), c.lengths.tolist(), c.refs.tolist())
        c.want, c.weight = c.pool.cpu(), c.gpu_weight.cpu()
        c.evict([90, 60, 33, rng.randrange(4, 12)], 4, 16)


def test_other_streams_and_no_source():
    for stream in (None, torch.cuda.Stream()):
        c = Cache([300, 200, 77], sets=2, share=((1, 0),), spare=40)
        c.evict([150, 50, 30], 3, 9, stream=stream, source=False, garbage=0xFF)


def test_replayed_from_graphs_that_share_their_scratch():
    caches = [Cache([300, 200, 77], sets=2, share=((1, 0),), spare=40), Cache([500, 100], 32, 1, 2, 16, 1, spare=9, seed=3)]
    keeps, evict = [[150, 50, 30], [400, 99]], [rac.EvictConfig(c.sets, 2, 7) for c in caches]
    ws = torch.zeros(max(rac.rac_cache_evict_workspace(c.cfg, e) for c, e in zip(caches, evict)), dtype=torch.uint8, device="cuda")
    graphs, out = [], []
    for c, e, keep in zip(caches, evict, keeps):
        c.state = [t.clone() for t in (c.pool, c.table, c.lengths, c.refs, c.gpu_weight)]
        c.keep, c.evicted = i32(keep), torch.zeros(c.cfg.seqs, dtype=torch.int32, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            rac.rac_cache_evict(c.cfg, e, c.pool, c.table, c.lengths, c.refs, c.gpu_weight, c.keep, c.evicted, ws)
        graphs.append(g)
    for c, keep in zip(caches, keeps):
        out.append(c.expect(keep, 2, 7)[0])
    for _ in range(3):
        for c, g, want in zip(caches, graphs, out):
            for t, was in zip((c.pool, c.table, c.lengths, c.refs, c.gpu_weight), c.state):
                t.copy_(was)
            g.replay()
        torch.cuda.synchronize()
        for c, want in zip(caches, out):
            assert c.evicted.tolist() == want
            c.equal()


def test_sums_and_pages_beyond_32_bit_offsets():
    """Sums of 2^32 bytes and more, and pages past 4 GiB."""
    cfg = rac.CacheConfig(1, 8, 128, 64, 20000, 300, 65536)  # positions: 2^22; 300 x 2^22 sums; 256 KiB a page
    pool = torch.empty(20000, 1, 2, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    table, lengths, refs = rac.rac_cache_new(cfg)
    ids = [19999, 18001, 17003, 16385]
    table[299, :4] = i32(ids)
    lengths[299] = 250
    refs[ids] = 1
    for i, p in enumerate(ids):
        pool[p] = i
    weight = torch.zeros(300, 1, 1 << 22, device="cuda")
    weight[299, 0, 100:250] = torch.arange(150, device="cuda").float()
    keep = torch.full((300,), -1, dtype=torch.int32, device="cuda")
    keep[299] = 70
    evict, evicted = rac.EvictConfig(1, 2, 3), torch.zeros(300, dtype=torch.int32, device="cuda")
    ws = torch.empty(rac.rac_cache_evict_workspace(cfg, evict), dtype=torch.uint8, device="cuda")
    rac.rac_cache_evict(cfg, evict, pool, table, lengths, refs, weight, keep, evicted, ws)
    torch.cuda.synchronize()
    assert int(evicted[299]) == 180 and int(evicted.abs().sum()) == 180 and int(lengths[299]) == 70
    # places 0, 1, the 65 largest of the middle (182 .. 246) and the last three
    assert weight[299, 0, :70].tolist() == [0.0, 0.0] + [float(v) for v in range(82, 147)] + [147.0, 148.0, 149.0]
    assert not weight[299, 0, 70:].any() and table[299, :3].tolist() == [19999, 18001, -1]
    assert pool[19999, 0, :, :, 0].unique().tolist() == [0.0] and pool[19999, 0, :, :, 2:12].unique().tolist() == [2.0]
    assert pool[19999, 0, :, :, 12:].unique().tolist() == [3.0] and pool[18001, 0, :, :, :6].unique().tolist() == [3.0]
    assert int(refs.sum()) == 2


@pytest.mark.parametrize("seqs,pages,width,page", [(6, 60, 9, 8), (1100, 300, 5, 16), (3, 500, 40, 64)])
@pytest.mark.parametrize("sets", [1, 6])
def test_broken_device_arrays_between_guards(seqs, pages, width, page, sets):
    say(f"[gpu] evict with broken arrays, {seqs} sequences, {pages} pages of {page}, {sets} sets")
    cfg = rac.CacheConfig(2, 3, 32, page, pages, seqs, width, 0)
    for seed in range(6):
        rng, g = random.Random(seed), Guarded()
        held = torch.randint(-1, pages, (seqs, width), dtype=torch.int32, generator=torch.Generator().manual_seed(seed))
        table, refs = g(nonsense(rng, held, pages)), g(nonsense(rng, torch.randint(0, 4, (pages,), dtype=torch.int32), 3))
        lengths = g(nonsense(rng, torch.randint(0, width * page + 1, (seqs,), dtype=torch.int32), width * page))
        keep = g.read_only(nonsense(rng, torch.randint(-1, width * page, (seqs,), dtype=torch.int32), width * page))
        pool = g(torch.zeros(rac.rac_cache_pool_bytes(cfg), dtype=torch.uint8))
        weight, evicted = g(torch.randn(seqs, sets, width * page)), g(torch.zeros(seqs, dtype=torch.int32))
        source = g(torch.zeros(seqs, sets, width * page, dtype=torch.int32))
        evict = rac.EvictConfig(sets, rng.choice([0, 3, 1 << 30]), rng.choice([0, 9, 1 << 30]))
        ws = g(torch.full((rac.rac_cache_evict_workspace(cfg, evict),), 0xFF, dtype=torch.uint8))
        rac.rac_cache_evict(cfg, evict, pool, table, lengths, refs, weight, keep, evicted, ws, source=source)
        g.check()
