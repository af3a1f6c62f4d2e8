"""Commits that ask for more pages than are free.  Sequences are served in order,
each from what those before it left: one that is refused takes nothing, and one
that needs no page is never refused for want of pages."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests.gpu_util import say
from tests.test_gpu_cache import Pair, config

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


class Served(R.Model):
    """The bookkeeping with the sequences served one after the other."""

    def commit(self, accepted):
        refs = self.refs()
        free = [p for p in range(self.pages) if refs[p] == 0]
        committed, copied, writes = [], [], []
        for s, n in enumerate(accepted):
            length, at = self.lengths[s], -(-self.lengths[s] // self.page)
            last = -(-(length + n) // self.page)
            tail = self.table[s][at - 1] if length % self.page else -1
            copies = tail >= 0 and refs[tail] > 1
            if length % self.page and (copies or tail < 0):
                at -= 1
            if n == 0 or last > self.width or last - at > len(free):
                committed.append(0)
                continue
            committed.append(n)
            got, free = free[:last - at], free[last - at:]
            if copies:
                copied.append((tail, got[0], length % self.page))
            self.table[s][at:last] = got
            for i in range(n):
                writes.append((s, i, self.table[s][(length + i) // self.page], (length + i) % self.page))
            self.lengths[s] = length + n
        return committed, copied, writes


def served(cfg, seed=0):
    p = Pair(cfg, seed)
    p.model = Served(cfg.pages, cfg.page_tokens, cfg.seqs, cfg.max_pages)
    return p


def test_a_refused_sequence_takes_nothing_from_those_after_it():
    p = served(config(seqs=4, pages=3, width=9, layers=1, heads=1, dim=16))
    assert p.commit([0, 3, 0, 0]) == [0, 3, 0, 0]
    # four pages of two; none; one of two; two of one
    assert p.commit([25, 1, 8, 9]) == [0, 1, 8, 0]
    assert p.commit([1, 4, 0, 8]) == [1, 4, 0, 0]
    assert p.commit([7, 0, 1, 1]) == [7, 0, 0, 0]  # nothing is free: places in pages that are there
    p.fork([0, 0, 1, 3], keep_to=[3, 3, 8, 0])
    assert p.commit([2, 2, 8, 1]) == [2, 0, 0, 0]  # (the first copies the page that it shares, the second cannot)
    assert p.commit([0, 2, 0, 0]) == [0, 2, 0, 0]  # (and has it alone)


def test_random_lives_under_pressure():
    say("[gpu] random lives of a cache that is too small")
    refused = after = 0
    for seed in range(8):
        p = served(config(seqs=9, pages=14, width=6, layers=1, heads=1, dim=16), seed=seed)
        rng = p.rng
        for _ in range(14):
            if rng.random() < 0.4:
                p.fork([rng.randrange(-1, 9) if rng.random() < 0.4 else d for d in range(9)],
                       keep_to=[rng.randrange(0, 48) for _ in range(9)])
            else:
                drafted = [rng.choice([0, 1, 2, 7, 8, 9, 20, 40]) for _ in range(9)]
                got = p.commit(drafted)
                no = [s for s, n in enumerate(drafted) if n and not got[s]]
                refused += len(no)
                after += sum(n > 0 for s, n in enumerate(got) if no and s > no[0])
    assert refused > 50 and after > 50  # (both happen)


@pytest.mark.parametrize("seqs", [1500, 4096])
def test_many_sequences_and_too_few_pages(seqs):
    say(f"[gpu] {seqs} sequences, too few pages")
    p = served(rac.CacheConfig(1, 1, 16, 8, 5000, seqs, 12, R.BF16))
    drafted = [(s * 7) % 60 for s in range(seqs)]
    got = p.commit(drafted)
    no = [s for s, n in enumerate(drafted) if n and not got[s]]
    assert no and any(got[no[0]:])
    p.fork([s // 2 for s in range(seqs)], keep_to=[(s * 5) % 70 for s in range(seqs)])
    p.commit([(s * 3) % 40 for s in range(seqs)])


def test_more_than_4096_pages_from_a_pool_of_more_than_16384():
    p = served(rac.CacheConfig(1, 1, 16, 8, 40000, 5, 14000, R.BF16))
    assert p.commit([90000, 7, 60000, 0, 1]) == [90000, 7, 60000, 0, 1]
    p.fork([0, -1, 1, 2, 0], keep_to=[80001, 0, 0, 60000, 70000])
    # (most free pages lie behind the first 16384)
    assert p.commit([30000, 100000, 40000, 1, 3]) == [30000, 100000, 40000, 1, 3]


def test_demands_that_add_up_to_more_than_32_bits():
    """Ranges of drafted rows that overlap, as a broken draft_start has them: 2047
    sequences that ask for 2^20 + 1024 pages each, of a pool of 64."""
    rows, seqs = (1 << 23) + 8192, 4096
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("24 GiB of device memory are not free")
    say("[gpu] a demand of 2^31 pages")
    cfg = rac.CacheConfig(1, 1, 16, 8, 64, seqs, rows // 8, R.BF16)
    table, lengths, refs = rac.rac_cache_new(cfg)  # (16 GiB)
    pool = torch.full((rac.rac_cache_pool_bytes(cfg) // 2,), 7, dtype=torch.int16, device="cuda")
    k = torch.randn(1, rows, 1, 16, device="cuda").bfloat16()
    start = torch.tensor([0, rows] * (seqs // 2) + [0], dtype=torch.int32, device="cuda")
    start[-3:] = torch.tensor([rows - 9, rows, rows], dtype=torch.int32)
    out = torch.full((seqs,), -3, dtype=torch.int32, device="cuda")
    ws = torch.empty(rac.rac_cache_commit_workspace(cfg), dtype=torch.uint8, device="cuda")
    rac.rac_cache_commit(cfg, pool, table, lengths, refs, k, k, start, out, ws)
    torch.cuda.synchronize()
    want = [0] * seqs
    want[-2] = 9  # (the last rows once more)
    assert out.tolist() == want and lengths.tolist() == want
    assert refs.tolist() == [1, 1] + [0] * 62 and table[-2, :3].tolist() == [0, 1, -1]
    assert int((table >= 0).sum()) == 2
    pages = pool.view(64, 2, 8, 16)
    got = torch.cat([pages[0], pages[1, :, :1]], 1)
    assert torch.equal(got, k[0, -9:, 0].view(torch.int16).expand(2, 9, 16))
    assert (pages[1, :, 1:] == 7).all() and (pages[2:] == 7).all()
    del table, k
    torch.cuda.empty_cache()
