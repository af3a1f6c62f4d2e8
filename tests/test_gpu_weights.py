"""The attention weight that cached and drafted tokens receive against its binary64
form (tests/eviction_reference.py, where the tolerance is derived).

As in the attention's tests, every place that no sequence owns holds NaN."""
from __future__ import annotations

import math
import random

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests import eviction_reference as E
from tests.gpu_util import say
from tests.test_gpu_cache_guards import Guarded, nonsense
from tests.test_gpu_tree_attention import ODD, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


class Sums:
    """The sums of a batch: what they held, and a call of rac_tree_weights."""

    def __init__(self, b, per_head=False, seed=0):
        c = b.cfg
        self.b, self.sets = b, c.layers * c.kv_heads if per_head else 1
        gen = torch.Generator().manual_seed(seed)
        self.weight = torch.rand(c.seqs, self.sets, c.max_pages * c.page_tokens, generator=gen)
        self.draft = torch.rand(self.sets, b.k.shape[0], generator=gen)
        self.lse = b.run()[1]

    def run(self, stream=None, strided=False, garbage=0, drafts=True):
        b = self.b
        dev = lambda t: None if t is None else t.cuda()
        apart = (lambda t: torch.cat([t, torch.full_like(t, math.nan)], 1).cuda()[:, :t.shape[1]]) if strided else dev
        weight, draft = self.weight.cuda(), self.draft.cuda() if drafts else None
        ws = torch.full((rac.rac_tree_weights_workspace(b.cfg, b.tree),), garbage, dtype=torch.uint8, device="cuda")
        args = (b.cfg, b.tree, b.layer, dev(b.pool), dev(b.table), dev(b.lengths), apart(b.q), dev(b.q_start), apart(b.k),
                dev(self.lse), weight, ws)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        rac.rac_tree_weights(*args, draft_weight=draft, draft_start=dev(b.d_start), mask=dev(b.words), stream=stream)
        torch.cuda.synchronize()
        return weight.cpu(), None if draft is None else draft.cpu()

    def check(self, weight, draft):
        b, c = self.b, self.b.cfg
        scale, first = b.scale or 1.0 / math.sqrt(b.dim), b.layer * c.kv_heads if self.sets > 1 else 0
        want, tol = self.weight.double().clone(), torch.zeros_like(self.weight, dtype=torch.float64)
        dwant, dtol = self.draft.double().clone(), torch.zeros_like(self.draft, dtype=torch.float64)
        worst = 0.0
        for s, (length, m, n) in enumerate(b.shapes):
            if not m:
                continue
            q0, d0 = int(b.q_start[s]), int(b.d_start[s])
            see = R.visible(length, n, m, b.window, None if b.masks[s] is None else torch.from_numpy(b.masks[s]), b.there[s])
            k = torch.cat([b.past[s][0].transpose(0, 1), b.k[d0:d0 + n].double()])
            got, slack, terms = E.weights(b.q[q0:q0 + m].double(), k, see, self.lse[q0:q0 + m].double(), scale)
            if self.sets == 1:
                got, slack, terms = got.sum(0, keepdim=True), slack.sum(0, keepdim=True), terms * c.kv_heads
            at = slice(first, first + got.shape[0])
            before = self.weight[s, at, :length].double()
            tol[s, at, :length] = E.tolerance(got[:, :length], slack[:, :length], terms, before)
            want[s, at, :length] += got[:, :length]
            before = self.draft[at, d0:d0 + n].double()
            dtol[at, d0:d0 + n] = E.tolerance(got[:, length:], slack[:, length:], terms, before)
            dwant[at, d0:d0 + n] += got[:, length:]
        for what, x, y, t in (("committed", weight, want, tol), ("drafted", draft, dwant, dtol)):
            if x is None or not x.numel():
                continue
            off = (x.double() - y).abs()
            assert torch.isfinite(x).all(), what
            assert (off <= t).all(), f"{what}: off by {float((off / t.clamp(min=1e-30)).max()):.2f} of the bound"
            worst = max(worst, float((off / t.clamp(min=1e-30)).max()))
        return worst


def check(b, per_head=False, **how):
    s = Sums(b, per_head)
    return s.check(*s.run(**how))


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("q_heads,kv_heads,dim,page", [
    (8, 8, 64, 16), (7, 1, 80, 8), (12, 3, 128, 32), (4, 2, 16, 64), (16, 1, 256, 16), (6, 2, 112, 128), (3, 3, 192, 8),
    (40, 2, 96, 256)])
def test_ragged_trees(kind, q_heads, kv_heads, dim, page):
    say(f"[gpu] weights type {kind} heads {q_heads}/{kv_heads} x {dim}, pages of {page}")
    b = Batch(ODD, q_heads, kv_heads, dim, page, kind, mask="tree", seed=dim, gap=2)
    say(f"[gpu]   worst {check(b):.2f}, by head {check(b, True):.2f} of the bound")


@pytest.mark.parametrize("mask", ["none", "tree", "random"])
@pytest.mark.parametrize("window", [0, 1, 2, 5, 64, 100, 5000])
def test_windows_and_masks(mask, window):
    say(f"[gpu] weights mask {mask} window {window}")
    b = Batch(ODD + [(1000, 4, 4), (200, 70, 70)], 6, 2, 64, 16, window=window, mask=mask, seed=window, stray_bits=True)
    check(b)
    check(b, True)


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("shapes", [
    [(5000, 1, 1)], [(4097, 1, 1), (3, 1, 1), (2900, 1, 1)], [(1, 130, 130)], [(777, 200, 200), (0, 65, 65)],
    [(1500, 33, 33), (20, 64, 64), (600, 16, 16)]], ids=str)
def test_long_axes_and_many_rows(kind, shapes):
    say(f"[gpu] weights type {kind} {shapes}")
    for q_heads, kv_heads, dim in ((8, 2, 128), (4, 4, 64)):
        b = Batch(shapes, q_heads, kv_heads, dim, 16, kind, mask="none", seed=len(shapes))
        check(b)
        check(b, True)


@pytest.mark.parametrize("shapes", [
    [(50, 2, 9), (0, 1, 6), (130, 4, 70), (9, 3, 3)], [(50, 9, 2), (0, 4, 0), (10, 3, 1)],
    [(40, 5, 0), (0, 2, 0), (64, 1, 0)]], ids=["last level", "rows ahead", "no drafts"])
@pytest.mark.parametrize("window", [0, 6])
def test_queries_that_are_not_the_drafted_tokens(shapes, window):
    for mask in ("none", "random"):
        check(Batch(shapes, 4, 2, 64, 16, mask=mask, window=window, seed=5))


def test_more_than_64_drafted_tokens_under_a_mask():
    for mask, window in (("tree", 0), ("random", 0), ("random", 40), ("tree", 3)):
        check(Batch([(100, 130, 130), (0, 200, 200), (33, 65, 65)], 4, 4, 64, 16, mask=mask, branch=3, window=window, seed=9))


def test_more_sequences_than_lanes_and_threads():
    for count in (70, 300, 1030):
        b = Batch([(17 * i % 90, 1 + i % 3, 1 + i % 3) for i in range(count)], 4, 2, 64, 16, mask="tree", seed=count, layers=1,
                  layer=0)
        check(b)
        check(b, True)


def test_positions_without_a_page_get_nothing():
    holes = {(0, 0), (0, 3), (1, 0), (1, 1), (2, 2)}
    for window in (0, 50):
        b = Batch([(100, 3, 3), (32, 2, 2), (40, 1, 1), (70, 1, 1)], 4, 2, 64, 16, mask="tree", holes=holes, window=window)
        check(b)
        s = Sums(b)
        weight, _ = s.run()
        assert torch.equal(weight[0, :, 0:16], s.weight[0, :, 0:16]) and torch.equal(weight[0, :, 48:64], s.weight[0, :, 48:64])


def test_rows_that_see_nothing_give_nothing():
    b = Batch([(0, 4, 4), (16, 3, 3)], 4, 2, 64, 16, mask="random", holes={(1, 0)}, seed=3)
    b.words[0] = b.words[5] = 0
    b.masks[0][0] = b.masks[1][1] = False
    check(b)


@pytest.mark.parametrize("kind", [R.BF16, R.FP16])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_non_finite_keys_reach_only_their_own_sums(kind, value):
    """A drafted key that some rows must not see: the others' sums are as if it had been any
    other (its own score makes the lse of the rows that see it what it is)."""
    b = Batch([(40, 5, 5), (0, 3, 3), (100, 33, 33)], 8, 2, 64, 16, kind, mask="tree", seed=1)
    s = Sums(b)
    clean = s.run()
    at = int(b.d_start[2]) + 20
    sees = torch.from_numpy(b.masks[2][:, 20])
    q0 = int(b.q_start[2])
    s.lse[q0:q0 + 33][sees] = -math.inf  # (so give nothing)
    want = s.run()
    b.k[at] = value
    got = s.run()
    keep = torch.ones(b.k.shape[0], dtype=torch.bool)
    keep[at] = False
    assert torch.equal(got[0], want[0]) and torch.equal(got[1][:, keep], want[1][:, keep])
    assert torch.equal(got[1][:, at], s.draft[:, at]) and not torch.equal(clean[0], want[0])


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_non_finite_cached_key_leaves_the_others(value):
    b = Batch([(100, 3, 3), (70, 20, 20)], 8, 2, 64, 16, mask="tree", seed=1)
    s = Sums(b)
    want = s.run()
    for j in (3, 69):
        b.pool[int(b.table[1, j // 16]), b.layer, 0, :, j % 16] = value
    got = s.run()
    keep = torch.ones(want[0].shape[2], dtype=torch.bool)
    keep[[3, 69]] = False
    assert torch.equal(got[0][1][:, keep], want[0][1][:, keep]) and torch.equal(got[0][0], want[0][0])
    assert torch.equal(got[1], want[1])


def test_scores_far_apart_and_scales():
    for spread in (0.0, 30.0):
        check(Batch([(100, 4, 4), (1, 2, 2), (700, 1, 1)], 4, 1, 128, 16, mask="tree", spread=spread, seed=4))
    check(Batch([(100, 4, 4)], 4, 1, 64, 16, mask="tree", scale=3.5, seed=4))


def test_strides_streams_and_no_drafted_sums():
    b = Batch(ODD, 6, 2, 80, 16, mask="tree", seed=6)
    s = Sums(b)
    want = s.run()
    s.check(*want)
    for got in (s.run(strided=True, garbage=255), s.run(stream=torch.cuda.Stream()), s.run(garbage=0x7F)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    weight, none = s.run(drafts=False)
    s.check(weight, none)


def test_every_row_gives_one_in_all():
    """The weights of a row sum to 1 over what it sees, whatever they are."""
    for kind in (R.BF16, R.FP8):
        b = Batch([(3000, 5, 5), (100, 1, 1), (9000, 3, 3)], 8, 2, 64, 16, kind, mask="tree", seed=8)
        s = Sums(b)
        s.weight.zero_()
        s.draft.zero_()
        weight, draft = s.run()
        # (each weight is off by 2^-14 at most here, and rows times heads of them make a sum)
        for q, (_, m, _) in enumerate(b.shapes):
            d0, d1 = int(b.d_start[q]), int(b.d_start[q + 1])
            total = float(weight[q].double().sum() + draft[:, d0:d1].double().sum())
            assert abs(total - 8 * m) <= 8 * m * 2.0 ** -14


def test_the_same_call_gives_the_same_bits():
    b = Batch([(3000, 5, 5), (100, 1, 1), (9000, 3, 3)], 8, 2, 64, 16, mask="tree", seed=8)
    for per_head in (False, True):
        s = Sums(b, per_head)
        first = s.run()
        for g in (170, 255, 0):
            again = s.run(garbage=g)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_pages_beyond_32_bit_offsets():
    cfg = rac.CacheConfig(1, 8, 128, 64, 20000, 2, 4, R.BF16)  # 256 KiB a page
    pool = torch.empty(20000, 1, 2, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    pool[:4] = torch.randn(4, 1, 2, 8, 64, 128, device="cuda", generator=gen)
    high = [19999, 18001, 17003, 16385]
    for i, p in enumerate(high):
        pool[p] = pool[i]
    lengths = torch.tensor([200, 129], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 16, 128, device="cuda", generator=gen).bfloat16()
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    k = torch.randn(2, 8, 128, device="cuda", generator=gen).bfloat16()
    lse = torch.full((2, 16), 5.0, device="cuda")
    tree, outs = rac.TreeConfig(16, 2, 1, 1), []
    for ids in ([0, 1, 2, 3], high):
        table = torch.tensor([ids, ids[:3] + [-1]], dtype=torch.int32, device="cuda")
        weight, ws = torch.zeros(2, 1, 256, device="cuda"), torch.empty(rac.rac_tree_weights_workspace(cfg, tree), dtype=torch.uint8, device="cuda")
        rac.rac_tree_weights(cfg, tree, 0, pool, table, lengths, q, start, k, lse, weight, ws)
        outs.append(weight.cpu())
    assert torch.equal(outs[0], outs[1]) and (outs[0][0, 0, :200] > 0).all() and not outs[0][0, 0, 200:].any()


@pytest.mark.parametrize("kind", [R.BF16, R.FP8])
def test_broken_device_arrays_between_guards(kind):
    for name, shapes, q_heads, kv_heads, dim in (("few", ODD, 4, 2, 64), ("many", [(0, 33, 33), (700, 40, 40), (31, 9, 9)], 8, 2, 128),
                                                 ("wide", [(100, 1, 1), (9, 30, 30)], 4, 2, 192),
                                                 ("sequences", [(17 * i % 900, 2, 2) for i in range(70)], 4, 2, 80)):
        say(f"[gpu] weights with broken arrays, {name}, type {kind}")
        for seed in range(6):
            rng = random.Random(seed)
            b = Batch(shapes, q_heads, kv_heads, dim, 16, kind, mask="tree" if seed % 2 else "none", seed=seed,
                      window=(0, 0, 5, 100)[seed % 4])
            g, rows, S = Guarded(), b.tree.rows, len(shapes)
            lengths, table = nonsense(rng, b.lengths, 16 * b.cfg.max_pages), nonsense(rng, b.table, b.cfg.pages)
            q_start, d_start = nonsense(rng, b.q_start, rows), nonsense(rng, b.d_start, b.k.shape[0])
            if seed == 5:
                q_start = torch.tensor([(s % 2) * rows for s in range(S + 1)], dtype=torch.int32)
                d_start, lengths = q_start.clone(), torch.full_like(lengths, 1 << 30)
            sets = 1 if seed < 3 else b.cfg.layers * kv_heads
            weight = g(torch.zeros(S, sets, b.cfg.max_pages * 16))
            draft = g(torch.zeros(sets, b.k.shape[0]))
            ws = g(torch.zeros(rac.rac_tree_weights_workspace(b.cfg, b.tree), dtype=torch.uint8))
            rac.rac_tree_weights(
                b.cfg, b.tree, b.layer, g.read_only(b.pool.view(torch.uint8)), g.read_only(table), g.read_only(lengths),
                g.read_only(b.q), g.read_only(q_start), g.read_only(b.k), g.read_only(torch.zeros(rows, q_heads)), weight, ws,
                draft_weight=draft, draft_start=g.read_only(d_start), mask=None if b.words is None else g.read_only(b.words))
            g.check()
            at = b.cfg.kv_heads * b.layer if sets > 1 else 0
            assert not weight[:, :at].any() and not weight[:, at + (kv_heads if sets > 1 else 1):].any()


def test_graphs_that_share_their_scratch():
    made = []
    for seed, shapes in ((1, [(3000, 2, 2), (40, 1, 1)]), (2, [(700, 30, 30)])):
        b = Batch(shapes, 8, 2, 64, 16, mask="tree", seed=seed)
        s = Sums(b)
        dev = lambda t: t.cuda()
        made.append((s, [dev(b.pool), dev(b.table), dev(b.lengths), dev(b.q), dev(b.q_start), dev(b.k), dev(s.lse)],
                     dev(s.weight), dev(s.draft), dev(b.words), dev(b.d_start)))
    ws = torch.empty(max(rac.rac_tree_weights_workspace(s.b.cfg, s.b.tree) for s, *_ in made), dtype=torch.uint8, device="cuda")
    graphs = []
    for s, a, weight, draft, words, start in made:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            rac.rac_tree_weights(s.b.cfg, s.b.tree, 1, *a, weight, ws, draft_weight=draft, draft_start=start, mask=words)
        graphs.append(g)
    for _ in range(3):
        for (s, a, weight, draft, *_), g in zip(made, graphs):
            weight.copy_(s.weight)
            draft.copy_(s.draft)
            g.replay()
        torch.cuda.synchronize()
        for s, a, weight, draft, *_ in made:
            want = s.run()
            assert torch.equal(weight.cpu(), want[0]) and torch.equal(draft.cpu(), want[1])


@pytest.mark.parametrize("per_head", [False, True])
def test_the_sums_of_appended_tokens(per_head):
    cfg = rac.CacheConfig(2, 3, 16, 8, 200, 5, 20)
    sets = 6 if per_head else 1
    gen = torch.Generator().manual_seed(1)
    weight, draft = torch.rand(5, sets, 160, generator=gen), torch.rand(sets, 30, generator=gen)
    start, lengths = [0, 4, 4, 14, 20, 30], [10, 0, 160, 33, 7]
    committed, path = [3, 0, 4, 2, 7], [[2, 0, 3, -1, -1, -1, -1], [-1] * 7, [9, 8, 7, 6, -1, -1, -1],
                                        [5, 1, -1, -1, -1, -1, -1], [0, 1, 2, 3, 4, 5, 6]]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for given in (True, False):
        for with_path in (True, False):
            got, want = weight.cuda(), weight.clone()
            for s, n in enumerate(committed):
                for i in range(n):
                    row = start[s] + (path[s][i] if with_path else i)
                    want[s, :, lengths[s] - n + i] = draft[:, row] if given else 0.0
            rac.rac_cache_weights_commit(cfg, i32(lengths), i32(committed), i32(start), draft.cuda() if given else None, got,
                                         path=i32(path) if with_path else None, draft_rows=30)
            assert torch.equal(got.cpu(), want)


def test_appended_sums_with_broken_arrays_between_guards():
    cfg = rac.CacheConfig(2, 3, 16, 8, 200, 300, 20)
    for seed in range(4):
        rng, g = random.Random(seed), Guarded()
        one = lambda n, top: g.read_only(nonsense(rng, torch.randint(0, top, (n,), dtype=torch.int32), top))
        weight, draft = g(torch.zeros(300, 6, 160)), g.read_only(torch.rand(6, 900))
        path = g.read_only(nonsense(rng, torch.zeros(300, 4, dtype=torch.int32), 4))
        rac.rac_cache_weights_commit(cfg, one(300, 160), one(300, 5), one(301, 900), draft, weight, path=path if seed % 2 else None)
        g.check()
