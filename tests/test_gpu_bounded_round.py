"""Rounds of drafted trees over a bounded cache, all calls together: rotary positions,
attention, the weight that tokens receive, log probabilities of the drafted tokens, the
commit of an accepted path with its weights, and eviction.

Beside the library a plain model keeps, per sequence, layer and head, which token is at
every position.  Each step is checked against its definition on what the step before left."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests import cache_reference as R
from tests import eviction_reference as E

pytestmark = pytest.mark.gpu

S, LAYERS, HEADS, GROUP, DIM, PAGE, NODES, VOCAB, BUDGET = 3, 2, 2, 3, 32, 8, 7, 501, 40


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def parent(i):
    return (i - 1) // 2


def path_to(i):
    return (path_to(parent(i)) if i else []) + [i]


class Rounds:
    """What a program keeps, and one round of its calls."""

    def __init__(self, seed, sets):
        self.gen, self.sets, Q, rows = torch.Generator().manual_seed(seed), sets, HEADS * GROUP, S * NODES
        self.cfg = rac.CacheConfig(LAYERS, HEADS, DIM, PAGE, 60, S, 9)
        self.tree = rac.TreeConfig(Q, rows, NODES, NODES)
        self.turn = rac.RotaryConfig(rows, Q, HEADS, DIM, DIM, layout=rac.RAC_ROTARY_HALF)
        self.freq = torch.tensor(rac.rac_rotary_frequencies(DIM, 10000.0), dtype=torch.float64, device="cuda")
        self.score = rac.LogprobConfig(rows, VOCAB, rows, 3)
        self.cut = rac.EvictConfig(sets, 2, 10)
        self.pool = torch.zeros(60, LAYERS, 2, HEADS, PAGE, DIM, dtype=torch.bfloat16, device="cuda")
        self.table, self.lengths, self.refs = rac.rac_cache_new(self.cfg)
        self.weight = torch.zeros(S, sets, 9 * PAGE, device="cuda")
        self.source = torch.zeros(S, sets, 9 * PAGE, dtype=torch.int32, device="cuda")
        self.ws = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (
            rac.rac_tree_attention_workspace(self.cfg, self.tree), rac.rac_tree_weights_workspace(self.cfg, self.tree),
            rac.rac_logprobs_workspace(self.score), rac.rac_cache_commit_workspace(self.cfg),
            rac.rac_cache_evict_workspace(self.cfg, self.cut))]
        self.start = i32([NODES * s for s in range(S + 1)])
        see = [sum(1 << j for j in path_to(i)) for i in range(NODES)]
        self.mask = torch.tensor([[w] for _ in range(S) for w in see], dtype=torch.int64, device="cuda")
        # (a root is scored by the row of its own sequence's last round; here it stays out of the rows)
        self.of = i32([NODES * s + parent(i) if i else -1 for s in range(S) for i in range(NODES)])
        new = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")
        self.q, self.qr = new(LAYERS, rows, Q, DIM, dtype=torch.bfloat16), new(LAYERS, rows, Q, DIM, dtype=torch.bfloat16)
        self.k, self.kr, self.v = (new(LAYERS, rows, HEADS, DIM, dtype=torch.bfloat16) for _ in range(3))
        self.out, self.lse = new(LAYERS, rows, Q, DIM, dtype=torch.bfloat16), new(LAYERS, rows, Q)
        self.logits, self.tokens = new(rows, VOCAB, dtype=torch.bfloat16), new(rows, dtype=torch.int32)
        self.logprob, self.row_lse, self.entropy = new(rows), new(rows), new(rows)
        self.ids, self.tops = new(rows, 3, dtype=torch.int32), new(rows, 3)
        self.draft, self.pos = new(sets, rows), new(rows, dtype=torch.int32)
        self.path, self.committed, self.evicted = new(S, 4, dtype=torch.int32), i32([0] * S), i32([0] * S)
        self.keep = i32([BUDGET, BUDGET - 7, -1])

    def draw(self, ages):
        """The inputs of a round: `ages` tokens each sequence has seen."""
        rnd = lambda t: t.copy_(torch.randn(t.shape, generator=self.gen))
        for t in (self.q, self.k, self.v, self.logits):
            rnd(t)
        self.tokens.copy_(torch.randint(0, VOCAB, self.tokens.shape, generator=self.gen))
        depth = [len(path_to(i)) - 1 for i in range(NODES)]
        self.pos.copy_(i32([a + depth[i] for a in ages for i in range(NODES)]))
        ends = torch.randint(0, NODES, (S,), generator=self.gen).tolist()
        self.paths = [path_to(e) for e in ends]
        self.path.copy_(i32([p + [-1] * (4 - len(p)) for p in self.paths]))

    def calls(self):
        self.draft.zero_()
        for l in range(LAYERS):
            rac.rac_rotary(self.turn, self.pos, self.freq, self.q[l], self.k[l], q_out=self.qr[l], k_out=self.kr[l])
            rac.rac_tree_attention(self.cfg, self.tree, l, self.pool, self.table, self.lengths, self.qr[l], self.start, self.kr[l],
                                   self.v[l], self.out[l], self.ws[0], mask=self.mask, lse=self.lse[l])
            rac.rac_tree_weights(self.cfg, self.tree, l, self.pool, self.table, self.lengths, self.qr[l], self.start, self.kr[l],
                                 self.lse[l], self.weight, self.ws[1], draft_weight=self.draft, mask=self.mask)
        rac.rac_logprobs(self.score, self.logits, self.tokens, self.logprob, self.row_lse, self.ws[2], token_rows=self.of,
                         entropy=self.entropy, top_ids=self.ids, top_logprobs=self.tops)
        rac.rac_cache_commit(self.cfg, self.pool, self.table, self.lengths, self.refs, self.kr, self.v, self.start,
                             self.committed, self.ws[3], path=self.path)
        rac.rac_cache_weights_commit(self.cfg, self.lengths, self.committed, self.start, self.draft, self.weight, path=self.path)
        rac.rac_cache_evict(self.cfg, self.cut, self.pool, self.table, self.lengths, self.refs, self.weight, self.keep,
                            self.evicted, self.ws[4], source=self.source)

    def state(self):
        return [self.pool, self.table, self.lengths, self.refs, self.weight]

    def results(self):
        return self.state() + [self.qr, self.kr, self.out, self.lse, self.logprob, self.row_lse, self.entropy, self.ids,
                               self.tops, self.draft, self.committed, self.evicted]


@pytest.mark.parametrize("sets", [1, LAYERS * HEADS])
def test_rounds(sets):
    r = Rounds(sets, sets)
    held = [[[] for _ in range(LAYERS * HEADS)] for _ in range(S)]  # (key, value) at every position
    ages = [0] * S
    for turn in range(24):
        r.draw(ages)
        before, old_lengths = r.weight.cpu(), r.lengths.tolist()
        r.calls()
        torch.cuda.synchronize()
        q, k, v, lse, out = r.qr.cpu(), r.kr.cpu(), r.v.cpu(), r.lse.cpu().double(), r.out.cpu()
        # rotary: against complex numbers, to a bf16 rounding
        turns = r.pos.cpu().double()[:, None] * r.freq.cpu()
        by = torch.polar(torch.ones_like(turns), 2 * math.pi * turns)[None, :, None]
        for x, y in ((r.q, q), (r.k, k)):
            z = torch.complex(*x.cpu().double().chunk(2, dim=-1)) * by
            want = torch.cat([z.real, z.imag], -1)
            assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17 * 5).all()
        see = torch.zeros(NODES, NODES, dtype=torch.bool)
        for i in range(NODES):
            see[i, path_to(i)] = True
        grown = before.double()
        tol = torch.zeros_like(grown)
        draft = torch.zeros(sets, S * NODES, dtype=torch.float64)
        dtol = torch.zeros_like(draft)
        for s in range(S):
            rows, n = slice(NODES * s, NODES * s + NODES), old_lengths[s]
            sees = torch.cat([torch.ones(NODES, n, dtype=torch.bool), see], 1)
            for l in range(LAYERS):
                past = [torch.stack([torch.stack([t[i] for t in held[s][l * HEADS + h]]) if n else torch.zeros(0, DIM)
                                     for h in range(HEADS)], 1).double() for i in (0, 1)]
                kk, vv = torch.cat([past[0], k[l, rows].double()]), torch.cat([past[1], v[l, rows].double()])
                want, wl, size, reach, keys = R.attention(q[l, rows].double(), kk, vv, sees, DIM ** -0.5)
                t, tl = R.tolerances(R.BF16, want, wl, size, reach, keys.double(), float(vv.abs().max()), DIM)
                assert ((out[l, rows].double() - want).abs() <= t).all() and ((lse[l, rows] - wl).abs() <= tl).all()
                got, slack, terms = E.weights(q[l, rows].double(), kk, sees, lse[l, rows], DIM ** -0.5)
                at = slice(l * HEADS, l * HEADS + HEADS) if sets > 1 else slice(0, 1)
                if sets == 1:
                    got, slack, terms = got.sum(0, keepdim=True), slack.sum(0, keepdim=True), terms * HEADS
                tol[s, at, :n] += E.tolerance(got[:, :n], slack[:, :n], terms, grown[s, at, :n])
                grown[s, at, :n] += got[:, :n]
                dtol[at, rows] += E.tolerance(got[:, n:], slack[:, n:], terms, draft[at, rows])
                draft[at, rows] += got[:, n:]
        assert ((r.draft.cpu().double() - draft).abs() <= dtol).all()
        # log probabilities: children in their parents' rows, roots by no row
        x = torch.log_softmax(r.logits.cpu().double(), 1)
        for j, (row, token) in enumerate(zip(r.of.tolist(), r.tokens.tolist())):
            want = float(x[row, token]) if row >= 0 else 0.0
            assert abs(float(r.logprob[j]) - want) <= 2.0 ** -16
        assert torch.equal(r.ids.cpu().long(), torch.argsort(r.logits.cpu().float(), dim=1, descending=True, stable=True)[:, :3])
        # what was accepted is at the end; then the model is cut as the sources say, which the eviction's own tests prove
        source = r.source.cpu()
        for s in range(S):
            p = r.paths[s]
            assert int(r.committed[s]) == len(p)
            ages[s] += len(p)
            for g in range(LAYERS * HEADS):
                l, h = g // HEADS, g % HEADS
                held[s][g] += [(k[l, NODES * s + i, h], v[l, NODES * s + i, h]) for i in p]
            n, most = old_lengths[s] + len(p), int(r.keep[s])
            for g in range(sets):
                grown[s, g, old_lengths[s]:n] = draft[g, [NODES * s + i for i in p]]
                tol[s, g, old_lengths[s]:n] = dtol[g, [NODES * s + i for i in p]]
            if 0 <= most < n:
                assert int(r.evicted[s]) == n - most
                for g in range(sets):
                    src = source[s, g, :most].long()
                    # the sources are those of the largest sums: no token let go weighs more than one chosen
                    gone = sorted(set(range(2, n - 10)) - set(src.tolist()))
                    chosen = [j for j in src.tolist() if 2 <= j < n - 10]
                    slack = float(tol[s, g, :n].max())
                    assert max(grown[s, g, gone]) <= min(grown[s, g, chosen]) + 2 * slack
                    assert len(set(src.tolist())) == most and src[most - 10:].tolist() == list(range(n - 10, n))
                    grown[s, g, :n] = torch.cat([grown[s, g, src], torch.zeros(n - most, dtype=torch.float64)])
                    tol[s, g, :n] = torch.cat([tol[s, g, src], torch.zeros(n - most, dtype=torch.float64)])
                for g in range(LAYERS * HEADS):
                    held[s][g] = [held[s][g][j] for j in source[s, g if sets > 1 else 0, :most].tolist()]
            else:
                assert int(r.evicted[s]) == 0
            n = int(r.lengths[s])
            assert n == len(held[s][0])
            assert ((r.weight[s].cpu().double() - grown[s]).abs()[:, :n] <= tol[s][:, :n]).all()
            pages = r.pool[r.table[s, :-(-n // PAGE)].long()].cpu()
            for g in range(LAYERS * HEADS):
                for i, (a, b) in enumerate(held[s][g]):
                    assert torch.equal(pages[i // PAGE, g // HEADS, 0, g % HEADS, i % PAGE], a)
                    assert torch.equal(pages[i // PAGE, g // HEADS, 1, g % HEADS, i % PAGE], b)
        if int(r.lengths[2]) > 60:  # (the sequence that is not asked begins anew)
            rac.rac_cache_fork(r.cfg, i32([0, 1, -1]), r.table, r.lengths, r.refs)
            held[2], ages[2] = [[] for _ in range(LAYERS * HEADS)], 0
    assert r.lengths.tolist()[:2] == [BUDGET, BUDGET - 7]
    counts = torch.bincount(r.table[r.table >= 0].long(), minlength=60)
    assert torch.equal(counts.int(), r.refs)


@pytest.mark.parametrize("sets", [1, LAYERS * HEADS])
def test_a_captured_round_replays_the_same(sets):
    eager, captured = Rounds(5, sets), Rounds(5, sets)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.calls()
    ages = [0] * S
    for turn in range(20):
        eager.draw(ages)
        captured.draw(ages)
        eager.calls()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.results(), captured.results()):
            assert torch.equal(a.view(torch.uint8) if a.dtype.is_floating_point else a, b.view(torch.uint8) if b.dtype.is_floating_point else b)
        ages = [a + len(p) for a, p in zip(ages, eager.paths)]
        if max(eager.lengths.tolist()) > 60:
            for x in (eager, captured):
                rac.rac_cache_fork(x.cfg, i32([0, 1, -1]), x.table, x.lengths, x.refs)
