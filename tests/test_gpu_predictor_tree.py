"""The reference predictor over drafted trees and a paged cache against its
binary64 oracle: every node is an ordinary sequence whose inputs are the
committed ones and its path.  The bar is the one of tests/test_gpu_predictor.py.
The oracle's turned queries are rounded to bf16, as the contract of the step
over trees has it."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from oracle import predictor as P
from paper_2608_04991_amd import workloads as wl
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def bf16_queries(q, keys, values):
    return ATTEND(P.to_bf16(q), keys, values)


ATTEND = P.attend


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Tree:
    """Predictor states of a few sequences, and the inputs that led to them."""

    def __init__(self, cfg, seqs, pages, page=8, seed=0):
        self.cfg, self.rng = cfg, np.random.default_rng(seed)
        self.weights = wl.predictor_weights(cfg.hidden, cfg.model, cfg.ffn, seed)
        self.blob = torch.from_numpy(rac.predictor_pack(cfg, self.weights)).cuda()
        self.cache = rac.CacheConfig(1, cfg.heads, 64, page, pages, seqs, pages // seqs)
        self.pool = torch.full((rac.rac_cache_pool_bytes(self.cache) // 2,), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.table, self.lengths, self.refs = rac.rac_cache_new(self.cache)
        self.inputs = [[] for _ in range(seqs)]  # bf16 patterns of the committed inputs

    def states(self, n):
        return wl.f32_to_bf16_bits(self.rng.standard_normal((n, self.cfg.hidden), dtype=np.float32))

    def oracle(self, inputs):
        """What the predictor makes of the last of a sequence's inputs."""
        c = self.cfg
        p = P.Predictor(self.weights, c.hidden, c.model, c.heads, c.ffn, c.window, 1)
        P.attend = bf16_queries
        try:
            for t, x in enumerate(inputs):
                _, inter = p.step(x[None], [t])
        finally:
            P.attend = ATTEND
        return inter["r"][0], inter["y"][0]

    def step(self, rows, x, draft, mask=None):
        """rows: (sequence, slot, position) of each row, by sequence; x their
        inputs; draft: (k, v, rows of each sequence)."""
        S, c = self.cache.seqs, self.cfg
        count = [sum(s == b for s, _, _ in rows) for b in range(S)]
        tree = rac.TreeConfig(c.heads, len(rows), max(count), max(draft[2]), c.window)
        ws = torch.empty(rac.rac_predictor_tree_workspace(c, self.cache, tree), dtype=torch.uint8, device="cuda")
        out = torch.empty(len(rows), c.hidden, dtype=torch.bfloat16, device="cuda")
        rac.rac_predictor_tree_step(
            c, self.cache, tree, self.blob, self.pool, self.table, self.lengths, i32([0] + list(np.cumsum(count))),
            i32([0] + list(np.cumsum(draft[2]))), i32([r[1] for r in rows]), i32([r[2] for r in rows]),
            torch.from_numpy(x.view(np.int16)).cuda(), draft[0], draft[1], out, ws,
            mask=None if mask is None else torch.tensor(mask, dtype=torch.int64, device="cuda")[:, None])
        torch.cuda.synchronize()
        return P.bf16_to_f64(out.view(torch.int16).cpu().numpy().view(np.uint16))

    def check(self, got, inputs):
        r, y = self.oracle(inputs)
        ry = np.sqrt(np.mean(y * y))
        err = np.abs(got - r)
        self.worst = max(getattr(self, "worst", 0), err.mean() / (2.0 ** -9 * np.abs(r).mean() + 2.0 ** -10 * ry))
        assert np.all(err <= 2.0 ** -8 * np.abs(r) + 2.0 ** -6 * ry), float(np.max(err) / ry)
        assert err.mean() <= 2.0 ** -9 * np.abs(r).mean() + 2.0 ** -10 * ry

    def draft(self, sizes):
        n = sum(sizes)
        new = lambda: torch.full((n, self.cfg.heads, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        return new(), new(), sizes

    def commit(self, draft, path):
        out = i32([0] * self.cache.seqs)
        ws = torch.empty(rac.rac_cache_commit_workspace(self.cache), dtype=torch.uint8, device="cuda")
        most = max(map(len, path))
        rac.rac_cache_commit(self.cache, self.pool, self.table, self.lengths, self.refs, draft[0][None], draft[1][None],
                             i32([0] + list(np.cumsum(draft[2]))), out, ws, path=i32([p + [-1] * (most - len(p)) for p in path]))
        torch.cuda.synchronize()
        assert out.tolist() == [len(p) for p in path]


@pytest.mark.parametrize("window", [5, 300])
def test_levels_of_trees_and_their_accepted_paths(window):
    say(f"[gpu] predictor over trees, window {window}")
    cfg = rac.PredictorConfig(512, 128, 2, 256, window, 64)
    T = Tree(cfg, 3, 36, seed=window)
    # prompts of 0, 7 and 20 inputs, a causal chunk each
    sizes = [0, 7, 20]
    x = T.states(27)
    d = T.draft(sizes)
    rows = [(s, sum(sizes[:s]) + i, i) for s in range(3) for i in range(sizes[s])]
    got = T.step(rows, x, d)
    for (s, _, i), g, xi in zip(rows, got, x):
        T.inputs[s].append(xi)
        T.check(g, T.inputs[s])
    T.commit(d, [list(range(n)) for n in sizes])
    # two rounds of trees: node i hangs from node (i - 1) // 2, level by level
    for nodes in ([7, 3, 6], [1, 7, 4]):
        d = T.draft(nodes)
        first = [sum(nodes[:s]) for s in range(3)]
        given = {}
        for level in range(3):
            rows, mask, paths, x = [], [], [], []
            for s in range(3):
                for i in range(2 ** level - 1, min(2 ** (level + 1) - 1, nodes[s])):
                    path = [i]
                    while path[0]:
                        path.insert(0, (path[0] - 1) // 2)
                    given[s, i] = T.states(1)[0]
                    rows.append((s, first[s] + i, len(T.inputs[s]) + level))
                    mask.append(sum(1 << j for j in path))
                    paths.append(T.inputs[s] + [given[s, j] for j in path])
                    x.append(given[s, i])
            if not rows:
                continue
            got = T.step(rows, np.stack(x), d, mask)
            for g, p in zip(got, paths):
                T.check(g, p)
        accepted = [[0], [0, 2] if nodes[1] > 2 else [0], [0, 1, 3] if nodes[2] > 3 else [0, 1]]
        T.commit(d, accepted)
        for s, p in enumerate(accepted):
            T.inputs[s] += [given[s, i] for i in p]
    # a fork goes on by itself
    rac.rac_cache_fork(T.cache, i32([1, 1, 1]), T.table, T.lengths, T.refs)
    T.inputs = [list(T.inputs[1]) for _ in range(3)]
    for _ in range(2):
        d, x = T.draft([1, 1, 1]), T.states(3)
        got = T.step([(s, s, len(T.inputs[s])) for s in range(3)], x, d)
        for s in range(3):
            T.inputs[s].append(x[s])
            T.check(got[s], T.inputs[s])
        T.commit(d, [[0]] * 3)


def test_glm_shape_batch_of_trees():
    say("[gpu] predictor 4096/512/8/2048 over 24 trees of 10 nodes")
    cfg = rac.PredictorConfig(4096, 512, 8, 2048, 64, 256)
    T = Tree(cfg, 24, 96, page=16, seed=3)
    sizes = [10] * 24
    d, x = T.draft(sizes), T.states(240)
    paths = []
    for i in range(10):
        paths.append((paths[(i - 1) // 3] if i else []) + [i])
    mask = [sum(1 << j for j in paths[i]) for _ in range(24) for i in range(10)]
    got = T.step([(s, 10 * s + i, len(paths[i]) - 1) for s in range(24) for i in range(10)], x, d, mask)
    for s, i in ((0, 0), (3, 4), (11, 9), (23, 7)):
        T.check(got[10 * s + i], [x[10 * s + j] for j in paths[i]])


def test_a_row_without_a_place_stores_nothing():
    cfg = rac.PredictorConfig(512, 128, 2, 256, 16, 8)
    T = Tree(cfg, 2, 8)
    d, x = T.draft([2, 1]), T.states(3)
    T.step([(0, 0, 0), (0, -1, 1), (1, 99, 0)], x, d)
    assert torch.isfinite(d[0][0]).all() and torch.isnan(d[0][1:]).all() and torch.isnan(d[1][1:]).all()
