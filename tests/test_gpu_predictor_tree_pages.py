"""The reference predictor over drafted trees with 8-bit pages.  The oracle holds
what is committed in 8 bits and rounds the turned queries to bf16, as the contract
of the step over trees has it.  The bar is the one of tests/test_gpu_predictor.py."""
from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from oracle import predictor as P
from tests.gpu_util import say
from tests.test_gpu_predictor_tree import Tree, bf16_queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


def e4m3(x, scale):
    """What an 8-bit page holds for bf16 values x, as binary64."""
    t = torch.from_numpy(x.astype(np.float32)) / np.float32(scale)
    return t.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).double().numpy() * scale


class Pages(Tree):
    """A tree over 8-bit pages."""

    def __init__(self, cfg, seqs, pages, page=8, seed=0):
        super().__init__(cfg, seqs, pages, page, seed)
        self.cache = rac.CacheConfig(1, cfg.heads, 64, page, pages, seqs, pages // seqs, rac.RAC_CACHE_FP8, 0.0625, 0.03125)
        self.pool = torch.full((rac.rac_cache_pool_bytes(self.cache),), 127, dtype=torch.uint8, device="cuda")  # (NaN)

    def check(self, got, committed, path):
        c = self.cfg
        p = P.Predictor(self.weights, c.hidden, c.model, c.heads, c.ffn, c.window, 1)
        attend, P.attend = P.attend, bf16_queries
        try:
            for t, x in enumerate(committed + path):
                _, inter = p.step(x[None], [t])
                if t < len(committed):
                    line = p.cache[0, t % c.window]
                    line[0], line[1] = e4m3(line[0], self.cache.k_scale), e4m3(line[1], self.cache.v_scale)
        finally:
            P.attend = attend
        r, y = inter["r"][0], inter["y"][0]
        ry, err = np.sqrt(np.mean(y * y)), np.abs(got - r)
        self.worst = max(getattr(self, "worst", 0.0), float(np.max(err / (2.0 ** -8 * np.abs(r) + 2.0 ** -6 * ry))))
        self.mean = max(getattr(self, "mean", 0.0), float(err.mean() / (2.0 ** -9 * np.abs(r).mean() + 2.0 ** -10 * ry)))
        assert self.worst <= 1 and self.mean <= 1, (self.worst, self.mean)


@pytest.mark.parametrize("window", [6, 300])
@pytest.mark.parametrize("hidden,model", [(512, 128), (2048, 512)])
def test_prompts_and_rounds_of_trees(window, hidden, model):
    cfg = rac.PredictorConfig(hidden, model, model // 64, 2 * model, window, 64)
    T = Pages(cfg, 3, 36, seed=window)
    sizes = [5, 0, 19]
    x, d = T.states(24), T.draft(sizes)
    rows = [(s, sum(sizes[:s]) + i, i) for s in range(3) for i in range(sizes[s])]
    given = [[], [], []]
    for (s, _, i), g, xi in zip(rows, T.step(rows, x, d), x):
        given[s].append(xi)
        T.check(g, [], given[s])
    T.commit(d, [list(range(n)) for n in sizes])
    T.inputs = given
    # node i hangs from node (i - 1) // 2, all levels in one step
    paths = []
    for i in range(7):
        paths.append((paths[(i - 1) // 2] if i else []) + [i])
    for accepted in ([0, 2], [0, 1, 4], [0]):
        x, d = T.states(21), T.draft([7, 7, 7])
        rows = [(s, 7 * s + i, len(T.inputs[s]) + len(paths[i]) - 1) for s in range(3) for i in range(7)]
        got = T.step(rows, x, d, [sum(1 << j for j in paths[i]) for _ in range(3) for i in range(7)])
        for r, (s, _, _) in enumerate(rows):
            T.check(got[r], T.inputs[s], [x[7 * s + j] for j in paths[r % 7]])
        T.commit(d, [accepted] * 3)
        for s in range(3):
            T.inputs[s] = T.inputs[s] + [x[7 * s + i] for i in accepted]
    say(f"[gpu] predictor {hidden}/{model} window {window}, 8-bit pages: "
        f"{T.worst:.2f} of an element's bound, {T.mean:.2f} of the mean's")
