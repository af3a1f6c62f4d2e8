"""How exactly the tree attention holds its softmax weights.

The bound of an output, from the contract: a score is an fp32 sum of D products
(off by at most D 2^-23 of the sum of their magnitudes); exponentials, rescaling
and sums add less than 2^-18 relative; a weight goes to the matrix cores within
`r` of itself, u for one 16-bit number and u^2 for two (u = 2^-8 in bf16, 2^-11 in
fp16), fp16 weights far below the row's largest within 2^-36 of that one; the
output is rounded once (fp16 ones below the normal range to 2^-25)."""
from __future__ import annotations

import math

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


def attend(kind, scores, values, rows, heads, dim, seqs=1):
    """`rows` equal rows and `heads` query heads of one key-value head over keys
    that differ in the first channel only, in each of `seqs` sequences: a key's
    score is its entry of `scores`, every channel of its value its entry of
    `values`.  Returns out [rows][heads][dim] and lse of the last sequence."""
    page, n, act = 64, len(scores), R.ACT[kind]
    width = -(-n // page)
    cfg = rac.CacheConfig(1, 1, dim, page, width, seqs, width, kind)
    both = torch.zeros(2, width * page, dim)
    both[0, :n, 0], both[1, :n] = scores, values[:, None]
    held = both.to(R.STORED[kind])
    assert torch.equal(held.float(), both)  # (every input is exact)
    pool = held.reshape(2, width, page, dim).transpose(0, 1).contiguous().cuda()
    table = torch.arange(width, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    q = torch.zeros(seqs * rows, heads, dim, dtype=act, device="cuda")
    q[..., 0] = 1.0
    tree = lambda scale: rac.TreeConfig(heads, seqs * rows, rows, 0, 0, scale)

    def run(scale):
        ws = torch.empty(rac.rac_tree_attention_workspace(cfg, tree(scale)), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        lse = torch.empty(seqs * rows, heads, device="cuda")
        start = torch.arange(0, seqs * rows + 1, rows, dtype=torch.int32, device="cuda")
        rac.rac_tree_attention(cfg, tree(scale), 0, pool.view(torch.uint8), table,
                               torch.full((seqs,), n, dtype=torch.int32, device="cuda"), q, start, None, None, out, ws,
                               lse=lse)
        torch.cuda.synchronize()
        return out[-rows:].double().cpu(), lse[-rows:].double().cpu()

    return run


def check(kind, scale, scores, values, out, lse, dim, two):
    scale = torch.tensor(scale, dtype=torch.float32).double()
    s, v = scale * scores.double(), values.double()
    w = torch.softmax(s, 0)
    want, size, total = (w @ v).item(), (w @ v.abs()).item(), torch.exp(s - s.max()).sum().item()
    u = R.ROUND[kind]
    ds = dim * 2.0 ** -23 * s.abs().max().item()
    low = 2.0 ** -36 * len(scores) * v.abs().max().item() / total if kind == R.FP16 else 0.0
    bound = u * abs(want) + (1 + u) * (((u * u if two else u) + 2 * ds + 2.0 ** -18) * size + low)
    if kind == R.FP16:
        bound += 2.0 ** -25
    off = (out - want).abs().max().item() / bound
    assert off <= 1, f"{off:.2f} of the bound (want {want:.3e}, got {out.min():.3e} .. {out.max():.3e})"
    wl = torch.logsumexp(s, 0).item()
    assert (lse - wl).abs().max() <= ds + 2.0 ** -18 + 2.0 ** -22 * abs(wl)
    return off


@pytest.mark.parametrize("kind", [R.BF16, R.FP16, R.FP8])
@pytest.mark.parametrize("dim,rows,heads", [
    (16, 1, 1), (64, 1, 8), (64, 16, 1), (80, 1, 5), (128, 2, 8), (128, 1, 1), (144, 1, 1), (192, 3, 4), (256, 1, 16),
    (256, 16, 1)])
@pytest.mark.parametrize("keys,seqs", [(700, 1), (9001, 1), (330, 70)])
def test_few_rows_keep_what_rounding_a_weight_leaves(kind, dim, rows, heads, keys, seqs):
    """Every second key has the largest weight, the others one that lies half way
    between two 16-bit numbers, with values of the other sign that cancel the former."""
    u = R.ROUND[kind] / 2  # between two numbers below 1 there are u, half way is u / 2 off
    w = (math.floor((1 / 1.75) / u) + 0.5) * u
    scores = torch.zeros(keys)
    scores[1::2] = -1.0
    values = torch.ones(keys)
    values[1::2] = -1.75
    out, lse = attend(kind, scores, values, rows, heads, dim, seqs)(-math.log(w))
    off = check(kind, -math.log(w), scores, values, out, lse, dim, two=True)
    say(f"[gpu] weights half way, type {kind}, {rows} x {heads} rows of {dim}, {seqs} x {keys} keys: {off:.2f} of the bound")


@pytest.mark.parametrize("dim,rows,heads", [(64, 1, 1), (64, 8, 4), (64, 40, 1), (64, 70, 4), (128, 1, 8), (128, 24, 2),
                                            (128, 130, 1), (128, 130, 4), (256, 1, 1), (256, 40, 2)])
@pytest.mark.parametrize("below", [8.0, 12.5, 14.25, 17.375])
def test_fp16_weights_far_below_the_largest(dim, rows, heads, below):
    """One key of 32 (an attention sink of value 0) far above the others, whose
    small weights alone make the output."""
    scores = torch.full((16384,), -below)
    scores[::32] = 0.0
    values = torch.full((16384,), 1024.0)
    values[::32] = 0.0
    out, lse = attend(R.FP16, scores, values, rows, heads, dim)(1.0)
    off = check(R.FP16, 1.0, scores, values, out, lse, dim, two=rows * heads <= 16)
    say(f"[gpu] fp16 weights e^-{below}, {rows} x {heads} rows of {dim}: {off:.2f} of the bound")
