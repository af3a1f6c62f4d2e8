"""Log probabilities of logits whose scaled values leave the range of fp32."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests.test_gpu_logprobs import Call, gradients, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


@pytest.mark.parametrize("vocab,top", [(100, 0), (100, 5), (9001, 64), (40000, 5), (40000, 0), (2400001, 3)])
@pytest.mark.parametrize("named", [False, True])
def test_an_lse_out_of_range_is_not_taken_for_a_number(vocab, top, named):
    """Above the range: NaN in what is formed with it, and in the gradient; below: -infinity
    and zeros, as of a row of masked words.  Other rows keep their bits."""
    x = normal(8, vocab, torch.float32, vocab)
    t = torch.arange(8, dtype=torch.int32, device="cuda")
    rows = t.clone() if named else None
    want = Call(x, t, 4.0, top, token_rows=rows)
    y = x.clone()
    y[2, 7], y[2, 2] = 2e38, 2e38       # lse: 8e38
    y[4] = -2e38                         # lse: -8e38
    y[5, 5] = 8e37                       # 3.2e38, just inside
    got = Call(y, t, 4.0, top, token_rows=rows)
    assert math.isnan(got.lse[2]) and math.isnan(got.logprob[2]) and (not top or torch.isnan(got.tops[2, :2]).all())
    assert abs(float(got.entropy[2]) - math.log(2)) < 1e-5 and (not top or got.ids[2, :2].tolist() == [2, 7][:top])
    assert got.lse[4] == -math.inf and got.logprob[4] == -math.inf and abs(float(got.entropy[4]) - math.log(vocab)) < 1e-4
    assert got.lse[5] == torch.tensor(8e37, device="cuda") * 4 and got.logprob[5] == 0 and got.entropy[5] == 0
    same = [0, 1, 3, 6, 7]
    assert all(torch.equal(a[same], b[same]) for a, b in zip(got.results(), want.results()))
    if not named:
        one = torch.ones(8, device="cuda")
        for gl, ge in ((one, None), (None, one), (one, one)):
            g, h = gradients(got, gl, ge), gradients(want, gl, ge)
            assert torch.isnan(g[2]).all() and not g[4].any() and torch.equal(g[same], h[same])
