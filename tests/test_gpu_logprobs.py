"""Log probabilities of tokens, entropy, alternatives and gradients against their
definitions in binary64."""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")

import paper_2608_04991_amd as rac
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

TYPES = {rac.RAC_TYPE_BF16: torch.bfloat16, rac.RAC_TYPE_FP16: torch.float16, rac.RAC_TYPE_FP32: torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rac.library()


class Call:
    def __init__(self, logits, tokens, scale=0.0, top=0, token_rows=None, entropy=True, stream=None, garbage=0xAB):
        rows, vocab = logits.shape
        kind = {v: k for k, v in TYPES.items()}[logits.dtype]
        self.logits, self.tokens, self.token_rows = logits, tokens, token_rows
        self.cfg = rac.LogprobConfig(rows, vocab, tokens.numel(), top, kind, scale)
        new = lambda *s, dtype=torch.float32: torch.full(s, 77, dtype=dtype, device="cuda")
        self.logprob, self.lse = new(tokens.numel()), new(rows)
        self.entropy = new(rows) if entropy else None
        self.ids, self.tops = (new(rows, top, dtype=torch.int32), new(rows, top)) if top else (None, None)
        self.ws = torch.full((rac.rac_logprobs_workspace(self.cfg),), garbage, dtype=torch.uint8, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.run(stream)
        torch.cuda.synchronize()

    def run(self, stream=None):
        rac.rac_logprobs(self.cfg, self.logits, self.tokens, self.logprob, self.lse, self.ws, token_rows=self.token_rows,
                         entropy=self.entropy, top_ids=self.ids, top_logprobs=self.tops, stream=stream)

    def results(self):
        return [t.clone() for t in (self.logprob, self.lse, self.entropy, self.ids, self.tops) if t is not None]

    def check(self):
        """Tolerances.  With A the largest finite |c x|: an exponent is off by 2^-24 of
        |c x| for the rounded factor, of the reference and of itself, so e by less than
        2^-21 (A + 2); the sums add one rounding a step, vocab / 256 / 4 + 24 of them.
        Call the sum of both E, relative.  lse is off by E and 2^-23 of itself; the
        entropy ln s - t / s, with t a mean of numbers of size H + 8 (the reference
        lies up to 8 powers of two below the largest), by (3 H + 40) E; a log
        probability by lse's and 2^-23 of c x."""
        c = self.cfg.scale or 1.0
        x = self.logits.double() * c
        finite = torch.where(torch.isfinite(x), x, 0.0)
        A = finite.abs().amax(1)
        E = 2.0 ** -21 * (A + 2) + (x.shape[1] / 1024 + 24) * 2.0 ** -24
        lse = torch.logsumexp(x, 1)
        none = lse == -math.inf
        p = torch.exp(x - torch.where(none, 0.0, lse)[:, None])
        H = torch.where(none, 0.0, torch.special.entr(p).sum(1))
        el = E + 2.0 ** -23 * A
        assert torch.equal(self.lse == -math.inf, none)
        assert ((self.lse.double() - lse).abs() <= el)[~none].all()
        if self.entropy is not None:
            assert ((self.entropy.double() - H).abs() <= (3 * H + 40) * E).all() and (self.entropy >= 0).all()
        rows = torch.arange(len(x), device="cuda") if self.token_rows is None else self.token_rows.long()
        if self.tokens.numel():
            t = self.tokens.long()
            there = (t >= 0) & (t < x.shape[1]) & (rows >= 0) & (rows < len(x))
            r = rows.clamp(0, len(x) - 1)
            at = x[r, t.clamp(0, x.shape[1] - 1)]
            want = torch.where(there, torch.where(at == -math.inf, -math.inf, at - lse[r]), 0.0)
            same = self.logprob.double() == want
            assert (same | ((self.logprob.double() - want).abs() <= el[r] + 2.0 ** -22 * A[r])).all()
        n = self.cfg.top
        if n:
            raw = self.logits.float()
            order = torch.argsort(torch.where(raw == 0, 0.0, raw), dim=1, descending=True, stable=True)[:, :n]
            gone = raw.gather(1, order) == -math.inf
            ids = torch.full((len(x), n), -1, dtype=torch.int32, device="cuda")
            ids[:, :order.shape[1]] = torch.where(gone, -1, order).int()
            assert torch.equal(self.ids, ids)
            want = torch.full((len(x), n), -math.inf, dtype=torch.float64, device="cuda")
            want[:, :order.shape[1]] = torch.where(gone, -math.inf, x.gather(1, order) - torch.where(none, 0.0, lse)[:, None])
            same = self.tops.double() == want
            assert (same | ((self.tops.double() - want).abs() <= (el + 2.0 ** -22 * A)[:, None])).all()
        return self


def normal(rows, vocab, dtype, seed, spread=3.0, apart=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (spread * torch.randn(rows, vocab + apart, device="cuda", generator=gen)).to(dtype)
    return x[:, :vocab]


def some_tokens(rows, vocab, seed, odd=True):
    gen = torch.Generator().manual_seed(seed)
    t = torch.randint(0, vocab, (rows,), generator=gen, dtype=torch.int32)
    if odd and rows > 3:
        t[1], t[2], t[3] = -100, vocab, vocab - 1
    return t.cuda()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 2), (3, 7), (5, 8), (4, 9), (2, 63), (7, 1000), (64, 1025), (600, 517),
                                        (1, 50001), (3, 131071), (65, 32003), (513, 8191), (520, 33001), (2, 2400001)])
def test_rows_and_vocabularies(dtype, rows, vocab):
    say(f"[gpu] log probabilities {rows} x {vocab} {dtype}")
    x, t = normal(rows, vocab, dtype, rows + vocab), some_tokens(rows, vocab, rows)
    for top, scale, entropy in ((0, 0.0, True), (1, 0.7, True), (5, 1.3, False), (64, 1.0, True), (0, 1.0, False)):
        Call(x, t, scale, top, entropy=entropy).check()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
def test_rows_apart_at_any_place(dtype):
    for apart in (1, 3, 8, 13):
        whole = normal(9, 4099 + apart, dtype, apart)
        for off in (0, 1, 2, 5):
            if off <= apart:
                x = whole[:, off:off + 4099]
                Call(x, some_tokens(9, 4099, off), 0.0, 7).check()


@pytest.mark.parametrize("rows,vocab,count", [(5, 300, 9), (40, 70001, 100), (600, 1000, 10), (3, 64, 0)])
def test_several_tokens_of_a_row(rows, vocab, count):
    gen = torch.Generator().manual_seed(count)
    of = torch.randint(-1, rows + 1, (count,), generator=gen, dtype=torch.int32).cuda()  # (rows outside score 0)
    Call(normal(rows, vocab, torch.bfloat16, 3), some_tokens(count, vocab, 4), 1.25, 3, token_rows=of).check()
    if count == 0:
        Call(normal(rows, vocab, torch.bfloat16, 3), some_tokens(0, vocab, 4)).check()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
@pytest.mark.parametrize("vocab", [5, 700, 40000])
def test_masked_words(dtype, vocab):
    x = normal(70, vocab, dtype, 1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[torch.rand(70, vocab, device="cuda", generator=gen) < 0.97] = -math.inf
    x[3] = -math.inf             # a row that allows nothing
    x[4] = -math.inf
    x[4, vocab - 1] = 2.0        # and one that allows one word
    lowest = float(torch.finfo(dtype).min)
    x[5, ::2] = lowest           # masks of the lowest value
    x[6] = lowest
    x[7] = -math.inf
    x[7, vocab // 2] = lowest
    c = Call(x, some_tokens(70, vocab, 3), 0.0, 10)
    c.check()
    assert c.entropy[3] == 0 and c.entropy[4] == 0 and c.lse[4] == 2.0 and c.ids[3].tolist() == [-1] * 10
    assert c.ids[4].tolist() == [vocab - 1] + [-1] * 9


def test_ties_go_to_the_lower_word():
    for rows, vocab in ((3, 50000), (600, 5000), (3, 2400000)):
        x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
        x[1, ::3] = -0.0                    # (the same as 0)
        x[2] = normal(1, vocab, torch.bfloat16, 1)[0].round()  # few different values
        c = Call(x, some_tokens(rows, vocab, 1), 0.0, 64).check()
        assert c.ids[0].tolist() == list(range(64))


@pytest.mark.parametrize("top", [1, 5, 64])
@pytest.mark.parametrize("vocab", [64, 500, 697, 1500, 2047, 2048, 2049, 4090])
def test_short_rows_with_alternatives(vocab, top):
    """Rows of a block a thread or less: of random words, of ties with one another, and of few that are allowed."""
    say(f"[gpu] short rows of {vocab}, {top} alternatives")
    for dtype in (torch.bfloat16, torch.float32):
        x = normal(7, vocab, dtype, vocab, apart=3)
        x[1] = 0.0
        x[2] = x[2].round()
        x[3, : vocab - 20] = -math.inf
        x[4] = 1.0
        x[4, ::2] = 2.0
        x[5] = torch.arange(vocab, device="cuda").float().neg().to(dtype)
        Call(x, some_tokens(7, vocab, 2), 0.0, top).check()


def test_many_large_words_in_few_places():
    """More words than the bar of the threads' largest lets be ranked: of different value,
    all at the places of a few threads, and above many that tie."""
    vocab = 70000
    x = torch.full((4, vocab), -5.0, device="cuda")
    block = torch.arange(vocab, device="cuda") // 4
    at = (block % 256 < 20).nonzero().ravel()
    x[0, at] = torch.arange(len(at), device="cuda").float() / 64
    x[1, at] = 3.0
    x[1, at[-40:]] = torch.arange(40, device="cuda").float() + 4
    x[2] = torch.arange(vocab, device="cuda").float() / 4096
    x[3] = -x[2]
    for top in (1, 20, 33, 64):
        for rows in (slice(0, 4), slice(0, 1), slice(1, 2)):
            n = len(x[rows])
            Call(x[rows].repeat(1 if n < 4 else 130, 1), some_tokens(n * (1 if n < 4 else 130), vocab, 5), 0.0, top).check()


def test_a_nan_or_an_infinity_stays_in_its_row():
    for vocab in (100, 40000):
        x = normal(8, vocab, torch.float32, 9)
        t = some_tokens(8, vocab, 9, odd=False)
        want = Call(x, t, 0.0, 4)
        y = x.clone()
        y[2, 17], y[5, 3], y[6, 50] = math.nan, math.inf, math.nan
        got = Call(y, t, 0.0, 4)
        for r in range(8):
            if r in (2, 5, 6):
                assert math.isnan(got.lse[r]) and math.isnan(got.entropy[r]) and math.isnan(got.logprob[r])
                assert torch.isnan(got.tops[r]).all()
            else:
                assert all(torch.equal(a[r], b[r]) for a, b in zip(got.results(), want.results()))
        assert got.ids[5, 0] == 3 and 17 not in got.ids[2].tolist()
        assert torch.equal(got.ids[6], want.ids[6]) or 50 in want.ids[6].tolist()


def test_large_and_small_logits():
    for spread, dtype in ((1e-3, torch.float32), (300.0, torch.bfloat16), (6e4, torch.float16), (1e6, torch.float32)):
        x = normal(6, 9001, dtype, 2, spread).clamp(-float(torch.finfo(dtype).max), float(torch.finfo(dtype).max))
        Call(x, some_tokens(6, 9001, 3), 0.0, 5).check()


def test_offsets_beyond_32_bits():
    rows, vocab = 17000, 131072
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[rows - 1, vocab - 1] = x[16900, 5] = 20.0
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    t[rows - 1] = vocab - 1
    c = Call(x, t, 0.0, 2)
    flat = math.log(vocab)
    peak = 20.0 + math.log1p((vocab - 1) * math.exp(-20.0))
    assert abs(float(c.lse[0]) - flat) < 1e-4 and abs(float(c.lse[rows - 1]) - peak) < 1e-4
    assert abs(float(c.logprob[rows - 1]) - (20.0 - peak)) < 1e-4 and c.ids[rows - 1].tolist() == [vocab - 1, 0]
    assert c.ids[16900].tolist() == [5, 0]
    grad = torch.empty_like(x)
    rac.rac_logprobs_backward(c.cfg, x, t, c.lse, grad, grad_logprob=torch.ones(rows, device="cuda"))
    torch.cuda.synchronize()
    g = float(grad[rows - 1, vocab - 1])
    assert abs(g - (1.0 - math.exp(20.0 - peak))) <= 2.0 ** -8 * abs(g) + 1e-7
    assert float(grad[16900, 5]) < -0.99


def gradients(c, gl, ge, into=None):
    out = torch.full_like(c.logits, 7.0) if into is None else into
    rac.rac_logprobs_backward(c.cfg, c.logits, c.tokens, c.lse, out, grad_logprob=gl, grad_entropy=ge, entropy=c.entropy)
    torch.cuda.synchronize()
    return out


def check_gradients(c, x, got, gl, ge):
    """Of the formula, with the forward pass's lse and entropy.  An exponent is off by
    2^-23 (|c x| + |lse|) and the exponential by 2^-21 relative, products and sums by less
    than 2^-21 of their terms; the result is rounded once, at most eps / 2 of itself or, in
    fp16, half its smallest step."""
    scale = c.cfg.scale or 1.0
    y = x.double() * scale
    lse = c.lse.double()[:, None]
    none = lse == -math.inf
    lp = torch.where(none, -math.inf, y - lse)
    p = torch.exp(lp)
    t = c.tokens.long()
    there = (t >= 0) & (t < x.shape[1]) & ~none[:, 0]
    g = torch.where(there, 0.0 if gl is None else gl.double(), 0.0)[:, None]
    one = torch.zeros_like(y).scatter_(1, t.clamp(0, x.shape[1] - 1)[:, None], 1.0)
    h = torch.zeros_like(g) if ge is None else ge.double()[:, None]
    H = c.entropy.double()[:, None] if c.entropy is not None else torch.zeros_like(g)
    inner = torch.where(p > 0, lp + H, 0.0)
    want = scale * (g * (one - p) - h * p * inner)
    size = scale * (g.abs() * (one + p) + h.abs() * p * (inner.abs() + torch.where(p > 0, lp.abs(), 0.0) + H.abs() + 1))
    big = torch.where(torch.isfinite(y), y.abs(), 0.0) + torch.where(none, 0.0, lse.abs())
    tol = size * (2.0 ** -22 * big + 2.0 ** -19) + torch.finfo(got.dtype).eps / 2 * want.abs() + \
        (2.0 ** -25 if got.dtype == torch.float16 else 1e-37)
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (4, 9), (600, 517), (3, 50001), (65, 8200)])
def test_gradients_of_rows_and_vocabularies(dtype, rows, vocab):
    say(f"[gpu] gradients {rows} x {vocab} {dtype}")
    x = normal(rows, vocab, dtype, rows + vocab)
    x[rows // 2, ::3] = -math.inf
    if rows > 4:
        x[4] = -math.inf
    gen = torch.Generator(device="cuda").manual_seed(1)
    gl, ge = (torch.randn(rows, device="cuda", generator=gen) for _ in range(2))
    for scale in (0.0, 0.6):
        c = Call(x, some_tokens(rows, vocab, rows), scale)
        for a, b in ((gl, None), (None, ge), (gl, ge)):
            check_gradients(c, x, gradients(c, a, b), a, b)
    assert rows <= 4 or not gradients(c, gl, ge)[4].any()


@pytest.mark.parametrize("dtype", list(TYPES.values()), ids=str)
def test_gradients_in_place_and_of_rows_apart(dtype):
    gen = torch.Generator(device="cuda").manual_seed(1)
    gl, ge = (torch.randn(9, device="cuda", generator=gen) for _ in range(2))
    for apart, off, out_off in ((0, 0, 0), (5, 1, 1), (5, 0, 3), (8, 2, 1)):
        whole = normal(9, 3001 + apart, dtype, apart)
        x = whole[:, off:off + 3001]
        c = Call(x, some_tokens(9, 3001, off))
        frame = torch.full((9, 3001 + apart), 7.0, dtype=dtype, device="cuda")
        got = gradients(c, gl, ge, frame[:, out_off:out_off + 3001])
        check_gradients(c, x, got, gl, ge)
        rest = torch.ones(3001 + apart, dtype=torch.bool, device="cuda")
        rest[out_off:out_off + 3001] = False
        assert (frame[:, rest] == 7).all()  # (what lies between the rows is left alone)
        kept = x.clone()
        again = gradients(c, gl, ge, x)
        assert again.data_ptr() == x.data_ptr() and torch.equal(again, got)
        check_gradients(c, kept, again, gl, ge)


def test_gradients_against_differences():
    gen = torch.Generator().manual_seed(4)
    x = (2 * torch.randn(3, 50, generator=gen)).cuda()
    t = torch.tensor([7, 49, 0], dtype=torch.int32, device="cuda")
    gl, ge = torch.tensor([1.0, -0.5, 2.0], device="cuda"), torch.tensor([0.3, 1.0, -0.7], device="cuda")
    c = Call(x, t, 0.8)
    got = gradients(c, gl, ge)

    def loss(y):
        lp = torch.log_softmax(0.8 * y, 1)
        H = -(torch.exp(lp) * lp).sum(1)
        return float((gl.double() * lp[torch.arange(3), t.long()] + ge.double() * H).sum())

    h = 2.0 ** -12
    for r, v in ((0, 7), (0, 3), (1, 49), (1, 0), (2, 0), (2, 20)):
        e = torch.zeros(3, 50, dtype=torch.float64, device="cuda")
        e[r, v] = h
        d = (loss(x.double() + e) - loss(x.double() - e)) / (2 * h)
        # (third derivatives of size at most 6 (|gl| + |ge| (3 + H + |ln p|)) leave h^2; the kernel 2^-19)
        assert abs(d - float(got[r, v])) <= 60 * h * h + 2.0 ** -19 * 10


def test_the_same_call_gives_the_same_bits_whatever_the_scratch_holds():
    for rows, vocab, dtype in ((3, 90001, torch.float32), (70, 33000, torch.bfloat16), (700, 3001, torch.float16)):
        x, t = normal(rows, vocab, dtype, 5), some_tokens(rows, vocab, 5)
        want = Call(x, t, 0.0, 20, garbage=0).results()
        for garbage in (0xFF, 0x55):
            assert all(torch.equal(a, b) for a, b in zip(Call(x, t, 0.0, 20, garbage=garbage).results(), want))
        assert all(torch.equal(a, b) for a, b in zip(Call(x, t, 0.0, 20, stream=torch.cuda.Stream()).results(), want))


def test_replayed_from_graphs_that_share_their_scratch():
    calls = [Call(normal(r, v, torch.bfloat16, r), some_tokens(r, v, r), 0.0, 5) for r, v in ((4, 60000), (30, 40000))]
    ws = max((c.ws for c in calls), key=lambda w: w.numel())
    graphs = []
    for c in calls:
        c.ws = ws
        c.grad, c.gl = torch.zeros_like(c.logits), torch.ones(c.cfg.rows, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
            rac.rac_logprobs_backward(c.cfg, c.logits, c.tokens, c.lse, c.grad, grad_logprob=c.gl, grad_entropy=c.gl,
                                      entropy=c.entropy)
        graphs.append(g)
    for i in range(3):
        for c, g in zip(calls, graphs):
            c.logits.mul_(0.9).add_(0.1)
            g.replay()
        torch.cuda.synchronize()
        for c in calls:
            c.check()
            check_gradients(c, c.logits, c.grad, c.gl, c.gl)
