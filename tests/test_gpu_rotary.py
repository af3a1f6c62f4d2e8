"""Rotary positions against the definition in binary64."""
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


def definition(x, pos, freq, cfg):
    """The turned rows in binary64; a row with a negative position is itself."""
    half = cfg.rotary_dim // 2
    x, out = x.double(), x.double().clone()
    turns = pos.double()[:, None] * freq
    angle = 2.0 * math.pi * (turns - torch.round(turns))
    c, s = cfg.amplitude * torch.cos(angle)[:, None], cfg.amplitude * torch.sin(angle)[:, None]
    s = -s if cfg.transpose else s
    if cfg.layout == rac.RAC_ROTARY_HALF:
        a, b = slice(0, half), slice(half, 2 * half)
    else:
        a, b = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    return torch.where((pos >= 0)[:, None, None], out, x)


def tolerance(x, want, cfg):
    """The angle's fraction is rounded to fp32 (2^-25 turns, 2^-22.3 radians), sine
    and cosine to within 4 units of 2^-24, times the amplitude and twice each product
    and sum by 2^-24: less than 2^-20 of amplitude (|x| + |y|), and |x| + |y| is less
    than twice the largest of the head.  The result is rounded once, at most eps / 2 of
    itself, or half the smallest step (2^-25 for fp16)."""
    t = TYPES[cfg.type]
    return abs(cfg.amplitude) * 2.0 ** -19 * x.double().abs().amax(-1, keepdim=True) + torch.finfo(t).eps / 2 * want.abs() + 2.0 ** -25


def make(cfg, seed, spread=1.0, apart=0):
    gen = torch.Generator().manual_seed(seed)
    t = TYPES[cfg.type]
    new = lambda heads: (spread * torch.randn(cfg.rows, heads + apart, cfg.head_dim, generator=gen)).to(t).cuda()[:, :heads]
    return new(cfg.q_heads), new(cfg.k_heads) if cfg.k_heads else None


def check(cfg, pos, freq, seed=0, apart=0):
    q, k = make(cfg, seed, apart=apart)
    pos, freq = torch.tensor(pos, dtype=torch.int32, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda")
    fill = lambda x: None if x is None else torch.full_like(x, 7.0)
    qo, ko = fill(q), fill(k)
    rac.rac_rotary(cfg, pos, freq, q, k, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    for x, y in ((q, qo), (k, ko)):
        if x is None:
            continue
        want = definition(x, pos, freq, cfg)
        gone = (pos < 0)[:, None, None]
        assert ((y.double() - want).abs() <= tolerance(x, want, cfg))[~gone.expand_as(x)].all()
        assert (y[pos < 0] == 7).all()  # (rows of padding are not written)
        if cfg.rotary_dim < cfg.head_dim:
            assert torch.equal(y[..., cfg.rotary_dim:][pos >= 0], x[..., cfg.rotary_dim:][pos >= 0])
    # in place
    qi, ki = q.clone(), None if k is None else k.clone()
    rac.rac_rotary(cfg, pos, freq, qi, ki)
    torch.cuda.synchronize()
    for x, y, z in ((q, qo, qi), (k, ko, ki)):
        if x is not None:
            assert torch.equal(z[pos >= 0], y[pos >= 0]) and torch.equal(z[pos < 0], x[pos < 0])


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("layout", [rac.RAC_ROTARY_INTERLEAVED, rac.RAC_ROTARY_HALF])
@pytest.mark.parametrize("rows,q_heads,k_heads,dim,turned", [
    (1, 1, 0, 16, 16), (1, 1, 1, 16, 16), (9, 1, 0, 16, 16), (5, 3, 1, 64, 64), (17, 8, 8, 64, 32), (33, 7, 1, 80, 80),
    (3, 28, 4, 128, 64), (257, 2, 2, 96, 48), (2, 40, 8, 256, 256), (70, 1, 1, 112, 16), (4, 300, 2, 128, 128)])
def test_shapes_layouts_and_types(type, layout, rows, q_heads, k_heads, dim, turned):
    say(f"[gpu] rotary {rows} rows, heads {q_heads}+{k_heads} x {dim}, {turned} turned, layout {layout}, type {type}")
    for transpose in (False, True):
        cfg = rac.RotaryConfig(rows, q_heads, k_heads, dim, turned, type, layout, transpose, 1.0)
        pos = [(37 * i) % 1009 if i % 5 != 3 else -1 - i for i in range(rows)]
        check(cfg, pos, rac.rac_rotary_frequencies(turned, 10000.0), seed=rows)


@pytest.mark.parametrize("amplitude", [1.0, 1.1386, 0.0, -2.5])
def test_far_positions_and_amplitudes(amplitude):
    pos = [0, 1, 65535, 1 << 20, (1 << 24) + 1, (1 << 30) - 1, (1 << 31) - 1]
    for layout in (0, 1):
        cfg = rac.RotaryConfig(len(pos), 4, 2, 128, 128, rac.RAC_TYPE_FP32, layout, False, amplitude)
        check(cfg, pos, rac.rac_rotary_frequencies(128, 1e6, 8.0, 8192, 1.0, 32.0))


def test_rows_apart():
    cfg = rac.RotaryConfig(23, 5, 2, 64, 48, rac.RAC_TYPE_BF16, rac.RAC_ROTARY_HALF)
    check(cfg, list(range(23)), rac.rac_rotary_frequencies(48, 500.0), apart=3)


def test_the_gradient_is_the_transpose():
    """(R x) . y = x . (R' y), and R' R is amplitude^2."""
    gen = torch.Generator().manual_seed(3)
    for layout in (0, 1):
        new = lambda: torch.randn(11, 4, 96, generator=gen).cuda()
        x, y = new(), new()
        pos = torch.arange(100, 111, dtype=torch.int32, device="cuda")
        freq = torch.tensor(rac.rac_rotary_frequencies(64, 10000.0), dtype=torch.float64, device="cuda")
        there = rac.RotaryConfig(11, 4, 0, 96, 64, rac.RAC_TYPE_FP32, layout, False, 1.5)
        back = rac.RotaryConfig(11, 4, 0, 96, 64, rac.RAC_TYPE_FP32, layout, True, 1.5)
        rx, ty, trx = torch.empty_like(x), torch.empty_like(y), torch.empty_like(x)
        rac.rac_rotary(there, pos, freq, x, q_out=rx)
        rac.rac_rotary(back, pos, freq, y, q_out=ty)
        rac.rac_rotary(back, pos, freq, rx, q_out=trx)
        torch.cuda.synchronize()
        a, b = (rx.double() * y).sum(-1), (x.double() * ty).sum(-1)
        size = 1.5 * (x.abs().amax(-1) * y.abs().sum(-1)).double() * 2
        assert ((a - b).abs() <= 2.0 ** -19 * size).all()
        assert (trx[..., :64].double() - 2.25 * x[..., :64].double()).abs().max() <= 2.0 ** -17 * float(x.abs().max())


def test_the_gradient_against_differences():
    """d (R x) . y / d x by central differences of the binary64 definition."""
    cfg = rac.RotaryConfig(3, 2, 0, 32, 16, rac.RAC_TYPE_FP32, rac.RAC_ROTARY_HALF, False, 1.25)
    back = rac.RotaryConfig(3, 2, 0, 32, 16, rac.RAC_TYPE_FP32, rac.RAC_ROTARY_HALF, True, 1.25)
    x, _ = make(cfg, 1)
    y, _ = make(cfg, 2)
    pos = torch.tensor([5, 900, 77], dtype=torch.int32, device="cuda")
    freq = torch.tensor(rac.rac_rotary_frequencies(16, 100.0), dtype=torch.float64, device="cuda")
    g = torch.empty_like(y)
    rac.rac_rotary(back, pos, freq, y, q_out=g)
    h = 2.0 ** -10
    for r, head, c in ((0, 0, 0), (0, 1, 7), (1, 0, 8), (1, 1, 15), (2, 0, 3), (2, 1, 20)):
        e = torch.zeros_like(x, dtype=torch.float64)
        e[r, head, c] = h
        f = [float((definition(x.double() + d, pos, freq, cfg) * y.double()).sum()) for d in (e, -e)]
        # (the definition is linear: the difference is off by binary64 roundings of the sums, 2^-40 over 2 h)
        assert abs((f[0] - f[1]) / (2 * h) - float(g[r, head, c])) <= 2.0 ** -19 * 1.25 * float(y[r, head].abs().max()) + 2.0 ** -30


def test_non_finite_channels_stay_in_their_pair():
    for layout in (0, 1):
        cfg = rac.RotaryConfig(2, 2, 0, 64, 32, rac.RAC_TYPE_BF16, layout)
        q, _ = make(cfg, 5)
        q[0, 1, 3], q[1, 0, 40] = math.nan, math.inf
        pos = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
        freq = torch.tensor(rac.rac_rotary_frequencies(32, 10000.0), dtype=torch.float64, device="cuda")
        out = torch.empty_like(q)
        rac.rac_rotary(cfg, pos, freq, q, q_out=out)
        bad = (~torch.isfinite(out)).nonzero().tolist()
        pair = [2, 3] if layout == 0 else [3, 19]
        assert bad == [[0, 1, pair[0]], [0, 1, pair[1]], [1, 0, 40]]


def test_more_rows_than_workgroups_of_a_launch():
    """1.1 million rows of one head of 16 channels, eight a workgroup or one."""
    for heads, rows in ((1, 9_000_001), (32, 1_050_001)):
        cfg = rac.RotaryConfig(rows, heads, 0, 16, 16, rac.RAC_TYPE_BF16)
        q = torch.ones(rows, heads, 16, dtype=torch.bfloat16, device="cuda")
        pos = torch.arange(rows, dtype=torch.int32, device="cuda")
        freq = torch.tensor(rac.rac_rotary_frequencies(16, 10000.0), dtype=torch.float64, device="cuda")
        rac.rac_rotary(cfg, pos, freq, q)
        torch.cuda.synchronize()
        for r in (0, 1, rows // 2, rows - 2, rows - 1):
            want = definition(torch.ones(1, heads, 16, device="cuda"), pos[r:r + 1], freq, cfg)
            assert ((q[r:r + 1].double() - want).abs() <= 2.0 ** -18 + 2.0 ** -8 * want.abs()).all()


def test_replayed_from_a_graph_and_on_another_stream():
    cfg = rac.RotaryConfig(40, 6, 2, 64, 64, rac.RAC_TYPE_BF16, rac.RAC_ROTARY_HALF)
    q, k = make(cfg, 9)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    freq = torch.tensor(rac.rac_rotary_frequencies(64, 10000.0), dtype=torch.float64, device="cuda")
    want = [torch.empty_like(q), torch.empty_like(k)]
    rac.rac_rotary(cfg, pos, freq, q, k, q_out=want[0], k_out=want[1])
    got = [torch.zeros_like(q), torch.zeros_like(k)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rac.rac_rotary(cfg, pos, freq, q, k, q_out=got[0], k_out=got[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rac.rac_rotary(cfg, pos, freq, q, k, q_out=got[0], k_out=got[1])
    for i in range(3):
        pos += 1
        graph.replay()
        rac.rac_rotary(cfg, pos, freq, q, k, q_out=want[0], k_out=want[1])
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
