"""Plain forms of the paged cache's operators on the CPU: the attention of
drafted trees in binary64, and the bookkeeping as lists of pages."""
from __future__ import annotations

import math

import torch

BF16, FP16, FP8 = 0, 1, 2
ACT = {BF16: torch.bfloat16, FP16: torch.float16, FP8: torch.bfloat16}
STORED = {BF16: torch.bfloat16, FP16: torch.float16, FP8: torch.float8_e4m3fn}
ROUND = {BF16: 2.0 ** -8, FP16: 2.0 ** -11, FP8: 2.0 ** -8}  # of the 16-bit type


def visible(length, n, m, window, mask, there):
    """[m][length + n] booleans: what each of a sequence's m rows sees.  mask:
    [m][>= n] booleans or None; there: [length] booleans, positions with a page."""
    out = torch.zeros(m, length + n, dtype=torch.bool)
    for i in range(m):
        if mask is None:
            drafted = list(range(max(0, min(n, n - m + i + 1))))
        else:
            drafted = [j for j in range(min(n, mask.shape[1])) if mask[i, j]]
        first = 0
        if window:
            drafted = drafted[-window:]
            first = max(0, length - (window - len(drafted)))
        out[i, first:length] = there[first:length]
        out[i, [length + j for j in drafted]] = True
    return out


def attention(q, k, v, see, scale):
    """One sequence: q [m][Hq][D], k, v [keys][H][D], see [m][keys], binary64.
    Returns out, lse, and what the tolerances are made of: sum w |v|, the
    largest scale * sum |q k| a row sees, and the keys it sees."""
    m, Hq, D = q.shape
    H = k.shape[1]
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((m, Hq), -math.inf, dtype=torch.float64)
    reach = torch.zeros(m, Hq, dtype=torch.float64)
    for i in range(m):
        at = see[i].nonzero().ravel()
        if not len(at):
            continue
        for h in range(Hq):
            kk, vv = k[at, h // (Hq // H)], v[at, h // (Hq // H)]
            s = scale * (kk @ q[i, h])
            w = torch.softmax(s, 0)
            lse[i, h] = torch.logsumexp(s, 0)
            out[i, h] = w @ vv
            size[i, h] = w @ vv.abs()
            reach[i, h] = (scale * (kk.abs() @ q[i, h].abs())).max()
    return out, lse, size, reach, see.sum(1)


def tolerances(kind, out, lse, size, reach, keys, v_max, D):
    """Where they come from.  A score is an fp32 sum of D exact products: off by
    at most D 2^-23 of the sum of their magnitudes (`reach`); its exponential,
    the running rescaling and the sums add less than 2^-18 relative.  A weight
    is rounded to 16 bits (`u` of it; fp16 ones below the normal range by at
    most 2^-25 each, with the largest at least 1), and so is the output."""
    u = ROUND[kind]
    ds = D * 2.0 ** -23 * reach
    loose = (u + 2 * ds + 2.0 ** -18)[..., None] * size
    small = (keys * 2.0 ** -25 * v_max)[:, None, None] if kind == FP16 else 0.0
    return u * out.abs() + (1 + u) * (loose + small) + 1e-30, ds + 2.0 ** -18 + 2.0 ** -22 * lse.abs()


class Model:
    """The bookkeeping of a cache, by the words of the contract."""

    def __init__(self, pages, page, seqs, width):
        self.pages, self.page, self.seqs, self.width = pages, page, seqs, width
        self.table = [[-1] * width for _ in range(seqs)]
        self.lengths = [0] * seqs

    def refs(self):
        out = [0] * self.pages
        for row in self.table:
            for p in row:
                if p >= 0:
                    out[p] += 1
        return out

    def fork(self, parents, keep_from=None, keep_to=None):
        table, lengths = [r[:] for r in self.table], self.lengths[:]
        for d, parent in enumerate(parents):
            if not 0 <= parent < self.seqs:
                self.table[d], self.lengths[d] = [-1] * self.width, 0
                continue
            lo = keep_from[d] if keep_from is not None else 0
            hi = keep_to[d] if keep_to is not None else 1 << 40
            self.table[d] = [p if j * self.page < hi and (j + 1) * self.page > lo else -1
                             for j, p in enumerate(table[parent])]
            self.lengths[d] = max(0, min(lengths[parent], hi))

    def commit(self, accepted):
        """accepted: tokens of each sequence.  Returns (committed, copies, writes):
        copies of (from page, to page, tokens), writes of (sequence, index in its
        path, page, place)."""
        refs = self.refs()
        free = [p for p in range(self.pages) if refs[p] == 0]
        demand, plan = 0, []
        for s, n in enumerate(accepted):
            length, need, tail, copies = self.lengths[s], 0, -1, False
            if n and length + n <= self.width * self.page:
                need = -(-(length + n) // self.page) - -(-length // self.page)
                if length % self.page:
                    tail = self.table[s][length // self.page]
                    copies = tail >= 0 and refs[tail] > 1
                    need += copies or tail < 0
            else:
                n = 0
            plan.append((n, demand, need, tail, copies))
            demand += need
        committed, copied, writes = [], [], []
        for s, (n, base, need, tail, copies) in enumerate(plan):
            if base + need > len(free):
                n = 0
            committed.append(n)
            if not n:
                continue
            got = free[base:base + need]
            length = self.lengths[s]
            if copies:
                copied.append((tail, got[0], length % self.page))
            at = -(-length // self.page) - (1 if length % self.page and (copies or tail < 0) else 0)
            self.table[s][at:at + need] = got
            for i in range(n):
                writes.append((s, i, self.table[s][(length + i) // self.page], (length + i) % self.page))
            self.lengths[s] = length + n
        return committed, copied, writes


def accepted_tokens(path, drafted):
    """How many entries of a path name one of `drafted` rows before the first that does not."""
    n = 0
    while n < len(path) and 0 <= path[n] < drafted:
        n += 1
    return n


def stored(x, kind, scale):
    """What the cache holds for 16-bit x, as its own type."""
    if kind != FP8:
        return x
    return (x.float() / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def bits(x):
    """The bit patterns of x (an e4m3 NaN has no sign that means anything)."""
    return x.contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16)
