"""Plain forms, on the CPU, of the weight that cached tokens receive (binary64) and
of eviction by it (lists of pages and places, by the words of the contract)."""
from __future__ import annotations

import math

import torch


def weights(q, k, see, lse, scale):
    """One sequence: q [m][Hq][D], k [keys][H][D], see [m][keys], lse [m][Hq], binary64.
    Returns [H][keys], and what the tolerance is made of: the sum of p times the error
    that a score of its size may bring, and how many terms a sum has."""
    m, Hq, D = q.shape
    keys, H, _ = k.shape
    group = Hq // H
    out, slack = torch.zeros(H, keys, dtype=torch.float64), torch.zeros(H, keys, dtype=torch.float64)
    for i in range(m):
        at = see[i].nonzero().ravel()
        for h in range(Hq):
            if not len(at) or lse[i, h] == -math.inf:
                continue
            kk = k[at, h // group]
            p = torch.exp(scale * (kk @ q[i, h]) - lse[i, h])
            reach = scale * (kk.abs() @ q[i, h].abs())
            out[h // group, at] += p
            slack[h // group, at] += p * (D * 2.0 ** -23 * reach + 2.0 ** -21 * (lse[i, h].abs() + 2))
    return out, slack, m * group


def tolerance(want, slack, terms, before):
    """A score is an fp32 sum of D exact products, off by at most D 2^-23 of the sum of
    their magnitudes; its exponent takes 2^-22 (|score| + |lse|), with |score| <= |lse| + a
    few where it counts, and the exponential 2^-22.  A sum of n terms is off by n 2^-24 of
    itself, and so is what it is added to, once."""
    return 1.01 * slack + want * (terms + 8) * 2.0 ** -24 + (before + want) * 2.0 ** -23 + 1e-30


class Bounded:
    """A cache's bookkeeping: table, lengths and counts as lists, evicted as the contract
    says.  `moves` of an eviction: (sequence, set, new position, new page, old page, old
    position) of every place that is written."""

    def __init__(self, pages, page, table, lengths, refs):
        self.pages, self.page = pages, page
        self.table, self.lengths, self.refs = [list(r) for r in table], list(lengths), list(refs)

    def evict(self, weight, keep, first, recent, source=None):
        """weight: [seqs][sets][positions] (changed), keep: list."""
        P = self.page
        free = [p for p in range(self.pages) if self.refs[p] == 0]
        was = list(self.refs)
        taken, evicted, moves = 0, [], []
        plans = []
        for s, row in enumerate(self.table):
            L = max(0, min(self.lengths[s], len(row) * P))
            there = [j for j in range(-(-L // P)) if 0 <= row[j] < self.pages]
            places = [p for j in there for p in range(j * P, min((j + 1) * P, L))]
            m = len(places)
            if keep[s] < 0 or m <= keep[s]:
                plans.append(None)
                continue
            n = keep[s]
            r = min(recent, n)
            f = min(first, n - r)
            border, sets = n - r, []
            for w in weight[s]:
                value = [float(w[p]) for p in places]
                value = [-math.inf if math.isnan(v) else v for v in value]
                nan = [math.isnan(float(w[p])) for p in places]
                middle = sorted(range(f, m - r), key=lambda i: (nan[i], -value[i], i))[:n - f - r]
                stays = set(range(f)) | set(middle)
                holes = [i for i in range(border) if i not in stays]
                fills = sorted(i for i in stays if i >= border)
                assert len(holes) == len(fills)
                src = list(range(border)) + list(range(m - r, m))
                for h, g in zip(holes, fills):
                    src[h] = g
                sets.append(src)
            old = [row[j] for j in there]
            changed = [was[old[d]] > 1 and any(src[i] != i for src in sets for i in range(d * P, min((d + 1) * P, n)))
                       for d in range(-(-n // P))]
            plans.append((n, m, L, places, sets, old, changed))
        for s, plan in enumerate(plans):
            if plan is None:
                evicted.append(0)
                continue
            n, m, L, places, sets, old, changed = plan
            if sum(changed) > len(free) - taken:
                evicted.append(-1)
                continue
            evicted.append(m - n)
            new = []
            for d, c in enumerate(changed):
                if c:
                    new.append(free[taken])
                    taken += 1
                    self.refs[new[-1]] = 1
                    self.refs[old[d]] -= 1
                else:
                    new.append(old[d])
            for p in old[len(new):]:
                self.refs[p] -= 1
            for g, src in enumerate(sets):
                w = weight[s][g].clone()
                weight[s][g][:L] = 0
                for i, place in enumerate(src):
                    weight[s][g][i] = w[places[place]]
                    if source is not None:
                        source[s][g][i] = places[place]
                    if place != i or changed[i // P]:
                        moves.append((s, g, i, new[i // P], old[place // P], place))
            self.table[s][:] = new + [-1] * (len(self.table[s]) - len(new)) if L else self.table[s]
            self.lengths[s] = n
        return evicted, moves
