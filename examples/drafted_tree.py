"""Speculative decoding over a split model's uplink: a tree of drafted tokens a
sequence crosses in a few messages, one per level, each state coded against the
reference that the predictor makes from its parent's reconstruction.

A round, for every sequence at once:
  1. level by level, rac_predictor_tree_step turns the reconstructions of the
     parents into the references of their children, rac_encode codes the
     children's states against them (its reconstruction feeds the next level) and
     the receiver decodes against the references of its own predictor and cache,
     which are the same bits, for it makes the same calls,
  2. the tail verifies the drafts (here: a random path of each tree is accepted),
     rac_cache_commit appends the accepted path's keys and values to the cache,
  3. rac_cache_fork goes on with the best sequence of every group of beams.

    python examples/drafted_tree.py
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2608_04991_amd as rac
from paper_2608_04991_amd import workloads


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return i32(out)


class Side:
    """The predictor's states of `beams` sequences, as the sender and, from the
    same reconstructions, the receiver keep them."""

    def __init__(self, hidden, model, beams, window, page=16, most=512, seed=0):
        heads, ffn = model // 64, 4 * model
        self.cfg = rac.PredictorConfig(hidden, model, heads, ffn, window, 256)
        weights = workloads.predictor_weights(hidden, model, ffn, seed)
        self.blob = torch.from_numpy(rac.predictor_pack(self.cfg, weights)).cuda()
        width = -(-most // page)
        self.cache = rac.CacheConfig(1, heads, 64, page, 2 * beams * width, beams, width)
        self.pool = torch.zeros(rac.rac_cache_pool_bytes(self.cache), dtype=torch.uint8, device="cuda")
        self.table, self.lengths, self.refs = rac.rac_cache_new(self.cache)
        self.commit_ws = torch.empty(rac.rac_cache_commit_workspace(self.cache), dtype=torch.uint8, device="cuda")
        self.committed = torch.empty(beams, dtype=torch.int32, device="cuda")

    def drafts(self, nodes, last):
        """Room for the keys and values of `nodes` rows a sequence; `last` is the first one's input."""
        kv = (self.cache.seqs * nodes, self.cfg.heads, 64)
        self.nodes, self.recon = nodes, {0: last}
        self.k, self.v = (torch.empty(kv, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def predict(self, level, depth, paths, position):
        """References from the reconstructions of nodes `level` of every tree."""
        B, n, N = self.cache.seqs, len(level), self.nodes
        tree = rac.TreeConfig(self.cfg.heads, B * n, n, N, self.cfg.window)
        ws = torch.empty(rac.rac_predictor_tree_workspace(self.cfg, self.cache, tree), dtype=torch.uint8, device="cuda")
        mask = torch.tensor([sum(1 << j for j in paths[i]) for i in level] * B, dtype=torch.int64, device="cuda")[:, None]
        out = torch.empty(B * n, self.cfg.hidden, dtype=torch.bfloat16, device="cuda")
        rac.rac_predictor_tree_step(
            self.cfg, self.cache, tree, self.blob, self.pool, self.table, self.lengths, starts([n] * B), starts([N] * B),
            i32([b * N + i for b in range(B) for i in level]), i32([p + depth for p in position for _ in level]),
            torch.stack([self.recon[i] for i in level], 1).reshape(B * n, -1), self.k, self.v, out, ws, mask=mask)
        return out.reshape(B, n, -1)

    def commit(self, paths):
        most = max(map(len, paths))
        rac.rac_cache_commit(self.cache, self.pool, self.table, self.lengths, self.refs, self.k[None], self.v[None],
                             starts([self.nodes] * self.cache.seqs), self.committed, self.commit_ws,
                             path=i32([p + [-1] * (most - len(p)) for p in paths]))

    def follow(self, parents):
        rac.rac_cache_fork(self.cache, i32(parents), self.table, self.lengths, self.refs)


def main(hidden=4096, model=512, groups=4, beams=2, branch=2, depth=3, rounds=4, bits=4, window=64, seed=0):
    B = groups * beams
    rng = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=rng, device="cuda")
    sides = sender, receiver = [Side(hidden, model, B, window, seed=seed) for _ in range(2)]
    # node 0 is the last accepted token; node i hangs from node (i - 1) // branch
    sizes = [branch ** d for d in range(depth + 1)]
    nodes, paths = sum(sizes), [[0]]
    for i in range(1, nodes):
        paths.append(paths[(i - 1) // branch] + [i])
    levels, at = [], 0
    for n in sizes:
        levels.append(list(range(at, at + n)))
        at += n
    last = normal(B, hidden).bfloat16()  # sent raw: nothing precedes it
    position, sent, raw, err, ref = [0] * B, 0, 0, 0.0, 0.0
    for turn in range(rounds):
        for side in sides:
            side.drafts(nodes, last)
        state = {0: last.float()}
        for d in range(depth):
            parents, children = levels[d], levels[d + 1]
            for i in children:
                state[i] = 0.95 * state[(i - 1) // branch] + 0.3 * normal(B, hidden)
            x = torch.stack([state[i] for i in children], 1).bfloat16()
            of = [(i - 1) // branch - parents[0] for i in children]
            r, same = (side.predict(parents, d, paths, position)[:, of].contiguous() for side in sides)
            cfg = rac.RacConfig(B * len(children), hidden, 128, 128, bits, flags=rac.RAC_FLAG_XHAT_BF16)
            wire = torch.empty(rac.rac_wire_size(cfg), dtype=torch.uint8, device="cuda")
            ours, theirs = torch.empty_like(x), torch.empty_like(x)
            rac.rac_encode(cfg, x, r, None, wire, ours)
            rac.rac_decode(cfg, wire, same, None, theirs)
            if not torch.equal(r, same) or not torch.equal(ours, theirs):
                raise RuntimeError("sender and receiver differ")
            for j, i in enumerate(children):
                sender.recon[i], receiver.recon[i] = ours[:, j].contiguous(), theirs[:, j].contiguous()
            sent, raw = sent + wire.numel(), raw + 2 * x.numel()
            err, ref = err + float((x.float() - ours.float()).square().sum()), ref + float(x.float().square().sum())
        # the verified path of every tree: its last token's key and value come with the next round
        pick = torch.randint(1, nodes, (B,), generator=rng, device="cuda").tolist()
        for side in sides:
            side.commit([paths[i][:-1] for i in pick])
        last = torch.stack([sender.recon[i][b] for b, i in enumerate(pick)])
        position = [p + len(paths[i]) - 1 for p, i in zip(position, pick)]
        # every group goes on with its longest beam
        best = [max(range(g * beams, (g + 1) * beams), key=lambda b: position[b]) for g in range(groups)]
        parents = [best[b // beams] for b in range(B)]
        for side in sides:
            side.follow(parents)
        last, position = last[parents].contiguous(), [position[b] for b in parents]
        print(f"round {turn}: positions {position}, {sent / raw:.3f} of the raw bytes, NMSE {err / ref:.2e}", flush=True)
    torch.cuda.synchronize()
    if any(side.lengths.tolist() != position for side in sides):
        raise RuntimeError("the cache holds other lengths than were accepted")
    return sent / raw, err / ref


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("model", 512), ("groups", 4), ("beams", 2), ("branch", 2), ("depth", 3),
                        ("rounds", 4), ("bits", 4), ("window", 64), ("seed", 0)):
        p.add_argument(f"--{name}", type=int, default=value)
    main(**vars(p.parse_args()))
