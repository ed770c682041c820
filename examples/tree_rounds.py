"""Speculative decoding with a drafted tree instead of a chain, on the toy model of token_rounds.

A round:

  1. the drafter grows a tree from the last token: every node of a depth gets as many children as
     `fans` says, drawn from the drafter's distribution after it ("drawn"), or its likeliest tokens ("chosen");
  2. the nodes' keys and values go into the 8-bit cache, turned by the nodes' positions, the queries too
     (api.cache_append_rotary), and every node attends over the tokens before the tree, its ancestors and
     itself (api.tree_attend);
  3. the tree is verified along one path and the next token is drawn (api.tree_verify);
  4. the rows of the path move together in the cache (api.cache_keep); rejected nodes are
     overwritten by the next round;
  5. the drafter is trained towards the emitted tokens (api.token_scores_train).

    python examples/tree_rounds.py [--rounds 100] [--children drawn|chosen]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2606_13426_gb300 import api  # noqa: E402
from token_rounds import Toy  # noqa: E402


def tree_shape(fans):
    """Parents and depths of a tree whose nodes of depth d have fans[d] children each; parents come first."""
    parents, depths, level = [-1], [0], [0]
    for d, fan in enumerate(fans):
        level = [i for p in level for i in range(len(parents), len(parents) + fan) if not parents.append(p)]
        depths += [d + 1] * len(level)
    return parents, depths


def grow(draft, last, parents, depths, children, g):
    """Tokens [B, W] of the tree's nodes and the drafter's logits [B, W, V] after each."""
    B, V = last.shape[0], draft.shape[1]
    tokens = torch.empty(B, len(parents), dtype=torch.int32, device=last.device)
    tokens[:, 0] = last
    for d in range(1, max(depths) + 1):
        level = [i for i, x in enumerate(depths) if x == d]
        z = draft[tokens[:, [parents[i] for i in level]].long()]
        if children == "chosen":                  # the siblings' ranks in their order
            rank = [sum(parents[j] == parents[i] for j in range(i)) for i in level]
            best = z.topk(max(rank) + 1, dim=2).indices
            tokens[:, level] = torch.stack([best[:, k, r] for k, r in enumerate(rank)], 1).to(torch.int32)
        else:
            e = torch.empty(B, len(level), V, device=last.device).exponential_(generator=g)
            tokens[:, level] = (z - e.log()).argmax(2).to(torch.int32)
    return tokens, draft[tokens.long()]


def run(rounds=100, B=64, fans=(3, 2, 1), V=64, Hq=8, H=2, D=64, block=64, children="drawn", lr=4.0, seed=1, device="cuda"):
    """Runs the rounds; returns what was emitted, the cache and the rounds' statistics."""
    toy = Toy(V, Hq, H, D, seed, device)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    par, dep = tree_shape(fans)
    W, L = len(par), len(fans)
    pages_of = (rounds * (L + 1) + W) // block + 2
    cache = api.make_token_cache(B * pages_of, H, block, D, device)
    pages = torch.randperm(B * pages_of, generator=g, device=device).to(torch.int32).view(B, pages_of)
    lengths = torch.zeros(B, dtype=torch.int32, device=device)
    last = torch.randint(0, V, (B,), generator=g, device=device, dtype=torch.int32)
    first = last
    parents = torch.tensor(par, dtype=torch.int32, device=device).expand(B, W).contiguous()
    depths = torch.tensor(dep, dtype=torch.int32, device=device)
    freqs = api.rotary_freqs(D, device=device)
    emitted = [[] for _ in range(B)]
    history = []
    for r in range(rounds):
        tokens, draft_logits = grow(toy.draft, last, par, dep, children, g)
        # the target on the tree
        x, q, k, v = toy.qkv(tokens)
        q = api.cache_append_rotary(cache, k, v, pages, lengths, freqs, q=q, positions=lengths[:, None] + depths)
        attended = api.tree_attend(q, cache, pages, lengths + W, parents)["out"]
        target_logits = toy.logits(x, attended).float()
        res = api.tree_verify(target_logits, draft_logits if children == "drawn" else None, tokens, parents, seed=seed * 1000003 + r)
        accepted, path, nxt = res["accepted_len"], res["path"][:, :L + 1], res["next_token"]
        api.cache_keep(cache, res["path"], pages, lengths)
        lengths = lengths + 1 + accepted          # the root and the accepted nodes stay
        # emitted: the path's tokens behind the root, and the next; -1 behind them
        seen = torch.where(path >= 0, tokens.gather(1, path.clamp(min=0).long()), -1)
        out = torch.cat([seen[:, 1:], torch.full_like(nxt, -1)[:, None]], 1)
        out[torch.arange(B, device=device), accepted.long()] = nxt
        # a step of the drafter towards them
        n_out = int((accepted + 1).sum())
        weight = torch.full((B * (L + 1),), -1.0 / n_out, device=device)
        at = seen.clamp(min=0).long().view(-1)
        grad = api.token_scores_train(toy.draft[at], out.reshape(-1).contiguous(), weight)["d_logits"]
        toy.draft.index_add_(0, at, grad, alpha=-lr * n_out / B)
        for b, row_out in enumerate(out.tolist()):
            emitted[b] += [t for t in row_out if t >= 0]
        history.append(dict(accepted=float(accepted.float().mean())))
        last = nxt
    return dict(emitted=emitted, first=first.tolist(), history=history, lengths=lengths.tolist(), cache=cache, pages=pages, toy=toy)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rounds", type=int, default=100)
    ap.add_argument("--children", choices=("drawn", "chosen"), default="drawn")
    a = ap.parse_args()
    res = run(rounds=a.rounds, children=a.children)
    for r in range(0, a.rounds, 10):
        hs = res["history"][r:r + 10]
        print("rounds from %3d  accepted %.2f" % (r, sum(h["accepted"] for h in hs) / len(hs)))


if __name__ == "__main__":
    main()
