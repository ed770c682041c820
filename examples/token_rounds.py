"""Speculative decoding over tokens with the library's operators, on a toy model.

The target is one attention layer with random weights over a cache held in 8 bits; the drafter
sees the last token alone.  A round:

  1. the drafter proposes L tokens;
  2. the target's keys and values of the last token and the drafts go into the cache
     (api.cache_append), and all L + 1 positions attend over it at once (api.cache_attend);
  3. the drafts are verified and the next token is drawn (api.token_verify); the cache keeps the
     accepted tokens: its lengths alone say so, rejected ones are overwritten by the next round;
  4. the emitted tokens are scored under the target, with entropy and alternatives
     (api.token_scores), and the drafter is trained towards them: gradient of their log
     probability under its own logits (api.token_scores_train).

    python examples/token_rounds.py [--rounds 100] [--mode block|sample]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_13426_gb300 import api  # noqa: E402


class Toy:
    """Random weights: embeddings, one attention layer (Hq query heads on H key heads), a drafter."""

    def __init__(self, V, Hq, H, D, seed, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.V, self.Hq, self.H, self.D = V, Hq, H, D
        d = Hq * D

        def normal(*shape, scale):
            return scale * torch.randn(*shape, generator=g, device=device)
        self.embed = normal(V, d, scale=1.0).bfloat16()
        self.wq = normal(d, Hq * D, scale=d ** -0.5).bfloat16()
        self.wkv = normal(d, 2 * H * D, scale=d ** -0.5).bfloat16()
        self.wo = normal(Hq * D, d, scale=d ** -0.5).bfloat16()
        self.head = normal(d, V, scale=2.5 * d ** -0.5).bfloat16()
        self.draft = torch.zeros(V, V, device=device)          # the drafter's logits by last token

    def qkv(self, tokens):
        """Queries, keys and values of tokens [B, n]: slices of two products, read with their strides."""
        B, n = tokens.shape
        x = self.embed[tokens.long()]
        kv = (x @ self.wkv).view(B, n, 2 * self.H, self.D)
        return x, (x @ self.wq).view(B, n, self.Hq, self.D), kv[:, :, :self.H], kv[:, :, self.H:]

    def logits(self, x, attended):
        return (x + attended.flatten(2) @ self.wo) @ self.head


def run(rounds=100, B=64, L=4, V=64, Hq=8, H=2, D=64, block=64, mode="block", lr=4.0, seed=1, device="cuda"):
    """Runs the rounds; returns what was emitted and the rounds' statistics."""
    toy = Toy(V, Hq, H, D, seed, device)
    g = torch.Generator(device=device).manual_seed(seed + 1)
    pages_of = (rounds * (L + 1) + L) // block + 2
    cache = api.make_token_cache(B * pages_of, H, block, D, device)
    pages = torch.randperm(B * pages_of, generator=g, device=device).to(torch.int32).view(B, pages_of)
    lengths = torch.zeros(B, dtype=torch.int32, device=device)
    last = torch.randint(0, V, (B,), generator=g, device=device, dtype=torch.int32)
    row = torch.arange(B, device=device)
    emitted = [[] for _ in range(B)]
    history = []
    for r in range(rounds):
        # the drafter's tokens, drawn from its logits
        drafts, draft_logits, at = [], [], last
        for _ in range(L):
            z = toy.draft[at.long()]
            e = torch.empty(B, V, device=device).exponential_(generator=g)
            at = (z - e.log()).argmax(1).to(torch.int32)
            drafts.append(at)
            draft_logits.append(z)
        drafts, draft_logits = torch.stack(drafts, 1), torch.stack(draft_logits, 1)
        # the target on the window
        window = torch.cat([last[:, None], drafts], 1)
        x, q, k, v = toy.qkv(window)
        api.cache_append(cache, k, v, pages, lengths)
        attended = api.cache_attend(q, cache, pages, lengths + (L + 1))["out"]
        target_logits = toy.logits(x, attended).float()
        res = api.token_verify(target_logits, draft_logits, drafts, seed=seed * 1000003 + r, mode=mode)
        accepted, nxt = res["accepted_len"], res["next_token"]
        lengths = lengths + 1 + accepted                      # the last token and the accepted drafts stay
        # emitted tokens of the window: the accepted drafts and the next token; -1 behind them
        out = torch.cat([drafts, torch.full_like(drafts[:, :1], -1)], 1)
        step = torch.arange(L + 1, device=device)
        out = torch.where(step < accepted[:, None], out, -1)
        out[row, accepted.long()] = nxt
        scores = api.token_scores(target_logits.view(-1, V), out.reshape(-1).contiguous(), top_k=4)
        # a step of the drafter towards them
        n_out = int((accepted + 1).sum())
        seen = torch.cat([last[:, None], out[:, :-1]], 1)      # the token before each
        weight = torch.full((B * (L + 1),), -1.0 / n_out, device=device)
        z = toy.draft[seen.clamp(min=0).long()].view(-1, V)
        grad = api.token_scores_train(z, out.reshape(-1).contiguous(), weight)["d_logits"]
        toy.draft.index_add_(0, seen.clamp(min=0).long().view(-1), grad, alpha=-lr * n_out / B)
        for b, row_out in enumerate(out.tolist()):
            emitted[b] += [t for t in row_out if t >= 0]
        live = out.view(-1) >= 0
        history.append(dict(accepted=float(accepted.float().mean()), logprob=float(scores["logprob"][live].mean()),
                            entropy=float(scores["entropy"][live].mean()), alternatives=scores["top_ids"][0].tolist()))
        last = nxt
    return dict(emitted=emitted, history=history, lengths=lengths.tolist(), cache=cache)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rounds", type=int, default=100)
    ap.add_argument("--mode", choices=("block", "sample"), default="block")
    a = ap.parse_args()
    res = run(rounds=a.rounds, mode=a.mode)
    for r in range(0, a.rounds, 10):
        hs = res["history"][r:r + 10]
        mean = {k: sum(h[k] for h in hs) / len(hs) for k in ("accepted", "logprob", "entropy")}
        print("rounds from %3d  accepted %.2f  log probability %.3f  entropy %.3f  alternatives of the last %s" % (
            r, mean["accepted"], mean["logprob"], mean["entropy"], hs[-1]["alternatives"]))


if __name__ == "__main__":
    main()
