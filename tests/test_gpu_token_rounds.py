"""The token operators together, as examples/token_rounds.py runs them."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import __graft_entry__ as g
    g.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import token_rounds
    return token_rounds


@pytest.mark.parametrize("mode", ["block", "sample"])
def test_rounds_keep_their_books(example, mode):
    kw = dict(rounds=12, B=6, L=3, V=256, mode=mode)
    res = example.run(**kw)
    # every emitted token but the newest is in the cache, and the first token is there besides
    assert [len(e) for e in res["emitted"]] == res["lengths"]
    assert all(0 <= t < 256 for e in res["emitted"] for t in e)
    assert all(len(h["alternatives"]) == 4 and len(set(h["alternatives"])) == 4 for h in res["history"])
    again = example.run(**kw)
    assert again["emitted"] == res["emitted"] and again["history"] == res["history"]


def test_cached_tokens_are_the_emitted_ones(example):
    """The cache after the rounds holds the same keys as one prompt of the accepted tokens would, to the
    8 bits' rounding: scales only grow with rejected tokens (a factor of two in the step at most here)."""
    from paper_2606_13426_gb300 import api
    V, H, D, block = 128, 2, 64, 64
    res = example.run(rounds=10, B=3, L=3, V=V, Hq=4, H=H, D=D, block=block, seed=5)
    toy = example.Toy(V, 4, H, D, 5)
    g = torch.Generator(device="cuda").manual_seed(6)
    pages_of = (10 * 4 + 3) // block + 2
    pages = torch.randperm(3 * pages_of, generator=g, device="cuda").to(torch.int32).view(3, pages_of)
    first = torch.randint(0, V, (3,), generator=g, device="cuda", dtype=torch.int32)
    c = res["cache"]
    for b in range(3):
        n = res["lengths"][b]
        tokens = torch.tensor([int(first[b])] + res["emitted"][b][:-1], device="cuda")[None]
        assert tokens.shape[1] == n
        k, v = toy.qkv(tokens)[2:]
        fresh = api.make_token_cache(pages_of, H, block, D)
        table = torch.arange(pages_of, device="cuda", dtype=torch.int32)[None]
        api.cache_append(fresh, k, v, table, torch.zeros(1, dtype=torch.int32, device="cuda"))
        for j in range(-(-n // block)):
            rows = min(block, n - j * block)
            page = int(pages[b, j])
            for name in ("k", "v"):
                x = c[name][page].float() * c[name + "_scale"][page][:, None, None]
                y = fresh[name][j].float() * fresh[name + "_scale"][j][:, None, None]
                x, y = (x[:, :rows], y[:, :rows]) if name == "k" else (x[:, :, :rows], y[:, :, :rows])
                top = y.abs().amax()
                # half a unit of each (2^-4 relative), restated once more, and 2^-10 of the largest below it
                assert ((x - y).abs() <= 3 * 2.0 ** -4 * y.abs() + 2.0 ** -9 * top).all()


def test_training_the_drafter_raises_acceptance(example):
    res = example.run(rounds=60, B=32, L=4, V=128, seed=3)
    early = sum(h["accepted"] for h in res["history"][:10])
    late = sum(h["accepted"] for h in res["history"][-10:])
    assert late > early
