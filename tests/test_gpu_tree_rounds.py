"""The tree operators together, as examples/tree_rounds.py runs them."""
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
    import tree_rounds
    return tree_rounds


@pytest.mark.parametrize("children", ["drawn", "chosen"])
@pytest.mark.parametrize("fans", [(2, 2, 1), (4, 3, 2)])
def test_rounds_keep_their_books(example, children, fans):
    kw = dict(rounds=12, B=6, fans=fans, V=256, children=children)
    res = example.run(**kw)
    # every emitted token but the newest is in the cache, and the first token is there besides
    assert [len(e) for e in res["emitted"]] == res["lengths"]
    assert all(0 <= t < 256 for e in res["emitted"] for t in e)
    assert all(0 <= h["accepted"] <= len(fans) for h in res["history"])
    again = example.run(**kw)
    assert again["emitted"] == res["emitted"] and again["history"] == res["history"]


@pytest.mark.parametrize("block,Hq,D", [(64, 4, 64), (16, 8, 128)])
def test_cached_rows_are_those_of_the_emitted_tokens(example, block, Hq, D):
    """The rounds' cache holds what one prompt of the emitted tokens gives, turned by their positions in it.

    Each side's codes are off by half a step when first rounded, 2^-4 relative: 2.2 2^-4 of the rounded one.  Where the scale
    grows, by powers of two, what underflows is off by 2^-10 of the scale: the doublings' sum is twice the last one's, the
    move's and the prompt's are one each.  The products of other shapes may round to the bf16 beside, 2^-7 of an element, in a
    pair's two elements: 2^-6 of the page's largest."""
    from paper_2606_13426_gb300 import api
    V, H, B = 128, 2, 3
    res = example.run(rounds=14, B=B, fans=(3, 2, 2), V=V, Hq=Hq, H=H, D=D, block=block, seed=5)
    toy, c, pages = res["toy"], res["cache"], res["pages"]
    freqs = api.rotary_freqs(D)
    for b in range(B):
        n = res["lengths"][b]
        tokens = torch.tensor([res["first"][b]] + res["emitted"][b][:-1], device="cuda")[None]
        assert tokens.shape[1] == n
        k, v = toy.qkv(tokens)[2:]
        fresh = api.make_token_cache(pages.shape[1], H, block, D)
        table = torch.arange(pages.shape[1], device="cuda", dtype=torch.int32)[None]
        api.cache_append_rotary(fresh, k, v, table, torch.zeros(1, dtype=torch.int32, device="cuda"), freqs)
        for j in range(-(-n // block)):
            rows = min(block, n - j * block)
            page = int(pages[b, j])
            for name in ("k", "v"):
                x = c[name][page].float() * c[name + "_scale"][page][:, None, None]
                y = fresh[name][j].float() * fresh[name + "_scale"][j][:, None, None]
                x, y = (x[:, :rows], y[:, :rows]) if name == "k" else (x[:, :, :rows], y[:, :, :rows])
                low = 4 * 2.0 ** -10 * c[name + "_scale"][page][:, None, None] + 2.0 ** -6 * y.abs().amax()
                assert ((x - y).abs() <= 2.2 * 2.0 ** -4 * y.abs() + low).all()


def test_a_captured_round_is_the_eager_one(example):
    """Append, attention, verification and keeping in one graph, replayed on changed inputs."""
    from paper_2606_13426_gb300 import api
    g = torch.Generator(device="cuda").manual_seed(2)
    par, dep = example.tree_shape((3, 3, 2))
    B, W, V, H, G, D, block = 4, len(par), 512, 2, 4, 128, 64
    parents = torch.tensor(par, dtype=torch.int32, device="cuda").expand(B, W).contiguous()
    depths = torch.tensor(dep, dtype=torch.int32, device="cuda")
    pages = torch.randperm(B * 6, generator=g, device="cuda").to(torch.int32).view(B, 6)
    freqs = api.rotary_freqs(D)

    def inputs():
        return dict(k=torch.randn(B, W, H, D, generator=g, device="cuda").bfloat16(),
                    v=torch.randn(B, W, H, D, generator=g, device="cuda").bfloat16(),
                    q=torch.randn(B, W, H * G, D, generator=g, device="cuda").bfloat16(),
                    target=torch.randn(B, W, V, generator=g, device="cuda").bfloat16(),
                    draft=torch.randn(B, W, V, generator=g, device="cuda").bfloat16(),
                    tokens=torch.randint(0, V, (B, W), generator=g, device="cuda", dtype=torch.int32),
                    coins=torch.rand(B, W, generator=g, device="cuda") * .3,
                    lengths=torch.randint(0, 250, (B,), generator=g, device="cuda", dtype=torch.int32))

    def round_of(x, cache):
        q = api.cache_append_rotary(cache, x["k"], x["v"], pages, x["lengths"], freqs, q=x["q"], positions=x["lengths"][:, None] + depths)
        a = api.tree_attend(q, cache, pages, x["lengths"] + W, parents)
        r = api.tree_verify(x["target"], x["draft"], x["tokens"], parents, seed=7, coins=x["coins"])
        api.cache_keep(cache, r["path"], pages, x["lengths"])
        return dict(q=q, **a, **r)

    static = inputs()
    cache = api.make_token_cache(B * 6, H, block, D)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        round_of(static, cache)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = round_of(static, cache)
    for _ in range(3):
        x = inputs()
        for key in x:
            static[key].copy_(x[key])
        for key, t in cache.items():
            t.view(torch.uint8).zero_() if t.dtype != torch.float32 else t.fill_(1)
        graph.replay()
        other = api.make_token_cache(B * 6, H, block, D)
        want = round_of(x, other)
        for key in want:
            assert torch.equal(got[key].nan_to_num(), want[key].nan_to_num()), key
        assert all(torch.equal(cache[key].view(torch.uint8), other[key].view(torch.uint8)) for key in cache)
        assert int(want["accepted_len"].max()) > 0
