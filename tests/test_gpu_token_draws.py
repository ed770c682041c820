"""Draws from the seed in token_verify: the documented Philox counters, and the joint distribution of the
emitted tokens."""
import numpy as np
import pytest
import torch

from oracle import philox as OP

from test_gpu_tokens import BF16, F16, F32, api, gen, make_verify  # noqa: F401

pytestmark = pytest.mark.gpu

STREAM_RACE = 7


def host_draws(seed, B, L, V):
    """Coins [B, L] and race [B, V] by the counters that the header documents."""
    key = OP.key_of(seed)
    b = np.arange(B)[:, None]
    coins = OP.uniform_of(OP.philox4x32_10(b, np.arange(L)[None], OP.STREAM_COIN, 0, *key)[0])
    words = OP.philox4x32_10(b, np.arange((V + 3) // 4)[None], STREAM_RACE, 0, *key)
    race = -np.log(OP.uniform_of(np.stack(words, 2).reshape(B, -1)[:, :V]))
    return (torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda() for x in (coins, race))


@pytest.mark.parametrize("mode", ["block", "sample"])
@pytest.mark.parametrize("B,L,V,dtype,off", [(64, 3, 7, F32, 0), (20, 4, 1001, F32, 1), (9, 5, 4099, BF16, 3), (3, 2, 33000, F16, 5), (1, 4, 131072, BF16, 0),
                                             (2, 6, 50001, F32, 2), (16, 8, 40001, BF16, 1)])
def test_draws_from_the_seed_are_the_documented_ones(api, B, L, V, dtype, off, mode):
    """The call with a seed equals the call given the coins and the race that its counters stand for: rows that start
    anywhere, clusters of one CTA and of many.  (Logarithms differ in their last bits between host and kernel: a race that
    is decided by less than 1e-5 is left out.)"""
    seed = 0x123456789ABCDEF0 + V
    tl, dl, tok, _, _ = make_verify(gen(V + off), B, L, V, dtype)
    a = torch.zeros(B, L + 1, V + off + 2, dtype=dtype, device="cuda")[..., off:V + off]
    d = torch.zeros(B, L, V + off + 2, dtype=dtype, device="cuda")[..., off:V + off]
    a.copy_(tl)
    d.copy_(dl)
    coins, race = host_draws(seed, B, L, V)
    x = api.token_verify(a, d, tok, seed, mode)
    y = api.token_verify(a, d, tok, 0, mode, coins=coins, race=race)
    assert torch.equal(x["accepted_len"], y["accepted_len"])
    differ = (x["next_token"] != y["next_token"]).nonzero()[:, 0].tolist()
    for b in differ:
        j = int(x["accepted_len"][b])
        i, k = int(x["next_token"][b]), int(y["next_token"][b])
        assert mode == "sample" or j == L                # r is known without alpha there
        r = torch.softmax(a[b, j].double(), 0) - (torch.softmax(d[b, j].double(), 0) if j < L else 0)
        s = r / race[b].double()
        assert abs(float(s[i] - s[k])) <= 1e-5 * float(s[k])
    assert len(differ) <= 1


@pytest.mark.parametrize("mode", ["block", "sample"])
def test_the_first_two_emitted_tokens_follow_the_target(api, mode):
    """Rows that do not depend on what was emitted: the first two tokens are distributed as q_0 q_1, where a chain that
    emitted one is completed by a draw from q_1.  Chi-square over the V^2 pairs and over the second token alone, 1e-6 quantiles."""
    from scipy import stats
    g = gen(22)
    B, L, V = 200000, 3, 6
    tl = torch.randn(L + 1, V, generator=g, device="cuda").expand(B, L + 1, V).contiguous()
    dl = tl[:, :L] + 0.8 * torch.randn(L, V, generator=g, device="cuda")
    e = torch.empty(B, L, V, device="cuda").exponential_(generator=g)
    tok = (dl - e.log()).argmax(2).to(torch.int32)
    r = api.token_verify(tl, dl, tok, 79, mode)
    acc = r["accepted_len"].long()
    out = torch.cat([tok.long(), torch.zeros(B, 1, dtype=torch.long, device="cuda")], 1)
    out.scatter_(1, acc[:, None], r["next_token"].long()[:, None])
    fresh = torch.multinomial(torch.softmax(tl[0, 1], -1), B, replacement=True, generator=g)
    second = torch.where(acc == 0, fresh, out[:, 1])
    assert int((acc == 0).sum()) > B // 50 and int((acc == 1).sum()) > B // 50 and int((acc >= 2).sum()) > B // 50
    q = torch.softmax(tl[0].double(), -1).cpu()
    pair = torch.bincount(out[:, 0] * V + second, minlength=V * V).double().cpu()
    want = B * (q[0][:, None] * q[1][None]).flatten()
    assert float(want.min()) > 5
    assert float(((pair - want) ** 2 / want).sum()) < stats.chi2.ppf(1 - 1e-6, V * V - 1)
    two = torch.bincount(second, minlength=V).double().cpu()
    assert float(((two - B * q[1]) ** 2 / (B * q[1])).sum()) < stats.chi2.ppf(1 - 1e-6, V - 1)
