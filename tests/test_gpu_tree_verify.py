"""The verification of drafted trees against its definition in 64 bits: recursive rejection, one child after the
other, with the remainder of the target normalised each time.

Probabilities in fp32 are within 1e-6 of themselves, so that a threshold (q / p - beta) / M is within 4e-6 (q / p + beta) / M:
a decision is compared where its coin is not that near, and at least 0.02 of the target is left; log ratios to
3e-5 (1 + |value|), as those of token_verify.
"""
import math

import pytest
import torch

from test_gpu_tokens import BF16, F16, F32, INF, NAN, api, gen, make_verify, near  # noqa: F401
from test_gpu_token_draws import host_draws
from test_gpu_tree_attend import tree_of

pytestmark = pytest.mark.gpu


def softmax64(x, T):
    """Probabilities in 64 bits; zeros for a row of nothing but -inf, None for one with NaN or +inf."""
    x = x.double()
    if x.isnan().any() or (x == INF).any():
        return None
    if (x == -INF).all():
        return torch.zeros_like(x)
    return torch.softmax(x / T, 0)


def walk(target, draft, tokens, parents, coins, n, T, Td):
    """path, log ratios of the nodes tried, remainder at the end, whether a coin is near its threshold."""
    V = target.shape[1]
    path, ell, close = [0], {}, False
    while True:
        u = path[-1]
        kids = [i for i in range(u + 1, n) if int(parents[i]) == u]
        q = softmax64(target[u], T)
        rest = q
        went = None
        if kids:
            p = None if draft is None else softmax64(draft[u], Td)
            fair = q is not None and float(q.sum()) > 0 and (draft is None or p is not None)
            some = p is not None and float(p.sum()) > 0
            beta, mass = 0.0, 1.0
            for i in kids:
                x = int(tokens[i])
                if not 0 <= x < V or not fair:
                    continue
                lq = math.log(q[x]) if q[x] > 0 else -INF
                if draft is None:
                    ell[i], h = lq, float(rest[x])
                else:
                    lp = math.log(p[x]) if some and p[x] > 0 else -INF
                    ell[i] = -INF if lq == -INF else lq - lp
                    h = (INF if rest[x] > 0 else 0.0) if lp == -INF else float(rest[x] / p[x])
                eta = float(coins[i])
                close |= abs(eta - h) < 4e-6 * (abs(h) * mass + 2 * beta) / mass + 1e-6
                if eta < h:
                    went = i
                    break
                if draft is None:
                    rest = rest.clone()
                    rest[x] = 0
                elif some:
                    rest = (rest - p).clamp(min=0)
                left = float(rest.sum())
                beta, mass = beta + mass, mass * left
                close |= mass < 0.02                     # little is left of the target: its own rounding decides
                if left > 0:
                    rest = rest / left
        if went is None:
            return path, ell, rest, q, close
        path.append(went)


def make_tree(g, B, W, V, dtype, T=1.0, kind="tree", chosen=False, noise=0.6, parents=None):
    """Rows of a target and a drafter near it, children's tokens drawn from their parent's draft row (or its likeliest)."""
    target = 2.0 * torch.randn(B, W, V, generator=g, device="cuda")
    draft = (target + noise * torch.randn(B, W, V, generator=g, device="cuda")).to(dtype)
    par = [tree_of(kind, W, b) for b in range(B)] if parents is None else [parents] * B
    tokens = torch.zeros(B, W, dtype=torch.int32, device="cuda")
    for b in range(B):
        seen = [0] * W
        for i in range(W):
            u = par[b][i]
            if u < 0:
                continue
            if chosen:
                tokens[b, i] = draft[b, u].float().topk(min(V, seen[u] + 1)).indices[-1]
            else:
                e = torch.empty(V, device="cuda").exponential_(generator=g)
                tokens[b, i] = (draft[b, u].float() / T - e.log()).argmax()
            seen[u] += 1
    return (target.to(dtype), None if chosen else draft, tokens, torch.tensor(par, dtype=torch.int32, device="cuda"),
            torch.rand(B, W, generator=g, device="cuda"), torch.empty(B, V, device="cuda").exponential_(generator=g))


def check(api, target, draft, tokens, parents, coins, race, counts=None, T=1.0, Td=None, skips=None, **kw):
    B, W, V = target.shape
    r = api.tree_verify(target, draft, tokens, parents, counts=counts, temperature=T, draft_temperature=Td, coins=coins, race=race,
                        with_status=True, **kw)
    acc, nxt, paths = r["accepted_len"].tolist(), r["next_token"].tolist(), r["path"].tolist()
    skipped = 0
    for b in range(B):
        n = W if counts is None else min(W, int(counts[b]))
        if n <= 0:
            assert acc[b] == 0 and nxt[b] == -1 and paths[b] == [-1] * W and (r["log_ratio"][b] == 0).all() and int(r["status"][b]) == 0
            continue
        path, ell, rest, q, close = walk(target[b], None if draft is None else draft[b], tokens[b], parents[b], coins[b], n, T, Td or T)
        if close:
            skipped += 1
            continue
        assert paths[b] == path + [-1] * (W - len(path)) and acc[b] == len(path) - 1, (b, paths[b], path)
        want = torch.zeros(W, dtype=torch.float64, device="cuda")
        for i, e in ell.items():
            want[i] = e
        assert near(r["log_ratio"][b], want, 3e-5)
        i = nxt[b]
        if q is None or float(q.sum()) == 0:
            assert i == -1
            continue
        if float(rest.sum()) == 0:
            rest = q
        score = rest / race[b].double()
        slack = (1e-5 * q + 1e-5 * rest) / 0.02 / race[b].double()    # 1e-6 of q and of p, against what is left
        assert 0 <= i < V and float(rest[i]) > 0 and float(score[i] + slack[i]) >= float(score.max()) - float(slack[score.argmax()]), (b, i)
    assert skipped <= (max(2, B // 3) if skips is None else skips)
    return r


@pytest.mark.parametrize("chosen", [False, True])
@pytest.mark.parametrize("B,W,V,dtype,kind", [
    (1, 1, 2, F32, "tree"), (1, 2, 1, BF16, "chain"), (6, 4, 5, F32, "star"), (9, 16, 1000, F32, "tree"), (5, 12, 5001, BF16, "star"),
    (7, 33, 4099, F32, "tree"), (2, 64, 33000, F16, "tree"), (40, 9, 517, F16, "star"), (3, 64, 300, F32, "star"),
    (200, 7, 70, BF16, "tree"), (1, 24, 131072, BF16, "tree"), (2, 6, 200001, F32, "star")])
def test_tree_verify(api, B, W, V, dtype, kind, chosen):
    g = gen(B + 10 * W + V)
    t = make_tree(g, B, W, V, dtype, kind=kind, chosen=chosen)
    check(api, *t)
    check(api, *make_tree(g, B, W, V, dtype, 0.8, kind, chosen, noise=1.2), T=0.8)
    counts = torch.randint(-1, W + 2, (B,), generator=g, device="cuda", dtype=torch.int32)
    check(api, *t, counts=counts, T=1.1, Td=0.9)


def test_rows_of_larger_buffers(api):
    """Logits in padded buffers, rows on no 16-byte boundary, of different phases for target and draft."""
    g = gen(3)
    for dtype, V in ((BF16, 1003), (F32, 777)):
        target, draft, tokens, parents, coins, race = make_tree(g, 3, 8, V, dtype)
        tb = torch.randn(3, 9, V + 7, generator=g, device="cuda").to(dtype)
        db = torch.randn(3, 8, V + 6, generator=g, device="cuda").to(dtype)
        tb[:, 1:, 3:V + 3], db[:, :, 5:V + 5] = target, draft
        a = check(api, target, draft, tokens, parents, coins, race)
        b = check(api, tb[:, 1:, 3:V + 3], db[:, :, 5:V + 5], tokens, parents, coins, race)
        assert torch.equal(a["path"], b["path"]) and torch.equal(a["next_token"], b["next_token"])


def test_a_chain_is_sample_verification(api):
    """A tree of one path: token_verify in sample mode, bit by bit."""
    g = gen(9)
    for B, L, V, dtype in ((5, 4, 3001, F32), (3, 8, 32000, BF16), (16, 2, 100, F16)):
        tl, dl, tok, coins, race = make_verify(g, B, L, V, dtype)
        a = api.token_verify(tl, dl, tok, mode="sample", coins=coins, race=race)
        pad = torch.zeros(B, 1, V, device="cuda", dtype=dtype)
        tree = torch.cat([torch.zeros_like(tok[:, :1]), tok], 1)
        par = torch.arange(-1, L, device="cuda", dtype=torch.int32).expand(B, L + 1).contiguous()
        c = torch.cat([torch.zeros_like(coins[:, :1]), coins], 1)
        b = api.tree_verify(tl, torch.cat([dl, pad], 1), tree, par, coins=c, race=race)
        assert torch.equal(a["accepted_len"], b["accepted_len"]) and torch.equal(a["next_token"], b["next_token"])
        inside = torch.arange(L, device="cuda") <= a["accepted_len"][:, None]
        assert near(torch.where(inside, a["log_ratio"], 0.0), b["log_ratio"][:, 1:].double(), 2e-6)


def test_masks_bad_rows_and_tokens(api):
    from paper_2606_13426_gb300 import binding as Bd
    g = gen(4)
    B, V = 12, 600
    parents = [-1, 0, 0, 1, 1, 2, 0]
    W = len(parents)
    target, draft, tokens, par, coins, race = make_tree(g, B, W, V, F32, parents=parents)
    target[1, 0] = -INF                                 # a target without probabilities
    draft[2, 0] = -INF                                  # a draft without any
    target[3, 0, 5] = NAN
    draft[4, 0, 7] = NAN
    draft[5, 0, 9] = INF
    tokens[6, 1], tokens[6, 2] = -1, V                  # no tokens: passed over
    target[7, 0, tokens[7, 1].long()] = -INF            # an impossible token
    draft[8, 0, tokens[8, 1].long()] = -INF             # one that the draft calls impossible
    target[9, 0, 300:] = -INF                           # half of the target masked away, as of the draft
    draft[9, 0, 300:] = -INF
    target[10, 1:] = torch.finfo(torch.float32).min     # rows of the type's lowest value: flat ones
    tokens[11, 2] = tokens[11, 1]                        # twice the same token
    r = check(api, target, draft, tokens, par, coins, race, skips=4)
    status = r["status"].tolist()
    assert status[0] == 0 and status[1] == Bd.SDV_STATUS_EMPTY_ROW and status[2] & Bd.SDV_STATUS_EMPTY_ROW
    assert all(status[i] & Bd.SDV_STATUS_NONFINITE for i in (3, 4, 5)) and status[6] & Bd.SDV_STATUS_BAD_TOKEN
    target[4, 0], target[8, 0] = target[0, 0], target[0, 0]
    check(api, target, None, tokens, par, coins, race, skips=4)
    # trees that are none
    par = par.clone()
    par[0, 2], par[1, 1], par[2, 0] = 2, 5, 3
    st = api.tree_verify(target, draft, tokens, par, coins=coins, race=race, with_status=True)
    assert all(st["status"].tolist()[i] & Bd.SDV_STATUS_BAD_TREE for i in range(3)) and not st["status"][3:].bitwise_and(Bd.SDV_STATUS_BAD_TREE).any()


def test_nothing_left(api):
    """A draft equal to the target leaves nothing after a rejection (which its coin, at 1 or more, makes here): the target's
    own row is drawn from; chosen tokens that are all of the target likewise."""
    from paper_2606_13426_gb300 import binding as Bd
    g = gen(6)
    x = torch.randn(2, 3, 50, generator=g, device="cuda")
    par = torch.tensor([[-1, 0, 0]] * 2, device="cuda", dtype=torch.int32)
    tok = torch.tensor([[0, 3, 4]] * 2, device="cuda", dtype=torch.int32)
    coins = torch.full((2, 3), 2.0, device="cuda")
    race = torch.empty(2, 50, device="cuda").exponential_(generator=g)
    r = api.tree_verify(x, x.clone(), tok, par, coins=coins, race=race, with_status=True)
    assert r["accepted_len"].tolist() == [0, 0] and (r["status"] == Bd.SDV_STATUS_ZERO_DELTA).all()
    want = (torch.softmax(x[:, 0].double(), 1) / race.double()).argmax(1)
    assert torch.equal(r["next_token"].long(), want)
    y = torch.full((2, 3, 50), -INF, device="cuda")
    y[:, :, 3:5] = 1.0
    r = api.tree_verify(y, None, tok, par, coins=coins, race=race, with_status=True)
    assert (r["status"] == Bd.SDV_STATUS_ZERO_DELTA).all() and set(r["next_token"].tolist()) <= {3, 4}


@pytest.mark.parametrize("chosen", [False, True])
def test_emitted_tokens_follow_the_target(api, chosen):
    """The first two emitted tokens of a small tree, over many seeded calls, against the target's distribution."""
    g = gen(77)
    V, B = 5, 120_000
    parents = [-1, 0, 0, 0, 1, 1, 2, 3]
    W = len(parents)
    first, second = 1.3 * torch.randn(V, generator=g, device="cuda"), 1.3 * torch.randn(V, V, generator=g, device="cuda")
    d_first, d_second = first + torch.randn(V, generator=g, device="cuda"), second + torch.randn(V, V, generator=g, device="cuda")
    tokens = torch.zeros(B, W, dtype=torch.int64, device="cuda")
    target = torch.zeros(B, W, V, device="cuda")
    draft = torch.zeros(B, W, V, device="cuda")
    target[:, 0], draft[:, 0] = first, d_first
    rank = [0] * W
    for i in range(1, W):
        u = parents[i]
        if chosen:
            tokens[:, i] = draft[:, u].argsort(1, descending=True)[:, rank[u]]
        else:
            e = torch.empty(B, V, device="cuda").exponential_(generator=g)
            tokens[:, i] = (draft[:, u] - e.log()).argmax(1)
        rank[u] += 1
        target[:, i], draft[:, i] = second[tokens[:, i]], d_second[tokens[:, i]]
    tok = tokens.to(torch.int32)
    par = torch.tensor(parents, device="cuda", dtype=torch.int32).expand(B, W).contiguous()
    r = api.tree_verify(target, None if chosen else draft, tok, par, seed=123)
    path, nxt = r["path"].long(), r["next_token"].long()
    one = torch.where(path[:, 1] >= 0, tokens.gather(1, path[:, 1:2].clamp(min=0))[:, 0], nxt)
    p1 = torch.softmax(first.double(), 0)
    count = torch.bincount(one, minlength=V).double()
    chi = float(((count - B * p1) ** 2 / (B * p1)).sum())
    assert chi < 30.0                                   # four degrees of freedom: 5e-6
    has = path[:, 1] >= 0
    two = torch.where(path[:, 2] >= 0, tokens.gather(1, path[:, 2:3].clamp(min=0))[:, 0], nxt)
    for t in range(V):
        at = has & (one == t)
        m = int(at.sum())
        if m < 500:
            continue
        p2 = torch.softmax(second[t].double(), 0)
        count = torch.bincount(two[at], minlength=V).double()
        assert float(((count - m * p2) ** 2 / (m * p2)).sum()) < 30.0
    assert 0.5 < float(has.double().mean()) < 1.0


def test_seeded_draws_are_those_of_their_counters(api):
    """Without coins and race they come from the counters that the header names."""
    g = gen(8)
    for B, W, V, dtype in ((30, 6, 41, F32), (3, 20, 40001, BF16)):
        target, draft, tokens, par, _, _ = make_tree(g, B, W, V, dtype)
        seed = 0x123456789ABCDEF0 + V
        coins, race = host_draws(seed, B, W, V)
        a = api.tree_verify(target, draft, tokens, par, seed)
        b = api.tree_verify(target, draft, tokens, par, coins=coins, race=race)
        for k in ("accepted_len", "path", "log_ratio"):
            assert torch.equal(a[k], b[k]), k
        assert int((a["next_token"] != b["next_token"]).sum()) <= 1     # (logarithms differ in their last bits)


def test_graph_stream_and_callers_outputs(api):
    g = gen(10)
    target, draft, tokens, par, coins, race = make_tree(g, 4, 10, 9001, BF16)
    ref = api.tree_verify(target, draft, tokens, par, coins=coins, race=race, with_status=True)
    out = {k: torch.empty_like(v) for k, v in ref.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.tree_verify(target, draft, tokens, par, coins=coins, race=race, with_status=True, out=out)
    side.synchronize()
    assert all(torch.equal(out[k], ref[k]) for k in ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.tree_verify(target, draft, tokens, par, coins=coins, race=race, with_status=True, out=out)
    for seed in (1, 2):
        coins.copy_(torch.rand(4, 10, generator=gen(seed), device="cuda"))
        ref = api.tree_verify(target, draft, tokens, par, coins=coins, race=race, with_status=True)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], ref[k]) for k in ref)


def test_refusals(api):
    from paper_2606_13426_gb300 import binding as B
    x = torch.zeros(2, 3, 10, device="cuda")
    tok = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    par = torch.tensor([[-1, 0, 0]] * 2, dtype=torch.int32, device="cuda")
    for kw in (dict(temperature=0.0), dict(draft_temperature=-1.0), dict(temperature=float("nan"))):
        with pytest.raises(B.SDVError):
            api.tree_verify(x, x, tok, par, **kw)
    for bad in ((x, x[:, :2], tok, par), (x, x.to(BF16), tok, par), (x, x, tok.long(), par), (x, x, tok, par[:, :2]), (x.cpu(), x, tok, par),
                (x, x, tok, par.cpu())):
        with pytest.raises(ValueError):
            api.tree_verify(*bad)
    big = torch.zeros(1, 65, 4, device="cuda")
    with pytest.raises(B.SDVError):
        api.tree_verify(big, big, torch.zeros(1, 65, dtype=torch.int32, device="cuda"), torch.zeros(1, 65, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("chosen", [False, True])
def test_many_calls_at_once_agree(api, chosen):
    """Clusters side by side on a full GPU, many times over: all of a cluster's CTAs see the same tree."""
    g = gen(11)
    B, W, V = 48, 24, 20001
    target = torch.randn(B, W, V, generator=g, device="cuda")
    draft = None if chosen else torch.randn(B, W, V, generator=g, device="cuda")
    tokens = torch.randint(0, V, (B, W), generator=g, device="cuda", dtype=torch.int32)
    parents = torch.stack([torch.tensor(tree_of("tree", W, b)) for b in range(B)]).to(torch.int32).cuda()
    coins = torch.rand(B, W, generator=g, device="cuda") * (1e-4 if chosen else 1.0)
    first = api.tree_verify(target, draft, tokens, parents, seed=3, coins=coins, with_status=True)
    outs = [api.tree_verify(target, draft, tokens, parents, seed=3, coins=coins, with_status=True) for _ in range(300)]
    assert int(first["accepted_len"].max()) > 0 and not first["status"].any()
    for r in outs:
        assert all(torch.equal(r[key], first[key]) for key in first)
