"""The token operators (scores and their gradient, verification, the 8-bit cache and the
attention over it) against plain implementations in 64 bits.

Tolerances, with u = 2^-24 (fp32) and set from the kernels' arithmetic:
  * log s: a thread adds up at most 64 terms of these sizes one after another, a tree of 5 + 3 + 3
    steps joins them, the exponential is within 2^-22 and its argument within |d| u: below
    100 u = 6e-6 for the distributions here; log probabilities add the rounding of d.
    TOL = 1e-5 (1 + |value|).
  * entropy: the same relative errors on sum p |d|, which is below 20 here: 2e-5 (1 + |value|).
  * gradients: p (a + b d) with log p within TOL: 3e-5 times the sum of the terms' magnitudes, and
    the type's rounding (2^-8 bf16, 2^-11 f16 relative; 2^-25 absolute for f16 subnormals).
  * attention: probabilities are rounded to 11 bits (2^-11 relative), outputs to their type
    (2^-8 or 2^-11 relative): 2^-11 sum p |v| + the output's rounding; lse 2e-5 (1 + |lse|).
  * cache codes and scales are exact.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN, INF = math.nan, math.inf


@pytest.fixture(scope="module")
def api():
    import __graft_entry__ as g
    g.build()
    from paper_2606_13426_gb300 import api as A
    return A


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def near(got, ref, rtol):
    """Finite values within rtol (1 + |ref|), the others equal (a reference past fp32's range is
    its infinity)."""
    got, ref = got.double(), torch.where(ref.double().abs() < 3.4028235e38, ref.double(), ref.float().double())
    same = (got == ref) | (got.isnan() & ref.isnan())
    return bool((same | ((got - ref).abs() <= rtol * (1 + ref.abs()))).all())


# ------------------------------------------------------------------------------ scores
def plain_scores(x, tok, T, k):
    """Scores of finite or -inf logits in 64 bits, and the order of the alternatives."""
    z = x.double()
    N, V = z.shape
    m = z.amax(1)
    d = torch.where(z == -INF, -INF, (z - m[:, None])) / T
    d = torch.where(m[:, None] == -INF, -INF, d)
    s = d.exp().sum(1)
    lp = d - s.log()[:, None]
    lp = torch.where(m[:, None] == -INF, -INF, lp)
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, 0.0).sum(1)
    t = tok.long()
    bad = (t >= V) | (t < -1)
    at = lp.gather(1, t.clamp(0, V - 1)[:, None])[:, 0]
    logprob = torch.where(t == -1, 0.0, torch.where(bad, NAN, at))
    r = dict(logprob=logprob, entropy=H, row_max=m, log_sum=s.log(), lp=lp, p=p, bad=bad)
    if k:
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
        top = lp.gather(1, order)
        r["top_ids"] = torch.where(top == -INF, -1, order).to(torch.int32)
        r["top_logprob"] = top
    return r


def make_logits(g, N, V, dtype, pad=0, off=0, special=True):
    buf = 3.0 * torch.randn(off + N * (V + pad), generator=g, device="cuda")
    x = buf.to(dtype)[off:].view(N, V + pad)[:, :V]
    if special:
        if N > 2:
            x[1] = torch.where(torch.rand(V, generator=g, device="cuda") < 0.9, torch.tensor(-INF, device="cuda", dtype=dtype), x[1])
        if N > 3:
            x[3] = -INF                                   # nothing left
        if N > 4:
            x[4] = 1.25                                   # all equal: ties go to the lowest index
        if N > 5:
            x[5] = torch.finfo(dtype).min                 # masked by the type's lowest value, all of it
        if N > 6:
            x[6, : V // 2] = torch.finfo(dtype).min
        if N > 7:
            x[7] = (x[7] * 0.5).round()                   # many ties
    return x


def make_tokens(g, N, V):
    t = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    if N > 8:
        t[8] = -1
        t[2] = V
        t[0] = -2
    return t


SIZES = [(1, 1, 0, 0), (3, 2, 0, 0), (9, 7, 0, 1), (12, 33, 3, 0), (11, 1000, 0, 1), (10, 4099, 6, 3), (40, 5001, 0, 0),
         (700, 65, 1, 0), (10, 70001, 5, 0), (9, 65536, 0, 0)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("N,V,pad,off", SIZES)
def test_scores(api, N, V, pad, off, dtype):
    g = gen(N * 7 + V)
    x = make_logits(g, N, V, dtype, pad, off)
    tok = make_tokens(g, N, V)
    for k, T in ((0, 1.0), (min(V, 5), 0.7), (min(V, 32), 1.0)):
        r = api.token_scores(x, tok, top_k=k, temperature=T, with_status=True)
        o = plain_scores(x, tok, T, k)
        assert near(r["logprob"], o["logprob"], 1e-5)
        assert near(r["entropy"], o["entropy"], 2e-5)
        assert torch.equal(r["row_max"].double(), o["row_max"])
        assert near(r["log_sum"], o["log_sum"], 1e-5)
        if k:
            assert torch.equal(r["top_ids"], o["top_ids"])
            assert near(r["top_logprob"], o["top_logprob"], 1e-5)
        st = r["status"]
        assert torch.equal((st & 16) != 0, o["bad"])
        assert torch.equal((st & 8) != 0, o["row_max"] == -INF)
        assert not (st & 2).any()


def test_scores_of_rows_with_nan_or_inf(api):
    g = gen(1)
    x = make_logits(g, 6, 3001, F32, special=False)
    x[1, 2999] = NAN
    x[2, 5] = INF
    x[3, 0] = NAN
    tok = torch.tensor([0, 7, 5, 9, -1, 0], device="cuda", dtype=torch.int32)
    r = api.token_scores(x, tok, top_k=4, with_status=True)
    bad = torch.tensor([0, 1, 1, 1, 0, 0], device="cuda").bool()
    for k in ("logprob", "entropy", "row_max", "log_sum"):
        assert torch.equal(r[k].isnan(), bad)
    assert (r["top_ids"][bad] == -1).all() and r["top_logprob"][bad].isnan().all()
    assert torch.equal(r["status"], 2 * bad.int())
    o = plain_scores(x[~bad], tok[~bad], 1.0, 4)
    assert torch.equal(r["top_ids"][~bad], o["top_ids"])
    dx = api.token_scores_grad(x, tok, r, torch.ones(6, device="cuda"))
    assert dx[bad].isnan().all() and dx[~bad].isfinite().all()


def test_alternatives_concentrated_in_one_place(api):
    """The largest logits next to each other, at the ends, in one vector; sorted rows."""
    V = 40000
    x = torch.randn(5, V, generator=gen(3), device="cuda")
    x[0, 1000:1200] += 50
    x[1, :40] += 50
    x[2, -40:] += 50
    x[3] = x[3].sort().values
    x[4] = x[4].sort(descending=True).values
    for dtype in (F32, BF16):
        y = x.to(dtype)
        r = api.token_scores(y, top_k=32)
        o = plain_scores(y, torch.zeros(5, device="cuda", dtype=torch.int32), 1.0, 32)
        assert torch.equal(r["top_ids"], o["top_ids"])


def grad_ok(dx, x, tok, o, gl, gh, T):
    V = x.shape[1]
    p, lp, H = o["p"], o["lp"], o["entropy"]
    on = ((tok >= 0) & (tok < V)).double()
    up = gl.double() * on
    hot = torch.zeros_like(p).scatter_(1, tok.long().clamp(0, V - 1)[:, None], 1.0) * on[:, None]
    lpz = torch.where(p > 0, lp, 0.0)
    ref = (up[:, None] * (hot - p) - gh.double()[:, None] * p * (lpz + H[:, None])) / T
    ref = torch.where(x == -INF, 0.0, ref)
    size = (up.abs()[:, None] * (hot + p) + gh.double().abs()[:, None] * p * (lpz.abs() + H[:, None])) / T
    half = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}[x.dtype]
    tol = 3e-5 * size + half * ref.abs() * 1.01 + (2.0 ** -25 if x.dtype == F16 else 1e-37)
    return bool(((dx.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("N,V,pad,off", SIZES + [(3, 140001, 0, 0), (2, 210001, 0, 1)])
def test_gradient_matches_the_formula(api, N, V, pad, off, dtype):
    g = gen(N + 3 * V)
    x = make_logits(g, N, V, dtype, pad, off)
    tok = make_tokens(g, N, V)
    gl, gh = torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
    zero = torch.zeros(N, device="cuda")
    T = 0.8
    o = plain_scores(x, tok, T, 0)
    r = api.token_scores(x, tok, temperature=T, with_status=True)
    assert grad_ok(api.token_scores_grad(x, tok, r, gl, gh, temperature=T), x, tok, o, gl, gh, T)
    assert grad_ok(api.token_scores_grad(x, tok, r, gl, temperature=T), x, tok, o, gl, zero, T)
    assert grad_ok(api.token_scores_grad(x, tok, r, None, gh, temperature=T), x, tok, o, zero, gh, T)
    wide = torch.full((N, V + 3), 7.0, dtype=dtype, device="cuda")      # another layout of the rows
    t = api.token_scores_train(x, tok, gl, gh, temperature=T, d_logits=wide[:, :V], with_status=True)
    assert grad_ok(wide[:, :V], x, tok, o, gl, gh, T) and (wide[:, V:] == 7).all()
    for k in ("logprob", "entropy", "log_sum"):
        assert near(t[k], o[k], 2e-5)
    assert torch.equal(t["status"], r["status"])
    t = api.token_scores_train(x, None, None, gh, temperature=T)
    assert grad_ok(t["d_logits"], x, tok, o, zero, gh, T)
    for fused in (False, True):                                          # in place
        y = x.clone() if pad == 0 and off == 0 else x
        if fused:
            y2 = torch.empty_like(y)
            y2.copy_(y)
            t = api.token_scores_train(y2, tok, gl, gh, temperature=T, d_logits=y2)
            assert grad_ok(y2, x, tok, o, gl, gh, T) and near(t["logprob"], o["logprob"], 1e-5)
        else:
            y2 = torch.empty_like(y)
            y2.copy_(y)
            assert grad_ok(api.token_scores_grad(y2, tok, r, gl, gh, temperature=T, d_logits=y2), x, tok, o, gl, gh, T)


@pytest.mark.parametrize("T", [1e-9, 1e9])
def test_extreme_temperatures_with_masks(api, T):
    """Masked logits have no part in anything at either end of the temperatures: nearly one-hot, nearly flat."""
    g = gen(52)
    N, V = 6, 1500
    x = 3.0 * torch.randn(N, V, generator=g, device="cuda")
    masked = torch.rand(N, V, generator=g, device="cuda") < 0.5
    masked[:, 0] = False
    x[masked] = -INF
    tok = torch.zeros(N, dtype=torch.int32, device="cuda")
    one = torch.ones(N, device="cuda")
    r = api.token_scores_train(x, tok, one, one, temperature=T)
    live = (~masked).sum(1).double()
    dx = r["d_logits"].double()
    assert (dx[masked] == 0).all() and not dx.isnan().any()
    if T > 1:
        assert near(r["logprob"], -live.log(), 1e-5) and near(r["entropy"], live.log(), 1e-5)
        p = torch.where(masked, 0.0, 1 / live[:, None])
        want = ((torch.arange(V, device="cuda") == 0).double() - p) / T
        # p (log p + H): the parts of H - log s + d/T cancel to about 1e-6 of themselves, against 1
        assert ((dx - want).abs() <= 1e-5 / T * (p * live[:, None].log() + want.abs() * T)).all()
    else:
        assert (r["entropy"] == 0).all() and (x.gather(1, x.argmax(1)[:, None])[:, 0] == r["row_max"]).all()
    v = api.token_verify(x[None, :4], x[None, :3], x[:3].argmax(1).to(torch.int32)[None], 5, "block", temperature=T)
    assert int(v["accepted_len"]) == 3 and not masked[3, int(v["next_token"])]


def test_gradient_matches_differences(api):
    """Central differences of the forward kernel: step 1e-2, so that its 1e-5 (1 + |value|) weighs 4e-3
    at most here, and the third derivative's share is below 1e-4."""
    g = gen(5)
    N, V, T, h = 4, 23, 1.3, 1e-2
    x = torch.randn(N, V, generator=g, device="cuda")
    x[1, 3:9] = -INF
    tok = torch.tensor([3, 1, -1, 22], device="cuda", dtype=torch.int32)
    gl, gh = torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
    dx = api.token_scores_train(x, tok, gl, gh, temperature=T)["d_logits"]
    for v in range(V):
        up, dn = x.clone(), x.clone()
        up[:, v] += h
        dn[:, v] -= h
        a, b = (api.token_scores(y, tok, temperature=T) for y in (up, dn))
        f = (gl * (a["logprob"] - b["logprob"]) + gh * (a["entropy"] - b["entropy"])) / (2 * h)
        assert ((f - dx[:, v]).abs() <= 8e-3).all()


def test_scores_refuse(api):
    from paper_2606_13426_gb300 import binding as B
    x = torch.zeros(4, 10, device="cuda")
    t = torch.zeros(4, device="cuda", dtype=torch.int32)
    with pytest.raises(ValueError):
        api.token_scores(x.double(), t)
    with pytest.raises(ValueError):
        api.token_scores(x.t(), t)
    with pytest.raises(ValueError):
        api.token_scores(x, t.long())
    with pytest.raises(ValueError):
        api.token_scores(x.cpu(), t)
    for kw in (dict(top_k=11), dict(top_k=33), dict(top_k=-1), dict(temperature=0.0), dict(temperature=NAN), dict(temperature=-1.0),
               dict(temperature=1e-39)):
        with pytest.raises((B.SDVError, RuntimeError, ValueError)):
            api.token_scores(x, t, **kw)
    with pytest.raises(B.SDVError):
        api.token_scores_grad(x, t, api.token_scores(x, t))
    assert api.token_scores(x[:0], t[:0])["logprob"].shape == (0,)


# ------------------------------------------------------------------------------ verification
def plain_verify(tl, dl, tok, coins, race, mode, n, T, Td):
    """One chain in 64 bits: log ratios, the thresholds that its coins meet, accepted length for the
    coins, and r of the next token for every accepted length."""
    V = tl.shape[-1]

    def soft(z, t):
        z = z.double() / t
        return torch.softmax(z, -1) if bool((z > -INF).any()) else torch.zeros_like(z)
    q = [soft(tl[j], T) for j in range(n + 1)]
    p = [soft(dl[j], Td) for j in range(n)]
    ell, alpha = [], [1.0]
    for j in range(n):
        t = int(tok[j])
        a, b = (float(q[j][t]), float(p[j][t])) if 0 <= t < V else (NAN, 1.0)
        e = NAN if a != a else -INF if a == 0 else INF if b == 0 else math.log(a) - math.log(b)
        ell.append(e)
        alpha.append(0.0 if e != e or e == -INF else min(1.0, alpha[-1] * (math.exp(min(e, 50.0)))))
    thr = []
    for j in range(1, n + 1):
        if mode == "sample":
            thr.append(0.0 if ell[j - 1] != ell[j - 1] else math.exp(min(ell[j - 1], 0.0)))
        elif j == n or alpha[j] == 1.0:
            thr.append(alpha[j])
        else:
            v = float((alpha[j] * q[j] - p[j]).clamp(min=0).sum())
            thr.append(v / (v + 1 - alpha[j]))
    hit = [float(coins[j]) < thr[j] for j in range(n)]
    if mode == "sample":
        acc = hit.index(False) if False in hit else n
        alpha = [1.0] * (n + 1)
    else:
        acc = max([j + 1 for j in range(n) if hit[j]], default=0)
    close = any(abs(float(coins[j]) - thr[j]) < 2e-5 for j in range(n))
    r = q[acc] if acc == n else (alpha[acc] * q[acc] - p[acc]).clamp(min=0)
    return ell, acc, close, r


def make_verify(g, B, L, V, dtype, T=1.0, noise=0.7):
    tl = 2.0 * torch.randn(B, L + 1, V, generator=g, device="cuda")
    dl = (tl[:, :L] + noise * torch.randn(B, L, V, generator=g, device="cuda")).to(dtype)
    e = torch.empty(B, L, V, device="cuda").exponential_(generator=g)
    tok = (dl.float() / T - e.log()).argmax(2).to(torch.int32)
    return (tl.to(dtype), dl, tok, torch.rand(B, L, generator=g, device="cuda"),
            torch.empty(B, V, device="cuda").exponential_(generator=g))


def check_verify(api, tl, dl, tok, coins, race, mode, n=None, T=1.0, Td=None, free=()):
    B, L, V = dl.shape
    r = api.token_verify(tl, dl, tok, mode=mode, temperature=T, draft_temperature=Td, L_eff=n, coins=coins, race=race)
    acc, nxt, lr = r["accepted_len"].tolist(), r["next_token"].tolist(), r["log_ratio"]
    skipped = 0
    for b in range(B):
        nb = L if n is None else int(n[b])
        if nb < 0:
            assert acc[b] == 0 and nxt[b] == -1 and (lr[b] == 0).all()
            continue
        nb = min(nb, L)
        ell, a, close, rest = plain_verify(tl[b], dl[b], tok[b], coins[b], race[b], mode, nb, T, Td or T)
        assert near(lr[b, :nb], torch.tensor(ell, device="cuda", dtype=torch.float64), 3e-5), (lr[b], ell)
        assert (lr[b, nb:] == 0).all()
        if close:
            skipped += 1
            continue
        assert acc[b] == a, (b, acc[b], a)
        score = rest / race[b].double()
        if float(rest.sum()) < 1e-5:
            continue
        best = float(score.max())
        # a residual of differences: 1e-6 of q and p in each, against what is left
        slack = (4e-6 * torch.softmax(tl[b, a].double() / T, -1) * 2 + 4e-6 * rest) / race[b].double()
        i = nxt[b]
        assert 0 <= i < V and float(score[i] + slack[i]) >= best - float(slack[score.argmax()]), (b, i)
    assert skipped <= max(1, B // 4)
    return r


@pytest.mark.parametrize("mode", ["block", "sample"])
@pytest.mark.parametrize("B,L,V,dtype", [(1, 1, 2, F32), (3, 2, 5, BF16), (5, 4, 1000, F32), (4, 3, 5001, BF16), (7, 5, 4099, F32),
                                         (2, 8, 33000, F16), (30, 6, 517, F16), (2, 64, 300, F32), (200, 3, 70, F32)])
def test_verify(api, B, L, V, dtype, mode):
    g = gen(B + 10 * L + V)
    tl, dl, tok, coins, race = make_verify(g, B, L, V, dtype)
    check_verify(api, tl, dl, tok, coins, race, mode)
    n = torch.randint(-1, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_verify(api, tl, dl, tok, coins, race, mode, n, T=0.8)
    check_verify(api, tl, dl, tok, coins, race, mode, n, T=0.9, Td=1.2)


@pytest.mark.parametrize("B,L,V,dtype", [(16, 8, 32768, BF16), (16, 8, 40001, BF16), (3, 1, 3, F32), (2, 3, 20000, F32),
                                         (128, 8, 4096, F16), (128, 8, 5000, F16)])
def test_verify_with_statistics_taken_in_one_kernel_or_two(api, B, L, V, dtype):
    """Sizes on both sides of where the chains' clusters take their rows' statistics themselves."""
    g = gen(B + L + V)
    tl, dl, tok, coins, race = make_verify(g, B, L, V, dtype)
    n = torch.randint(-1, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_verify(api, tl, dl, tok, coins, race, "block", n, T=0.9)
    check_verify(api, tl, dl, tok, coins, race, "sample")


def test_verify_of_strided_and_unaligned_rows(api):
    g = gen(11)
    for dtype in (F32, BF16):
        B, L, V = 3, 4, 2049
        tl, dl, tok, coins, race = make_verify(g, B, L, V, dtype)
        a = torch.zeros(B, L + 1, V + 3, dtype=dtype, device="cuda")[..., 1:V + 1]
        b = torch.zeros(B, L + 2, V + 7, dtype=dtype, device="cuda")[:, 1:L + 1, 5:V + 5]
        a.copy_(tl)
        b.copy_(dl)
        x = check_verify(api, tl, dl, tok, coins, race, "block")
        y = check_verify(api, a, b, tok, coins, race, "block")
        assert torch.equal(x["accepted_len"], y["accepted_len"]) and torch.equal(x["next_token"], y["next_token"])


def test_verify_masks_and_bad_rows(api):
    g = gen(12)
    B, L, V = 12, 3, 600
    tl, dl, tok, coins, race = make_verify(g, B, L, V, F32)
    tl[0, :, 300:] = -INF                    # the target allows half of the tokens
    dl[1, :, :300] = -INF                    # the draft proposes from half of them
    tok[1] = 5                               # a token that the draft calls impossible
    tl[2, 1] = -INF                          # an empty target row
    dl[3, 0] = -INF                          # an empty draft row
    tl[4, 0, 17] = NAN
    dl[5, 1, 3] = INF
    tok[6, 0] = V
    tok[7, 1] = -1
    tl[8, 0] = torch.finfo(F32).min          # flat
    dl[9] = tl[9, :L]                        # a drafter that is right: all is accepted
    tl[10, :, 1:] = -INF                     # one token is left
    tl[11, L] = -INF                         # nothing to draw on full accept
    dl[11] = tl[11, :L]
    for mode in ("block", "sample"):
        ok = [0, 1, 8, 9, 10]
        check_verify(api, tl[ok], dl[ok], tok[ok], coins[ok], race[ok], mode)
        r = api.token_verify(tl, dl, tok, mode=mode, coins=coins, race=race, with_status=True)
        acc, nxt, st, lr = (r[k].tolist() for k in ("accepted_len", "next_token", "status", "log_ratio"))
        assert all(t < 300 for t in nxt[:1])
        assert lr[1] == [INF] * L
        assert lr[2][1] == -INF and st[2] & 8 and (acc[2] != 1 or nxt[2] == -1)
        assert st[3] & 8 and lr[3][0] == INF
        assert st[4] & 2 and acc[4] == 0 and nxt[4] == -1 and lr[4][0] != lr[4][0]
        assert st[5] & 2 and lr[5][1] != lr[5][1] and acc[5] <= 1
        assert st[6] & 16 and acc[6] == 0 and lr[6][0] != lr[6][0]
        assert st[7] & 16 and acc[7] <= 1
        assert acc[9] == L and all(abs(v) < 1e-5 for v in lr[9])
        assert nxt[10] == 0
        assert acc[11] == L and nxt[11] == -1


def test_verify_an_impossible_token_before_one_the_draft_calls_impossible(api):
    """alpha = 0 behind a token that the target masks, whatever follows: ell = +inf does not bring it back."""
    g = gen(13)
    B, L, V = 4, 4, 300
    tl, dl, tok, coins, race = make_verify(g, B, L, V, F32)
    tl[:, 1, 7] = -INF
    tok[:, 1] = 7                            # rejected, and with it all that follows
    dl[:, 2, 9] = -INF
    dl[:, 3, 9] = -INF
    tok[:, 2:] = 9
    coins[:] = 0.25
    for mode in ("block", "sample"):
        r = api.token_verify(tl, dl, tok, mode=mode, coins=coins, race=race)
        assert (r["accepted_len"] <= 1).all()
        assert r["log_ratio"][:, 1].tolist() == [-INF] * B and r["log_ratio"][:, 2:].flatten().tolist() == [INF] * 2 * B


def test_verify_with_nothing_left(api):
    """alpha q - p <= 0 everywhere, by a coin that no draw gives: the target's own row is drawn from."""
    tl = torch.zeros(1, 2, 100, device="cuda")
    dl = torch.zeros(1, 1, 100, device="cuda")
    tok = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    dl[0, 0, 0] = 1.0
    race = torch.full((1, 100), 2.0, device="cuda")
    race[0, 42] = 1.0
    tl[0, 0] = dl[0, 0]
    tl[0, 0, 7] = -INF                       # the rejected token: q = 0 there
    dl[0, 0, 7] = -INF
    tok[0, 0] = 7
    r = api.token_verify(tl, dl, tok, mode="sample", coins=torch.zeros(1, 1, device="cuda"), race=race, with_status=True)
    assert int(r["accepted_len"]) == 0 and int(r["status"]) & 1
    q = torch.softmax(tl[0, 0].double(), 0) / race[0].double()
    assert int(r["next_token"]) == int(q.argmax())


@pytest.mark.parametrize("mode", ["block", "sample"])
def test_emitted_tokens_follow_the_target(api, mode):
    """With draws from the seed, the first emitted token has the target's probabilities (chi-square of
    V - 1 degrees, its 1e-6 quantile), and so has the second where the first is a given one."""
    from scipy import stats
    g = gen(21)
    B, L, V = 40000, 3, 7
    tl = torch.randn(L + 1, V, generator=g, device="cuda").expand(B, L + 1, V).contiguous()
    dl = tl[:, :L] + torch.randn(L, V, generator=g, device="cuda")
    e = torch.empty(B, L, V, device="cuda").exponential_(generator=g)
    tok = (dl - e.log()).argmax(2).to(torch.int32)
    r = api.token_verify(tl, dl, tok, 77, mode)
    again = api.token_verify(tl, dl, tok, 77, mode)
    assert all(torch.equal(r[k], again[k]) for k in r)
    assert not torch.equal(api.token_verify(tl, dl, tok, 78, mode)["next_token"], r["next_token"])
    acc = r["accepted_len"].long()
    out = torch.cat([tok.long(), torch.zeros(B, 1, dtype=torch.long, device="cuda")], 1)
    out.scatter_(1, acc[:, None], r["next_token"].long()[:, None])
    q = torch.softmax(tl[0].double(), -1).cpu()
    first = torch.bincount(out[:, 0], minlength=V).double().cpu()
    assert float(((first - B * q[0]) ** 2 / (B * q[0])).sum()) < stats.chi2.ppf(1 - 1e-6, V - 1)
    two = out[acc >= 1]
    assert len(two) > B // 4
    # tokens here do not depend on each other, so that the pair (first, second) is q_0 q_1 on
    # chains with a second token once the unaccepted ones are drawn from q_1: test the first alone above
    assert int(two[:, 1].max()) < V


def test_verify_refuses(api):
    from paper_2606_13426_gb300 import binding as B
    g = gen(2)
    tl, dl, tok, coins, race = make_verify(g, 2, 3, 50, F32)
    with pytest.raises(ValueError):
        api.token_verify(tl[:, :3], dl, tok)
    with pytest.raises(ValueError):
        api.token_verify(tl, dl.to(BF16), tok)
    with pytest.raises(ValueError):
        api.token_verify(tl, dl, tok.long())
    with pytest.raises(ValueError):
        api.token_verify(tl, dl, tok, coins=coins[:, :2])
    with pytest.raises(B.SDVError):
        api.token_verify(tl, dl, tok, temperature=0.0)
    with pytest.raises(B.SDVError):
        api.token_verify(tl, dl, tok, draft_temperature=-1.0)
    with pytest.raises(KeyError):
        api.token_verify(tl, dl, tok, mode="greedy")
    big = torch.zeros(1, 66, 4, device="cuda")
    with pytest.raises(B.SDVError):
        api.token_verify(big, big[:, :65], torch.zeros(1, 65, dtype=torch.int32, device="cuda"))


# ------------------------------------------------------------------------------ cache
def e4m3(x):
    """The nearest e4m3 values in 64 bits, ties to even; infinities and what is above to 448."""
    a = x.abs().clamp(max=448)
    _, e = torch.frexp(a.clamp(min=2.0 ** -6))
    unit = ((e.long() - 4 + 1023) << 52).view(torch.float64)      # 2^(e - 4), exactly
    return torch.where(x.isnan(), NAN, torch.copysign(torch.round(a / unit) * unit, x))


def plain_append(cache, k_new, v_new, pages, lengths, counts):
    block = cache["k"].shape[2]
    got = dict(k=cache["k"].double(), v=cache["v"].double().transpose(2, 3).contiguous(), k_scale=cache["k_scale"].double(),
               v_scale=cache["v_scale"].double())
    for b in range(len(lengths)):
        n, new = int(lengths[b]), int(counts[b])
        for j in range(n // block, -(-(n + new) // block) if new > 0 else 0):
            page = int(pages[b, j])
            lo, hi = max(n, j * block), min(n + new, (j + 1) * block)
            kept = max(0, n - j * block)
            for codes, scales, x in ((got["k"], got["k_scale"], k_new), (got["v"], got["v_scale"], v_new)):
                y = x[b, lo - n:hi - n].double().transpose(0, 1)
                a = torch.where(y.isfinite(), y.abs(), 0.0).amax((1, 2))
                s = torch.full_like(a, 2.0 ** -126)
                for h in range(len(a)):
                    while 448 * float(s[h]) < float(a[h]):
                        s[h] *= 2
                if kept:
                    s = torch.maximum(s, scales[page])
                    for h in range(len(a)):
                        if s[h] != scales[page, h]:
                            codes[page, h, :kept] = e4m3(codes[page, h, :kept] * (scales[page, h] / s[h]))
                codes[page, :, lo - j * block:hi - j * block] = e4m3(y / s[:, None, None])
                scales[page] = s
    got["v"] = got["v"].transpose(2, 3)
    return got


def same(a, b):
    a, b = a.double(), b.double()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def random_cache(api, g, pages, H, block, D):
    c = api.make_token_cache(pages, H, block, D)
    for k in ("k", "v"):
        c[k].view(torch.uint8).copy_(torch.randint(0, 256, c[k].shape, generator=g, device="cuda", dtype=torch.uint8))
        c[k + "_scale"].copy_(2.0 ** torch.randint(-6, 3, (pages, H), generator=g, device="cuda"))
    return c


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("B,W,H,D,block", [(1, 1, 1, 64, 16), (5, 3, 2, 128, 64), (6, 9, 3, 64, 48), (4, 40, 2, 128, 16),
                                           (3, 300, 2, 64, 128), (2, 65, 1, 128, 64)])
def test_append(api, B, W, H, D, block, dtype):
    g = gen(B + W + block)
    M = (3 * block + W) // block + 1
    cache = random_cache(api, g, B * M + 2, H, block, D)
    pages = torch.randperm(B * M + 2, generator=g, device="cuda")[:B * M].to(torch.int32).view(B, M)
    lengths = torch.randint(0, 2 * block + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lengths[0] = 0
    if B > 2:
        lengths[1] = block
        lengths[2] = block - 1
    counts = torch.randint(0, W + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    fused = (4.0 * torch.randn(B, W, 3 * H + 1, D, generator=g, device="cuda")).to(dtype)   # keys and values inside one buffer
    fused[0, 0, 1] = 0
    for cnt in (None, counts):
        k_new, v_new = fused[:, :, H:2 * H], fused[:, :, 2 * H:3 * H]
        o = plain_append(cache, k_new, v_new, pages, lengths, [W] * B if cnt is None else cnt)
        st = torch.zeros(B, dtype=torch.int32, device="cuda")
        api.cache_append(cache, k_new, v_new, pages, lengths, counts=cnt, status=st)
        for k in ("k", "v", "k_scale", "v_scale"):
            assert same(cache[k], o[k]), k
        assert not st.any()
        fused = fused * 8                                  # the next append makes scales grow


def test_append_extreme_values_and_missing_pages(api):
    g = gen(31)
    cache = random_cache(api, g, 4, 2, 16, 64)
    before = {k: v.clone() for k, v in cache.items()}
    pages = torch.tensor([[0, 9], [1, -1]], device="cuda", dtype=torch.int32)
    lengths = torch.tensor([15, 30], device="cuda", dtype=torch.int32)
    x = torch.randn(2, 4, 2, 64, generator=g, device="cuda")
    x[0, 0, 0, :4] = torch.tensor([INF, -INF, NAN, 3e38], device="cuda")
    x[0, 0, 1] = 1e-42
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    api.cache_append(cache, x, x, pages, lengths, status=st)
    assert st.tolist() == [32, 32]
    ref = dict(before)
    o = plain_append(ref, x[:1], x[:1], pages[:1], [15], [1])   # only the token with a page
    for k in ("k", "v", "k_scale", "v_scale"):
        assert same(cache[k], o[k]), k


def test_append_to_pages_with_negative_scales(api):
    """A page whose scale a caller made negative gets its magnitude, or a larger one, and keeps its values."""
    g = gen(32)
    cache = random_cache(api, g, 2, 2, 32, 64)
    for k in ("k_scale", "v_scale"):
        cache[k].copy_(torch.tensor([[-4.0, -0.25], [-8.0, 2.0]], device="cuda"))
    pages = torch.tensor([[0], [1]], device="cuda", dtype=torch.int32)
    n = torch.tensor([7, 20], device="cuda", dtype=torch.int32)
    was = {k: cache[k].double() * cache[k + "_scale"].double()[:, :, None, None] for k in ("k", "v")}
    x = torch.rand(2, 3, 2, 64, generator=g, device="cuda") + 400.0
    api.cache_append(cache, x, x, pages, n)
    for k in ("k", "v"):
        s = cache[k + "_scale"]
        assert s.tolist() == [[4.0, 1.0], [8.0, 2.0]]
        now = cache[k].double() * s.double()[:, :, None, None]
        for b, m in ((0, 7), (1, 20)):
            old, new = (was[k][b], now[b]) if k == "k" else (was[k][b].transpose(1, 2), now[b].transpose(1, 2))
            # under a scale 4 times as large: half a step of the least codes, 2^-10, or 2^-4 of a value
            tol = torch.maximum(old[:, :m].abs() * 2.0 ** -4, s[b].double()[:, None, None] * 2.0 ** -10)
            tol[s[b] != 1.0] = 0
            assert torch.equal(new[:, :m].isnan(), old[:, :m].isnan())
            assert ((new[:, :m] - old[:, :m]).nan_to_num().abs() <= tol.nan_to_num()).all()
            assert ((new[:, m:m + 3] - x[b].double().transpose(0, 1)).abs() <= 2.0 ** -4 * 401).all()


def test_append_refuses(api):
    from paper_2606_13426_gb300 import binding as B
    c = api.make_token_cache(4, 2, 16, 64)
    x = torch.zeros(1, 2, 2, 64, device="cuda")
    pt = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n = torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        api.cache_append(c, x, x.to(BF16), pt, n)
    with pytest.raises(ValueError):
        api.cache_append(c, x, x, pt, n.long())
    with pytest.raises(ValueError):
        api.cache_append(c, x[..., :32], x[..., :32], pt, n)
    for block, D in ((24, 64), (144, 64), (16, 96)):
        with pytest.raises(B.SDVError):
            y = torch.zeros(1, 2, 2, D, device="cuda")
            api.cache_append(api.make_token_cache(2, 2, block, D), y, y, pt, n)


# ------------------------------------------------------------------------------ attention
def plain_attend(q, cache, pages, lengths, counts, scale, span):
    """Outputs, lse and sum p |v| in 64 bits."""
    B, W, Hq, D = q.shape
    P, H, block, _ = cache["k"].shape
    G = Hq // H
    out = torch.zeros(B, W, Hq, D, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(out)
    lse = torch.full((B, W, Hq), -INF, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, new = int(lengths[b]), min(int(counts[b]), W)
        used = pages[b, : -(-n // block)].long()
        ok = (used >= 0) & (used < P)
        page = used.clamp(0, P - 1)
        for h in range(H):
            k = (cache["k"][page, h].double() * cache["k_scale"][page, h].double()[:, None, None]).reshape(-1, D)[:n]
            v = (cache["v"][page, h].double() * cache["v_scale"][page, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:n]
            there = ok.repeat_interleave(block)[:n]
            for i in range(new):
                end = n - new + i + 1
                lo = max(0, end - span) if span else 0
                if end <= lo:
                    continue
                keep = there[lo:end]
                if not keep.any():
                    continue
                kk, vv = k[lo:end][keep], v[lo:end][keep]
                s = scale * (q[b, i, h * G:(h + 1) * G].double() @ kk.T)
                p = torch.softmax(s, 1)
                out[b, i, h * G:(h + 1) * G] = p @ vv
                mag[b, i, h * G:(h + 1) * G] = p @ vv.abs()
                lse[b, i, h * G:(h + 1) * G] = torch.logsumexp(s, 1)
    return out, lse, mag


def make_cache(api, g, pages, H, block, D):
    """Codes of normal values without NaN, scales that differ between pages and heads."""
    c = api.make_token_cache(pages, H, block, D)
    for k in ("k", "v"):
        c[k].copy_((60 * torch.randn(c[k].shape, generator=g, device="cuda")).clamp(-448, 448).to(torch.float8_e4m3fn))
        c[k + "_scale"].copy_((0.5 + torch.rand(pages, H, generator=g, device="cuda")) / 60)
    return c


def check_attend(api, q, cache, pages, lengths, counts=None, span=0, scale=None, **kw):
    B, W, Hq, D = q.shape
    r = api.cache_attend(q, cache, pages, lengths, counts=counts, span=span, scale=scale, **kw)
    out, lse, mag = plain_attend(q, cache, pages, lengths, [W] * B if counts is None else counts, D ** -0.5 if scale is None else scale, span)
    half = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -11
    tol = 2.0 ** -11 * mag + 1.01 * half * out.abs() + 1e-7
    err = (r["out"].double() - out).abs()
    assert (err <= tol).all(), "output off by %g of its bound" % float((err / tol).max())
    assert near(r["lse"], lse, 2e-5)
    return r


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("W,H,G,D,block,lengths", [
    (1, 1, 1, 64, 16, [1, 2, 15, 16, 17]),
    (1, 2, 8, 128, 64, [63, 64, 65, 0, 1, 500]),
    (9, 2, 4, 128, 64, [9, 10, 700, 64, 73, 0]),
    (5, 1, 7, 64, 48, [5, 47, 48, 49, 1000]),
    (3, 2, 5, 128, 16, [3, 33, 200]),
    (17, 1, 16, 64, 128, [17, 129, 900]),
    (1, 8, 4, 128, 32, [5000]),
    (2, 1, 3, 128, 80, [2, 81, 3001]),
])
def test_attend(api, W, H, G, D, block, lengths, dtype):
    g = gen(W + 3 * H + 5 * G + D + block)
    B = len(lengths)
    M = max(lengths) // block + 2
    cache = make_cache(api, g, B * M + 3, H, block, D)
    pages = torch.randperm(B * M + 3, generator=g, device="cuda")[:B * M].to(torch.int32).view(B, M)
    n = torch.tensor(lengths, device="cuda", dtype=torch.int32)
    fused = torch.randn(B, W, H * G + 2, D, generator=g, device="cuda").to(dtype)
    q = fused[:, :, 1:H * G + 1]
    check_attend(api, q, cache, pages, n)
    counts = torch.randint(0, W + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_attend(api, q, cache, pages, n, counts)
    check_attend(api, 3 * q, cache, pages, n, counts, span=20, scale=0.2)
    check_attend(api, q, cache, pages, n, span=1)


def test_attend_ignores_what_is_not_seen(api):
    """NaN codes behind the sequences' ends, in tokens of the window that earlier queries do not see and
    before the span; table entries of no page behind the tokens; what is seen shows."""
    g = gen(41)
    B, W, H, G, D, block = 2, 4, 1, 2, 64, 16
    cache = make_cache(api, g, 40, H, block, D)
    pages = torch.randperm(40, generator=g, device="cuda")[:24].to(torch.int32).view(2, 12)
    n = torch.tensor([100, 164], device="cuda", dtype=torch.int32)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
    ref = api.cache_attend(q, cache, pages, n, span=50)
    k, v = (cache[x].view(torch.uint8) for x in ("k", "v"))

    def poison(b, i):
        k[int(pages[b, i // block]), 0, i % block] = 0x7f
        v[int(pages[b, i // block]), 0, :, i % block] = 0xff
    for i in list(range(0, 47)) + list(range(100, 112)):
        poison(0, i)
    for i in range(0, 111):
        poison(1, i)
    pages[0, 7:] = -5
    pages[1, 11:] = 1 << 30
    got = api.cache_attend(q, cache, pages, n, span=50)
    assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    poison(0, 98)                                          # seen by the window's last two queries
    got = api.cache_attend(q, cache, pages, n, span=50)
    assert got["out"][0, 2:].isnan().all() and torch.equal(got["out"][0, :2], ref["out"][0, :2])
    assert torch.equal(got["out"][1], ref["out"][1])


def test_attend_missing_pages_and_zero_scales(api):
    g = gen(43)
    cache = make_cache(api, g, 40, 2, 16, 128)
    pages = torch.randperm(40, generator=g, device="cuda")[:30].to(torch.int32).view(3, 10)
    pages[0, 2] = -1
    pages[1, :] = 40
    cache["v_scale"][pages[2, :5].long()] = 0
    cache["k_scale"][pages[2, 5].long()] = 0
    n = torch.tensor([150, 40, 131], device="cuda", dtype=torch.int32)
    q = torch.randn(3, 2, 4, 128, generator=g, device="cuda").to(F16)
    st = torch.zeros(3, dtype=torch.int32, device="cuda")
    check_attend(api, q, cache, pages, n, status=st)
    assert st.tolist() == [32, 32, 0]


def test_attend_f16_outputs_are_rounded_once(api):
    """What is beside an f16 output's own rounding: scores to 2^-22 of the sum of their products' magnitudes (about 7 here, so that
    exponentials are off by 2^-17 at most, with a margin of 8), and probabilities of 22 bits."""
    g = gen(53)
    for W, G, D, m in ((1, 4, 128, 900), (9, 4, 128, 700), (5, 7, 64, 3000), (17, 1, 64, 65)):
        cache = make_cache(api, g, 200, 2, 32, D)
        pages = torch.randperm(200, generator=g, device="cuda").to(torch.int32).view(2, 100)
        n = torch.tensor([m, m // 2], device="cuda", dtype=torch.int32)
        q = torch.randn(2, W, 2 * G, D, generator=g, device="cuda").to(F16)
        out, lse, mag = plain_attend(q, cache, pages, n, [W, W], D ** -0.5, 0)
        got = api.cache_attend(q, cache, pages, n)["out"].double()
        assert ((got - out).abs() <= 2.0 ** -14 * mag + 1.01 * 2.0 ** -11 * out.abs() + 1e-7).all()


def test_attend_extreme_value_scales(api):
    """Keys and values of zeros as they are appended (the least scale), then some that are not zero; scales near both
    ends of fp32."""
    g = gen(49)
    cache = api.make_token_cache(6, 2, 32, 64)
    pages = torch.arange(6, device="cuda", dtype=torch.int32).view(2, 3)
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    zero = torch.zeros(2, 40, 2, 64, device="cuda")
    api.cache_append(cache, zero, zero, pages, none)
    n = none + 40
    q = torch.randn(2, 3, 4, 64, generator=g, device="cuda").to(BF16)
    r = api.cache_attend(q, cache, pages, n)
    assert not r["out"].any() and near(r["lse"], torch.log(torch.tensor([38.0, 39.0, 40.0], device="cuda", dtype=torch.float64))
                                       .view(1, 3, 1).expand(2, 3, 4), 2e-5)
    x = torch.randn(2, 30, 2, 64, generator=g, device="cuda")
    api.cache_append(cache, x, x, pages, n)
    check_attend(api, q, cache, pages, n + 30)
    for size in (2.0 ** -126, 2.0 ** -110, 2.0 ** 100, 1e38 / 448):
        c = make_cache(api, g, 6, 2, 32, 64)
        c["v_scale"].fill_(size)
        out, _, mag = plain_attend(q, c, pages, n, [3, 3], 0.125, 0)
        got = api.cache_attend(q, c, pages, n)["out"].double()
        # bf16's least step, 2^-133, twice (the result's rounding, and a sum's of fp32 results below 2^-126)
        assert ((got - out).abs() <= 2.0 ** -11 * mag + 1.01 * 2.0 ** -8 * out.abs() + 2.0 ** -132).all(), size
    c["v_scale"].copy_(torch.tensor([2.0 ** -126, 1.0, 2.0 ** 100], device="cuda").repeat(2)[:, None].expand(6, 2))
    out, _, mag = plain_attend(q, c, pages, n + 50, [3, 3], 0.125, 0)
    got = api.cache_attend(q, c, pages, n + 50)["out"].double()
    assert ((got - out).abs() <= 2.0 ** -11 * mag + 1.01 * 2.0 ** -8 * out.abs()).all()


def test_attend_rows_past_the_window_do_not_matter(api):
    """Queries i >= counts[b] may hold anything: large numbers there leave the others' results alone."""
    g = gen(50)
    cache = make_cache(api, g, 20, 2, 32, 128)
    pages = torch.arange(20, device="cuda", dtype=torch.int32).view(2, 10)
    n = torch.tensor([300, 77], device="cuda", dtype=torch.int32)
    counts = torch.tensor([2, 3], device="cuda", dtype=torch.int32)
    q = torch.randn(2, 4, 6, 128, generator=g, device="cuda").to(BF16)
    ref = check_attend(api, q, cache, pages, n, counts)
    for x in (1e30, 3e38, INF, NAN):
        q[0, 2:] = x
        q[1, 3:] = -x
        r = api.cache_attend(q, cache, pages, n, counts=counts)
        assert torch.equal(r["out"], ref["out"]) and torch.equal(r["lse"], ref["lse"])


def test_attend_spans_as_long_as_the_cache(api):
    """Spans of the cache's length and more, up to the largest int, see everything; with fewer tokens than queries too."""
    g = gen(51)
    cache = make_cache(api, g, 20, 2, 16, 64)
    pages = torch.arange(20, device="cuda", dtype=torch.int32).view(4, 5)
    n = torch.tensor([80, 4, 1, 33], device="cuda", dtype=torch.int32)
    q = torch.randn(4, 9, 2, 64, generator=g, device="cuda").to(BF16)
    ref = check_attend(api, q, cache, pages, n)
    for span in (80, 81, (1 << 31) - 1):
        r = check_attend(api, q, cache, pages, n, span=span)
        assert torch.equal(r["out"], ref["out"]) and torch.equal(r["lse"], ref["lse"])
    check_attend(api, q, cache, pages, n, span=79)


def test_attend_large_and_tiny_queries(api):
    """bf16 queries outside f16's range, scores far apart, values of very different scales."""
    g = gen(44)
    cache = make_cache(api, g, 30, 1, 32, 64)
    cache["v_scale"] *= 10.0 ** torch.linspace(-6, 6, 30, device="cuda")[:, None]
    pages = torch.randperm(30, generator=g, device="cuda").to(torch.int32).view(1, 30)
    n = torch.tensor([900], device="cuda", dtype=torch.int32)
    q = torch.randn(1, 3, 2, 64, generator=g, device="cuda")
    for size in (1e-30, 1.0, 1e6, 1e30):
        check_attend(api, (q * size).to(BF16), cache, pages, n, scale=0.1 / size)
    check_attend(api, (q * 40).to(BF16), cache, pages, n, scale=1.0)
    check_attend(api, (q * 0).to(BF16), cache, pages, n)


def test_attend_over_long_caches_and_many_sequences(api):
    g = gen(45)
    cache = make_cache(api, g, 1300, 2, 64, 64)
    pages = torch.randperm(1300, generator=g, device="cuda").to(torch.int32).view(1, 1300)
    q = torch.randn(1, 2, 8, 64, generator=g, device="cuda").to(BF16)
    check_attend(api, q, cache, pages, torch.tensor([83000], device="cuda", dtype=torch.int32))
    B = 700
    cache = make_cache(api, g, B * 2, 1, 16, 64)
    pages = torch.randperm(B * 2, generator=g, device="cuda").to(torch.int32).view(B, 2)
    n = torch.randint(0, 33, (B,), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn(B, 1, 1, 64, generator=g, device="cuda").to(BF16)
    check_attend(api, q, cache, pages, n)


@pytest.mark.parametrize("B", [256, 257, 3000])
def test_attend_over_batches_with_empty_sequences(api, B):
    """Runs of sequences without tokens or without queries, at the ends too, around the batch size from
    which the steps are added up by a kernel of their own."""
    g = gen(48 + B)
    cache = make_cache(api, g, 2000, 1, 16, 64)
    n = torch.zeros(B, dtype=torch.int32)
    live = torch.randperm(B - 20, generator=torch.Generator().manual_seed(B))[:40] + 10
    n[live] = torch.randint(1, 400, (40,), generator=torch.Generator().manual_seed(B + 1), dtype=torch.int32)
    n = n.cuda()
    counts = (torch.rand(B, generator=g, device="cuda") < 0.8).to(torch.int32)
    pages = torch.randint(0, 2000, (B, 25), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn(B, 1, 2, 64, generator=g, device="cuda").to(BF16)
    check_attend(api, q, cache, pages, n)
    check_attend(api, q, cache, pages, n, counts)
    check_attend(api, q, cache, pages, torch.zeros_like(n))
    n[0] = n[B - 1] = 333
    check_attend(api, q, cache, pages, n)


def test_cache_offsets_past_32_bits(api):
    """Pages behind the first 2^32 bytes of codes."""
    H, block, D = 4, 64, 128
    P = (1 << 32) // (H * block * D) + 40
    g = gen(46)
    cache = api.make_token_cache(P, H, block, D)
    pages = torch.arange(P - 8, P, device="cuda", dtype=torch.int32).view(2, 4)
    lengths = torch.zeros(2, device="cuda", dtype=torch.int32)
    k = torch.randn(2, 200, H, D, generator=g, device="cuda")
    api.cache_append(cache, k, k.flip(1), pages, lengths)
    n = torch.full((2,), 200, device="cuda", dtype=torch.int32)
    q = torch.randn(2, 2, H, D, generator=g, device="cuda").to(BF16)
    assert not cache["k"][: P - 8].view(torch.uint8)[-64:].any()
    check_attend(api, q, cache, pages, n)


def test_operators_on_another_stream_and_in_a_graph(api):
    g = gen(51)
    tl, dl, tok, coins, race = make_verify(g, 3, 4, 3000, BF16)
    cache = make_cache(api, g, 40, 2, 16, 64)
    pages = torch.arange(36, device="cuda", dtype=torch.int32).view(3, 12)
    n = torch.tensor([100, 64, 150], device="cuda", dtype=torch.int32)
    q = torch.randn(3, 4, 4, 64, generator=g, device="cuda").to(BF16)
    kv = torch.randn(3, 4, 2, 64, generator=g, device="cuda").to(BF16)

    def step():
        api.cache_append(cache, kv, kv, pages, n - 4)
        a = api.cache_attend(q, cache, pages, n)
        s = api.token_scores(tl.view(-1, 3000), top_k=5)
        t = api.token_scores_train(tl.view(-1, 3000), None, None, torch.ones(15, device="cuda"))
        v = api.token_verify(tl, dl, tok, 5)
        return [a["out"], a["lse"], s["top_ids"], s["entropy"], t["d_logits"], v["next_token"], v["accepted_len"]]
    ref = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_attend_refuses(api):
    from paper_2606_13426_gb300 import binding as B
    c = api.make_token_cache(4, 2, 16, 64)
    pt = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, 4, 64, device="cuda")
    with pytest.raises(B.SDVError):
        api.cache_attend(q, c, pt, n)                       # fp32 queries
    with pytest.raises(B.SDVError):
        api.cache_attend(q[:, :, :3].to(BF16), c, pt, n)    # 3 query heads on 2
    with pytest.raises(B.SDVError):
        api.cache_attend(q.to(BF16), c, pt, n, span=-1)
    with pytest.raises(B.SDVError):
        api.cache_attend(q.to(BF16), c, pt, n, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        api.cache_attend(q.to(BF16), c, pt.long(), n)
    with pytest.raises(ValueError):
        api.cache_attend(q.to(BF16), dict(c, v=c["k"]), pt, n)


def test_attend_scales_of_any_sign_and_lengths_past_the_table(api):
    g = gen(61)
    cache = make_cache(api, g, 60, 2, 16, 64)
    for k in ("k_scale", "v_scale"):
        cache[k] *= torch.where(torch.rand(60, 2, generator=g, device="cuda") < 0.4, -1.0, 1.0)
    pages = torch.randperm(60, generator=g, device="cuda")[:40].to(torch.int32).view(2, 20)
    n = torch.tensor([300, 177], device="cuda", dtype=torch.int32)
    q = torch.randn(2, 3, 6, 64, generator=g, device="cuda").to(BF16)
    ref = check_attend(api, q, cache, pages, n)
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    full = torch.tensor([320, 177], device="cuda", dtype=torch.int32)
    a = check_attend(api, q, cache, pages, full, status=st)
    assert st.tolist() == [0, 0]
    b = api.cache_attend(q, cache, pages, torch.tensor([5000, 177], device="cuda", dtype=torch.int32), status=st)
    assert st.tolist() == [32, 0] and torch.equal(a["out"], b["out"])
    # a scale that is no number shows in the rows that see its page, and in no others
    spare = torch.tensor([p for p in range(60) if p not in pages.flatten().tolist()], device="cuda")
    cache["v_scale"][spare] = NAN
    cache["k_scale"][spare] = INF
    assert torch.equal(api.cache_attend(q, cache, pages, n)["out"], ref["out"])
    cache["v_scale"][int(pages[0, 3]), 1] = INF
    cache["k_scale"][int(pages[1, 4]), 0] = NAN
    r = api.cache_attend(q, cache, pages, n)["out"].float()
    assert r[0, :, 3:].isnan().all() and torch.equal(r[0, :, :3], ref["out"][0, :, :3].float())
    assert r[1, :, :3].isnan().all() and torch.equal(r[1, :, 3:], ref["out"][1, :, 3:].float())
    # the last page of the window: its first query sees tokens before that page alone
    n = torch.tensor([290, 177], device="cuda", dtype=torch.int32)          # queries at 287, 288, 289
    ref = api.cache_attend(q, cache, pages[:, :], n)["out"]
    cache["v_scale"][int(pages[0, 18]), 0] = NAN                              # tokens 288 .. 303
    r = api.cache_attend(q, cache, pages, n)["out"]
    assert torch.equal(r[0, 0, :3], ref[0, 0, :3]) and r[0, 1:, :3].float().isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_a_few_whole_sizes(api, dtype):
    """Row sizes at which the rows' split over threads and clusters changes."""
    g = gen(71)
    for N, V in ((1, 8192 * 2), (5, 32768), (3, 32768 + 8), (2, 65536 * 2), (900, 4096), (400, 20000)):
        x = make_logits(g, N, V, dtype, special=False)
        tok = make_tokens(g, N, V)
        gl, gh = torch.randn(N, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
        t = api.token_scores_train(x, tok, gl, gh)
        o = plain_scores(x, tok, 1.0, 0)
        assert grad_ok(t["d_logits"], x, tok, o, gl, gh, 1.0)
        assert near(t["logprob"], o["logprob"], 1e-5) and near(t["entropy"], o["entropy"], 2e-5)


def test_host_tensors_are_refused_wherever_a_kernel_would_read_them(api):
    g = gen(34)
    cache = api.make_token_cache(4, 2, 16, 64)
    pt = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n = torch.full((1,), 2, dtype=torch.int32, device="cuda")
    x = torch.randn(1, 2, 2, 64, generator=g, device="cuda")
    for kv in ((x, x.cpu()), (x.cpu(), x), (x.cpu(), x.cpu())):
        with pytest.raises(ValueError):
            api.cache_append(cache, *kv, pt, n)
    host = torch.zeros(1 << 22, dtype=torch.uint8)
    with pytest.raises(ValueError):
        api.cache_attend(x.to(BF16), cache, pt, n, workspace=host)
    with pytest.raises(ValueError):
        api.cache_attend(x.to(BF16), cache, pt, n, workspace=host.cuda()[::2])
    tl, dl, tok, coins, race = make_verify(g, 2, 3, 50, F32)
    with pytest.raises(ValueError):
        api.token_verify(tl, dl, tok, workspace=host)
    for kw in (dict(coins=coins.cpu()), dict(race=race.cpu()), dict(L_eff=torch.ones(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            api.token_verify(tl, dl, tok, **kw)
    with pytest.raises(ValueError):
        api.token_verify(tl, dl.cpu(), tok)
    with pytest.raises(ValueError):
        api.token_verify(tl, dl, tok.cpu())
    for name in cache:
        with pytest.raises(ValueError):
            api.cache_attend(x.to(BF16), dict(cache, **{name: cache[name].cpu()}), pt, n)
    one = torch.ones(2, device="cuda")
    with pytest.raises(ValueError):
        api.token_scores_train(tl[:, 0], None, None, one, d_logits=tl[:, 0].cpu())
    with pytest.raises(ValueError):
        api.token_scores(tl[:, 0], out=dict(entropy=torch.zeros(2)))


@pytest.mark.parametrize("B,W,H", [(1, 1, 1), (1, 3, 2), (2, 1, 2), (3, 4, 1), (1, 1, 2)])
def test_append_takes_any_stride_of_an_axis_of_one_place(api, B, W, H):
    """Keys and values whose strides differ only where there is one sequence, one token or one head."""
    g = gen(33)
    caches = [api.make_token_cache(2 * B, H, 16, 64) for _ in range(2)]
    pages = torch.arange(2 * B, device="cuda", dtype=torch.int32).view(B, 2)
    n = torch.arange(B, device="cuda", dtype=torch.int32) * 7 + 5
    x, y = (torch.randn(B, W, H, 64, generator=g, device="cuda") for _ in range(2))
    api.cache_append(caches[0], x, y, pages, n)
    sizes, strides = list(y.shape), list(y.stride())
    for i in range(3):
        if sizes[i] == 1:
            strides[i] = 12345
    z = y.as_strided(sizes, strides)
    assert torch.equal(z, y) and z.stride() != y.stride()
    api.cache_append(caches[1], x, z, pages, n)
    assert all(torch.equal(caches[0][k].view(torch.uint8), caches[1][k].view(torch.uint8)) for k in caches[0])
    for other in [y[..., :32]] + ([torch.zeros(B, W, H, 72, device="cuda")[..., :64]] if B * W * H > 1 else []):
        with pytest.raises(ValueError):
            api.cache_append(caches[0], x, other, pages, n)


@pytest.mark.parametrize("B,L,V,dtype,T", [(4, 4, 32768, BF16, 1.0), (3, 8, 131072, F16, 1.0), (40, 6, 50001, BF16, 1.0), (200, 3, 70, BF16, 1.0),
                                           (8, 5, 32768, BF16, 0.8), (8, 5, 40001, F32, 1.3)])
def test_log_ratios_to_the_last_bits(api, B, L, V, dtype, T):
    """Log ratios beside the 64-bit ones.  Differences to the maximum are exact for 16-bit logits (to half a step of 2^-20 in 8 .. 16
    for fp32 ones, and so are quotients by a temperature: 2^-21 each); the sums' ratio is within 2^-22, its logarithm and the
    additions within half a step of the result."""
    tl, dl, tok, coins, race = make_verify(gen(B + V), B, L, V, dtype, T)
    r = api.token_verify(tl, dl, tok, coins=coins, race=race, temperature=T)
    q, p = (torch.log_softmax(x.double() / T, 2) for x in (tl[:, :L], dl))
    want = (q - p).gather(2, tok[..., None].long())[..., 0]
    steps = 0 if T == 1.0 and dtype != F32 else 4 * 2.0 ** -21
    err = (r["log_ratio"].double() - want).abs()
    assert (err <= 2.0 ** -21 + steps + 2.0 ** -22 * want.abs()).all(), float((err / (2.0 ** -21 + steps + 2.0 ** -22 * want.abs())).max())
