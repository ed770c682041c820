"""The attention of drafted trees over the 8-bit cache against its definition in 64 bits, row by row.

Tolerances, with u = 2^-24: a score is a sum of D products in fp32, in an order of the matrix unit's own and with its
truncations: within E = (2 D + 8) u of the sum of its products' magnitudes (the largest of a row's is
taken).  Its exponential adds 2^-20 (the argument's rounding below 2^3, ex2's 2^-22), the probability's two
halves 2^-16, sums over a step's 128 keys and over the steps (128 + n / 32) u.  An output is then within
2 (E + 2^-15 + (128 + n / 32) u) sum p |v| of the exact one, and half a unit of its type; lse within
E + 2^-19 + (128 + n / 32) u and 4 u of its own size.
"""
import random

import pytest
import torch

from test_gpu_tokens import BF16, F16, INF, NAN, api, gen, make_cache  # noqa: F401

pytestmark = pytest.mark.gpu

HALF = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
LEAST = {BF16: 2.0 ** -132, F16: 2.0 ** -25}


def tree_of(kind, W, seed=0):
    """Parents of a tree of W nodes."""
    rng = random.Random(seed + W)
    if kind == "chain":
        return list(range(-1, W - 1))
    if kind == "star":
        return [-1] + [0] * (W - 1)
    if kind == "roots":
        return [-1] * W
    if kind == "forest":                                # several roots, any parent before its child
        return [-1] + [rng.randint(-1, i - 1) for i in range(1, W)]
    return [-1] + [rng.randint(max(0, i - 6), i - 1) for i in range(1, W)]


def plain_tree(q, cache, pages, lengths, counts, parents, scale):
    """out, lse, sum p |v| and the largest sum of magnitudes under a score, in 64 bits."""
    B, W, Hq, D = q.shape
    P, H, block = cache["k"].shape[:3]
    G = Hq // H
    out = torch.zeros(B, W, Hq, D, dtype=torch.float64, device="cuda")
    mag, most = torch.zeros_like(out), torch.zeros(B, W, Hq, dtype=torch.float64, device="cuda")
    lse = torch.full((B, W, Hq), -INF, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, new = max(0, min(int(lengths[b]), pages.shape[1] * block)), max(0, min(int(counts[b]), W))
        if n < new or not new:
            continue
        used = pages[b, : -(-n // block)].long()
        there = ((used >= 0) & (used < P)).repeat_interleave(block)[:n]
        page = used.clamp(0, P - 1)
        seen = torch.zeros(new, n, dtype=torch.bool)
        seen[:, :n - new] = True
        for i in range(new):
            u = i
            while u >= 0:
                seen[i, n - new + u] = True
                p = int(parents[b][u])
                u = p if 0 <= p < u else -1
        seen = seen.cuda() & there
        for h in range(H):
            k = (cache["k"][page, h].double() * cache["k_scale"][page, h].double()[:, None, None]).reshape(-1, D)[:n]
            v = (cache["v"][page, h].double() * cache["v_scale"][page, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:n]
            for i in range(new):
                if not seen[i].any():
                    continue
                kk, vv = k[seen[i]], v[seen[i]]
                rows = q[b, i, h * G:(h + 1) * G].double()
                s = scale * (rows @ kk.T)
                p = torch.softmax(s, 1)
                out[b, i, h * G:(h + 1) * G] = p @ vv
                mag[b, i, h * G:(h + 1) * G] = p @ vv.abs()
                most[b, i, h * G:(h + 1) * G] = abs(scale) * (rows.abs() @ kk.abs().T).nan_to_num(0.0).amax(1)
                lse[b, i, h * G:(h + 1) * G] = torch.logsumexp(s, 1)
    return out, lse, mag, most


def widened(pages, tokens=200_000):
    """The page table in a much wider one: calls are laid out for the tokens that it could hold, so that the kernels for many
    rows and long sequences run on these."""
    more = torch.full((pages.shape[0], tokens // 16), -1, dtype=torch.int32, device="cuda")
    return torch.cat([pages, more], 1)


def check_tree(api, q, cache, pages, lengths, parents, counts=None, scale=None, **kw):
    """Both ways: as the table is, and in a wide one."""
    check_tree_as(api, q, cache, widened(pages), lengths, parents, counts, scale, **kw)
    return check_tree_as(api, q, cache, pages, lengths, parents, counts, scale, **kw)


def check_tree_as(api, q, cache, pages, lengths, parents, counts=None, scale=None, **kw):
    B, W, Hq, D = q.shape
    par = torch.as_tensor(parents, dtype=torch.int32, device="cuda").view(-1, W).expand(B, W).contiguous()
    r = api.tree_attend(q, cache, pages, lengths, par, counts=counts, scale=scale, **kw)
    cnt = [W] * B if counts is None else counts.tolist()
    out, lse, mag, most = plain_tree(q, cache, pages, lengths, cnt, par.tolist(), D ** -0.5 if scale is None else scale)
    n = float(lengths.max())
    sums = (128 + n / 32) * 2.0 ** -24
    E = (2 * D + 8) * 2.0 ** -24 * most
    got = r["out"].double()
    assert torch.equal(got.isnan(), out.isnan())
    tol = 2 * (E[..., None] + 2.0 ** -15 + sums) * mag + 1.01 * HALF[q.dtype] * out.abs() + LEAST[q.dtype]
    err = (got - out).abs().nan_to_num(0.0)
    assert (err <= tol.nan_to_num(INF)).all(), "output off by %g of its bound" % float((err / tol).nan_to_num(0.0).max())
    le = r["lse"].double()
    assert torch.equal(le.isnan(), lse.isnan()) and torch.equal(le == -INF, lse == -INF)
    err = (le - lse).abs().nan_to_num(0.0)
    assert (err <= (E + 2.0 ** -19 + sums + 2.0 ** -22 * lse.abs()).nan_to_num(INF)).all(), "lse off by %g" % float(err.max())
    return r


CASES = [                                               # W, H, G, D, block, lengths
    (1, 1, 1, 64, 16, [1, 2, 15, 16, 17]),
    (1, 2, 8, 128, 64, [63, 64, 65, 0, 1, 500]),
    (9, 2, 4, 128, 64, [9, 10, 700, 64, 73, 8, 0]),
    (5, 1, 7, 64, 48, [5, 47, 48, 49, 1000]),
    (16, 2, 5, 128, 16, [16, 33, 200, 129, 144]),
    (17, 1, 16, 64, 128, [17, 129, 900, 127, 128]),
    (33, 2, 4, 128, 64, [33, 160, 1300]),
    (64, 1, 1, 64, 80, [64, 65, 63, 3001]),
    (64, 2, 8, 128, 32, [64, 96, 2500]),
    (24, 8, 4, 128, 32, [5000]),
    (60, 1, 3, 128, 112, [61, 1201, 255, 256, 257]),
]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("W,H,G,D,block,lengths", CASES)
def test_tree_attend(api, W, H, G, D, block, lengths, dtype):
    g = gen(7 * W + 3 * H + 5 * G + D + block)
    B = len(lengths)
    M = max(lengths) // block + 2
    cache = make_cache(api, g, B * M + 3, H, block, D)
    pages = torch.randperm(B * M + 3, generator=g, device="cuda")[:B * M].to(torch.int32).view(B, M)
    n = torch.tensor(lengths, device="cuda", dtype=torch.int32)
    fused = torch.randn(B, W, H * G + 2, D, generator=g, device="cuda").to(dtype)
    q = fused[:, :, 1:H * G + 1]                        # rows of a larger buffer
    for kind in ("tree", "chain", "star", "forest"):
        check_tree(api, q, cache, pages, n, [tree_of(kind, W, b) for b in range(B)])
    counts = torch.randint(0, W + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_tree(api, q, cache, pages, n, tree_of("tree", W), counts)
    check_tree(api, 3 * q, cache, pages, n, tree_of("roots", W), counts, scale=-0.2)
    odd = torch.randn(B, W, H * G, D + 1, generator=g, device="cuda").to(dtype)[..., 1:]
    check_tree(api, odd, cache, pages, n, tree_of("tree", W))   # rows on no 16-byte boundary


def test_a_chain_is_a_window(api):
    """A tree of one path gives what cache_attend gives for the window."""
    g = gen(5)
    for D, W in ((64, 7), (128, 33)):
        cache = make_cache(api, g, 60, 2, 32, D)
        pages = torch.randperm(60, generator=g, device="cuda").to(torch.int32).view(3, 20)
        n = torch.tensor([600, 64, 333], device="cuda", dtype=torch.int32)
        q = torch.randn(3, W, 8, D, generator=g, device="cuda").to(BF16)
        par = torch.arange(-1, W - 1, device="cuda", dtype=torch.int32).expand(3, W).contiguous()
        b = api.cache_attend(q, cache, pages, n)
        for table in (pages, widened(pages)):
            a = api.tree_attend(q, cache, table, n, par)
            x, y = a["out"].double(), b["out"].double()
            assert ((x - y).abs() <= 2 * HALF[BF16] * y.abs() + 2.0 ** -12 * y.abs().amax()).all()
            assert ((a["lse"] - b["lse"]).abs() <= 3e-5 * (1 + b["lse"].abs())).all()


@pytest.mark.parametrize("W,G", [(6, 2), (48, 4)])
def test_what_is_no_tree_is_told(api, W, G):
    from paper_2606_13426_gb300 import binding as B
    g = gen(11)
    cache = make_cache(api, g, 24, 2, 16, 64)
    pages = torch.randperm(24, generator=g, device="cuda").to(torch.int32).view(4, 6)
    n = torch.tensor([80, W, W - 1, 96], device="cuda", dtype=torch.int32)
    q = torch.randn(4, W, 2 * G, 64, generator=g, device="cuda").to(BF16)
    par = [tree_of("tree", W) for _ in range(4)]
    par[0][4] = 4                                       # its own parent; one behind it; one below -1
    par[0][3] = W + 3
    par[1][2] = -7
    status = torch.zeros(4, device="cuda", dtype=torch.int32)
    check_tree(api, q, cache, pages, n, par, status=status)
    assert status.tolist() == [B.SDV_STATUS_BAD_TREE] * 3 + [0]
    # behind the nodes in use anything may stand
    counts = torch.tensor([3, 2, 4, W], device="cuda", dtype=torch.int32)
    status.zero_()
    check_tree(api, q, cache, pages, n, par, counts, status=status)
    assert status.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("W,G", [(5, 1), (40, 4)])
def test_nodes_that_are_not_seen_do_not_matter(api, W, G, wide):
    """NaN codes of a sibling's branch and behind the sequence, pages that do not exist."""
    from paper_2606_13426_gb300 import binding as B
    g = gen(12)
    block, D = 16, 128
    cache = make_cache(api, g, 20, 1, block, D)
    pages = torch.arange(20, device="cuda", dtype=torch.int32).view(2, 10)
    pages = widened(pages) if wide else pages
    n = torch.tensor([100, 64], device="cuda", dtype=torch.int32)
    q = torch.randn(2, W, G, D, generator=g, device="cuda").to(BF16)
    par = tree_of("star", W)
    before = check_tree_as(api, q, cache, pages, n, par)
    k8, v8 = cache["k"].view(torch.uint8), cache["v"].view(torch.uint8)
    for b in range(2):                                  # everything behind the sequence's end
        last = int(n[b])
        for t in range(last, 10 * block):
            k8[pages[b, t // block].long(), 0, t % block] = 0x7f
            v8[pages[b, t // block].long(), 0, :, t % block] = 0xff
    after = check_tree_as(api, q, cache, pages, n, par)
    assert torch.equal(before["out"], after["out"]) and torch.equal(before["lse"], after["lse"])
    # a NaN code in one leaf's key and another one's value: those two rows alone
    at = [100 - W + 2, 100 - W + 3]
    k8[pages[0, at[0] // block].long(), 0, at[0] % block, 5] = 0xff
    v8[pages[0, at[1] // block].long(), 0, 7, at[1] % block] = 0x7f
    r = check_nan(api, q, cache, pages, n, par, {(0, 2), (0, 3)})
    live = torch.ones(2, W, dtype=torch.bool, device="cuda")
    live[0, 2:4] = False
    assert torch.equal(r["out"][live], after["out"][live])
    # in the context: every row of that sequence
    v8[pages[1, 0].long(), 0, 3, 2] = 0x7f
    check_nan(api, q, cache, pages, n, par, {(0, 2), (0, 3)} | {(1, i) for i in range(W)})
    # pages that do not exist
    pages[1, 1], pages[0, 2] = 99, -1
    status = torch.zeros(2, device="cuda", dtype=torch.int32)
    k8[pages[1, 0].long()] = 0
    v8[pages[1, 0].long()] = 0
    r = api.tree_attend(q, cache, pages, n, torch.tensor([par, par], device="cuda", dtype=torch.int32), status=status)
    assert (status & B.SDV_STATUS_BAD_PAGE).bool().all()
    v8[pages[0, at[1] // block].long(), 0, 7, at[1] % block] = 0
    k8[pages[0, at[0] // block].long(), 0, at[0] % block, 5] = 0
    check_tree_as(api, q, cache, pages, n, par)


def check_nan(api, q, cache, pages, n, par, rows):
    """All of the rows that see a NaN code are NaN, the others as they are without."""
    W = q.shape[1]
    r = api.tree_attend(q, cache, pages, n, torch.tensor([par] * q.shape[0], device="cuda", dtype=torch.int32))
    want = torch.zeros(q.shape[0], W, dtype=torch.bool)
    for b, i in rows:
        want[b, i] = True
    want = want.cuda()
    assert torch.equal(r["out"].isnan().all(-1).all(-1), want) and torch.equal(r["out"].isnan().any(-1).any(-1), want)
    assert torch.equal(r["lse"].isnan().all(-1), want)
    return r


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("W,G", [(4, 2), (40, 4)])
def test_extreme_scales_queries_and_scores(api, W, G, dtype, wide):
    """Value scales far apart, of either sign and zero; key scales that make sharp rows and scores past 2^24; queries of very
    different size; NaN and infinite queries, which are their own rows' affair."""
    g = gen(21)
    B, H, block, D, M = 2, 2, 32, 64, 40
    cache = make_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    pages = widened(pages) if wide else pages
    n = torch.tensor([M * block - 7, 300], device="cuda", dtype=torch.int32)
    par = tree_of("tree", W)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(dtype)
    for k in (10, 40, 80) if dtype == BF16 else (6, 10):
        c = {a: t.clone() for a, t in cache.items()}
        c["v_scale"] *= torch.exp2(torch.floor(k * (torch.rand(B * M, H, generator=g, device="cuda") - 0.5)))
        c["v_scale"][::5] *= -1
        c["v_scale"][3::11] = 0
        c["k_scale"][1::4] *= -1
        c["k_scale"][2::9] = 0
        for sharp in (1.0, 8.0):
            check_tree_as(api, (sharp * q).to(dtype), c, pages, n, par)
    big = {a: t.clone() for a, t in cache.items()}
    big["k_scale"] *= 2.0 ** 30
    r = api.tree_attend(q, big, pages, n, torch.tensor([par] * B, device="cuda", dtype=torch.int32))
    out, lse, _, _ = plain_tree(q, big, pages, n, [W] * B, [par] * B, D ** -0.5)
    assert r["out"].isfinite().all() and ((r["lse"].double() - lse).abs() <= 2.0 ** -16 * lse.abs()).all()
    sizes = torch.exp2(torch.randint(-20, 5, (B, W, H * G, 1), generator=g, device="cuda").float()) if dtype == BF16 else 1.0
    check_tree_as(api, (q.float() * sizes).to(dtype), cache, pages, n, par)
    bad = q.clone()
    bad[0, 1, 0, 3] = NAN
    bad[1, 2, 1, 0] = INF
    r = api.tree_attend(bad, cache, pages, n, torch.tensor([par] * B, device="cuda", dtype=torch.int32))
    ref = api.tree_attend(q, cache, pages, n, torch.tensor([par] * B, device="cuda", dtype=torch.int32))
    rows = torch.zeros(B, W, H * G, dtype=torch.bool, device="cuda")
    rows[0, 1, 0] = rows[1, 2, 1] = True
    assert r["out"][rows].isnan().all() and r["lse"][rows].isnan().all()
    x, y = r["out"][~rows].double(), ref["out"][~rows].double()
    assert ((x - y).abs() <= 2 * HALF[dtype] * y.abs() + 2.0 ** -12 * y.abs().amax()).all()


@pytest.mark.parametrize("W,H,G,D", [(1, 2, 4, 128), (12, 1, 8, 64), (32, 2, 4, 128), (64, 1, 5, 64)])
def test_bf16_outputs_are_rounded_once(api, W, H, G, D):
    """An output is the rounding of a number within 2^-13 sum p |v| of the exact one."""
    g = gen(31 + W)
    cache = make_cache(api, g, 100, H, 32, D)
    pages = torch.randperm(100, generator=g, device="cuda").to(torch.int32).view(2, 50)
    n = torch.tensor([1500, 321], device="cuda", dtype=torch.int32)
    par = torch.tensor([tree_of("tree", W)] * 2, device="cuda", dtype=torch.int32)
    for sharp in (1.0, 3.0):
        q = (sharp * torch.randn(2, W, H * G, D, generator=g, device="cuda")).to(BF16)
        out, _, mag, most = plain_tree(q, cache, pages, n, [W, W], par.tolist(), D ** -0.5)
        got = torch.cat([api.tree_attend(q, cache, t, n, par)["out"].double()[None] for t in (pages, widened(pages))])
        tol = (2.0 ** -13 + 2 * (2 * D + 8) * 2.0 ** -24 * most[..., None]) * mag
        low, high = (out - tol).float().to(BF16).double(), (out + tol).float().to(BF16).double()
        assert (low <= got).all() and (got <= high).all()


def test_many_sequences_and_long_caches(api):
    g = gen(41)
    for B, W, H, G, D, block, most in ((300, 6, 2, 2, 64, 16, 90), (520, 20, 1, 8, 64, 16, 70), (2, 40, 2, 4, 128, 128, 40000)):
        M = most // block + 2
        cache = make_cache(api, g, B * M, H, block, D)
        pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
        n = torch.randint(0, most + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        if B > 100:
            n[::7] = 0
            n[3::50] = W
        q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
        check_tree(api, q, cache, pages, n, [tree_of("tree", W, b) for b in range(B)])


def test_offsets_past_32_bits(api):
    H, block, D = 4, 64, 128
    P = (1 << 32) // (H * block * D) + 40
    g = gen(46)
    cache = api.make_token_cache(P, H, block, D)
    pages = torch.arange(P - 8, P, device="cuda", dtype=torch.int32).view(2, 4)
    lengths = torch.zeros(2, device="cuda", dtype=torch.int32)
    k = torch.randn(2, 200, H, D, generator=g, device="cuda")
    api.cache_append(cache, k, k.flip(1), pages, lengths)
    n = torch.full((2,), 200, device="cuda", dtype=torch.int32)
    for W in (2, 40):
        q = torch.randn(2, W, 4 * H, D, generator=g, device="cuda").to(BF16)
        check_tree(api, q, cache, pages, n, tree_of("tree", W))


@pytest.mark.parametrize("B,W,H,G,D,block,most", [(30, 59, 8, 4, 128, 64, 790), (14, 46, 4, 16, 128, 32, 717),
                                                  (107, 52, 4, 4, 128, 64, 624), (60, 33, 8, 8, 64, 16, 400)])
def test_many_short_sequences_time_and_again(api, B, W, H, G, D, block, most):
    """Runs of several short items, whose queries follow one another: every call gives the same, and what 64 bits give."""
    g = gen(B)
    M = -(-most // block)
    cache = make_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    n = torch.randint(W, most + 1, (B,), generator=g, device="cuda").to(torch.int32)
    par = torch.stack([torch.tensor(tree_of("tree", W, b)) for b in range(B)]).to(torch.int32).cuda()
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
    wide = widened(pages)
    calls = [api.tree_attend(q, cache, wide, n, par) for _ in range(40)]
    for r in calls[1:]:
        assert torch.equal(r["out"], calls[0]["out"]) and torch.equal(r["lse"], calls[0]["lse"])
    check_tree_as(api, q, cache, wide, n, [tree_of("tree", W, b) for b in range(B)])


def test_graphs_streams_and_shared_workspaces(api):
    """Captured calls that share a workspace, replayed in turn with lengths that change; another stream; outputs of the
    caller; the same bits each time."""
    from paper_2606_13426_gb300 import binding as B
    g = gen(51)
    cache = make_cache(api, g, 120, 2, 16, 128)
    pages = torch.arange(120, device="cuda", dtype=torch.int32).view(3, 40)
    n = torch.tensor([500, 64, 333], device="cuda", dtype=torch.int32)
    calls = []
    wide = widened(pages)
    for W, G in ((7, 2), (40, 4)):
        q = torch.randn(3, W, 2 * G, 128, generator=g, device="cuda").to(BF16)
        par = torch.tensor([tree_of("tree", W, b) for b in range(3)], device="cuda", dtype=torch.int32)
        calls.append((q, par, pages if W == 7 else wide))
    size = max(B.sdv_tree_attend_workspace_bytes(3, q.shape[1], q.shape[2], 2, 128) for q, _, _ in calls)
    ws = torch.empty(size, device="cuda", dtype=torch.uint8)
    ref = [api.tree_attend(q, cache, t, n, p) for q, p, t in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [api.tree_attend(q, cache, t, n, p) for q, p, t in calls]
    side.synchronize()
    assert all(torch.equal(a[k], b[k]) for a, b in zip(ref, got) for k in ("out", "lse"))
    graphs, outs = [], []
    for q, p, t in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(api.tree_attend(q, cache, t, n, p, workspace=ws))
        graphs.append(graph)
    for lengths in ([500, 64, 333], [64, 639, 41], [0, 40, 600]):
        n.copy_(torch.tensor(lengths, dtype=torch.int32))
        ref = [api.tree_attend(q, cache, t, n, p) for q, p, t in calls]
        for _ in range(2):
            for graph in graphs:
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for a, b in zip(ref, outs) for k in ("out", "lse"))


def test_refusals(api):
    from paper_2606_13426_gb300 import binding as B
    c = api.make_token_cache(4, 2, 16, 64)
    pt = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    par = torch.full((1, 1), -1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, 4, 64, device="cuda")
    with pytest.raises(B.SDVError):
        api.tree_attend(q, c, pt, n, par)                   # fp32 queries
    q = q.to(BF16)
    with pytest.raises(B.SDVError):
        api.tree_attend(q[:, :, :3], c, pt, n, par)         # 3 query heads on 2
    with pytest.raises(ValueError):
        api.tree_attend(q, c, pt, n, par.long())
    with pytest.raises(ValueError):
        api.tree_attend(q, c, pt, n, par.cpu())
    with pytest.raises(ValueError):
        api.tree_attend(q, c, pt, n, par.expand(1, 2).contiguous())
    with pytest.raises(B.SDVError):
        api.tree_attend(q, c, pt, n, par, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(B.SDVError):                         # 65 nodes
        api.tree_attend(q.expand(1, 65, 4, 64).contiguous(), c, pt, n, par.expand(1, 65).contiguous())
