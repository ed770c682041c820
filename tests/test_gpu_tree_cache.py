"""Appending with rotation, and moving kept rows, against plain forms in 64 bits.

Tolerances: a turned element is a product sum of two terms in fp32, its cosine and sine within 2^-22: within 2^-21
(|x_a| + |x_b|) of the exact one; a position's angle adds pos 2^-52.  A code is that number's rounding: half a
step, 2^-4 of it, or 2^-10 of the scale below the normal ones, and what was turned a little off may round the
other way.  A scale may be the next one where the largest magnitude is within 2^-20 of 448 powers of two.
Values, and rows that are moved, are exact.
"""
import math

import pytest
import torch

from test_gpu_tokens import BF16, F16, F32, INF, NAN, api, e4m3, gen, plain_append, random_cache, same  # noqa: F401
from test_gpu_tree_attend import tree_of

pytestmark = pytest.mark.gpu

HALF = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}


def turn(x, pos, freqs, pairs):
    """x [n, heads, D] turned by pos [n] in 64 bits, and each element's |x_a| + |x_b|."""
    x = x.double()
    rot = 2 * freqs.numel()
    t = pos.double()[:, None] * freqs
    c, s = t.cos()[:, None], t.sin()[:, None]
    y, size = x.clone(), x.abs()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if pairs == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def held(cache, pages, b, n, new):
    """Keys and values [new, H, D] that stand behind the first n tokens of sequence b, and their scales [new, H]."""
    block = cache["k"].shape[2]
    at = torch.arange(n, n + new, device="cuda")
    page, row = pages[b].long()[at // block], at % block
    k = cache["k"].view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn).double() * cache["k_scale"][page].double()[..., None]
    v = cache["v"].view(torch.uint8)[page, :, :, row].view(torch.float8_e4m3fn).double() * cache["v_scale"][page].double()[..., None]
    return k, v, cache["k_scale"][page].double()


def check_rotary(api, cache, k, v, pages, lengths, freqs, pairs, q, positions=None, counts=None, out=None):
    B, W = k.shape[:2]
    before = {a: t.clone() for a, t in cache.items()}
    k64, v64, q64 = k.clone(), v.clone(), q.clone()
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    got_q = api.cache_append_rotary(cache, k, v, pages, lengths, freqs, pairs=pairs, q=q, positions=positions, counts=counts, status=status,
                                    out=out)
    new = [W] * B if counts is None else counts.tolist()
    # values, and what neighbours hold: as of the plain append
    ref = plain_append(before, k64, v64, pages, lengths, [min(max(c, 0), W) for c in new])
    assert same(cache["v"].double(), ref["v"]) and same(cache["v_scale"], ref["v_scale"])
    assert not status.any()
    tiny = 2.0 ** -149 if q.dtype != F16 else 2.0 ** -25
    for b in range(B):
        n, c = int(lengths[b]), min(max(new[b], 0), W)
        pos = torch.arange(n, n + W, device="cuda") if positions is None else positions[b]
        assert (got_q[b, c:] == 0).all()
        if not c:
            continue
        off = (pos[:c].abs().double() * 2.0 ** -52 + 2.0 ** -21)[:, None, None]
        y, size = turn(k64[b, :c], pos[:c], freqs, pairs)
        kk, _, s = held(cache, pages, b, n, c)
        tol = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s[..., None]) * 1.001 + off * size
        assert ((kk - y).abs() <= tol).all(), float(((kk - y).abs() / tol).max())
        # the scale is the least that holds the page's new keys, or what the page had
        for page in set(pages[b].long()[torch.arange(n, n + c, device="cuda") // cache["k"].shape[2]].tolist()):
            rows = (pages[b].long()[torch.arange(n, n + c, device="cuda") // cache["k"].shape[2]] == page)
            top = y[rows].abs().amax((0, 2)) / 448
            old = before["k_scale"][page].double() if n % cache["k"].shape[2] and page == int(pages[b, n // cache["k"].shape[2]]) else None
            sc = cache["k_scale"][page].double()
            least = torch.exp2(torch.ceil(torch.log2(top.clamp(min=2.0 ** -126) * (1 - 2.0 ** -20))))
            most = torch.exp2(torch.ceil(torch.log2(top.clamp(min=2.0 ** -126) * (1 + 2.0 ** -20))))
            if old is not None:
                least, most = torch.maximum(least, old), torch.maximum(most, old)
            assert (sc >= least).all() and (sc <= most).all()
        y, size = turn(q64[b, :c], pos[:c], freqs, pairs)
        assert ((got_q[b, :c].double() - y).abs() <= 1.001 * HALF[q.dtype] * y.abs() + off * size + tiny).all()
    # tokens that were there: restated where the scale grew, else untouched
    for b in range(B):
        n = int(lengths[b])
        if n:
            was, now = held(before, pages, b, 0, n), held(cache, pages, b, 0, n)
            grew = now[2] != was[2]
            tol = torch.where(grew[..., None], torch.maximum(2.0 ** -4 * was[0].abs(), 2.0 ** -10 * now[2][..., None]), 0.0)
            assert (((now[0] - was[0]).abs() <= tol) | (was[0].isnan() & now[0].isnan())).all()
    return got_q


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pairs,rots", [("halves", (0, 32, 20, 2)), ("neighbours", (0, 34, 2))])
@pytest.mark.parametrize("B,W,H,G,D,block", [(1, 1, 1, 1, 64, 16), (5, 3, 2, 3, 128, 64), (6, 9, 3, 1, 64, 48), (3, 40, 2, 4, 128, 16),
                                             (2, 300, 2, 2, 64, 128), (2, 130, 1, 8, 128, 128), (1, 700, 8, 1, 128, 64)])
def test_append_rotary(api, B, W, H, G, D, block, pairs, rots, dtype):
    g = gen(B + W + block + len(rots))
    M = (3 * block + W) // block + 1
    for rot in rots:
        rot = rot or D
        cache = api.make_token_cache(B * M, H, block, D)
        pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
        lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
        freqs = api.rotary_freqs(rot)
        rows = 0.7 * torch.randn(B, 2 * block + 3, 2 * H, D, generator=g, device="cuda")
        first = torch.randint(0, 2 * block + 3, (B,), generator=g, device="cuda", dtype=torch.int32)
        api.cache_append(cache, rows[:, :, :H], rows[:, :, H:], pages, lengths, counts=first)
        fused = (torch.randn(B, W, H * (G + 2), D, generator=g, device="cuda") * 2.0 ** torch.randint(-3, 4, (B, W, 1, 1), generator=g, device="cuda")).to(dtype)
        q, k, v = fused[:, :, :H * G], fused[:, :, H * G:H * (G + 1)], fused[:, :, H * (G + 1):]
        counts = torch.randint(0, W + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if rot != D else None
        positions = None
        if W <= 40:
            depth = torch.tensor([[0] + [i // 3 + 1 for i in range(W - 1)]] * B, device="cuda", dtype=torch.int32)
            positions = first[:, None] + depth
        check_rotary(api, cache, k, v, pages, first, freqs, pairs, q, positions, counts)


@pytest.mark.parametrize("D", [64, 128])
def test_append_rotary_of_any_window(api, D):
    """Every window against its tokens one by one: what a CTA holds grows with it."""
    g = gen(D)
    for block in (16, 48, 64, 80, 128):
        k = torch.randn(1, 130, 1, D, generator=g, device="cuda").to(BF16)
        pages = torch.arange(3 + 130 // block, device="cuda", dtype=torch.int32)[None]
        n = torch.zeros(1, dtype=torch.int32, device="cuda")
        freqs = api.rotary_freqs(D)
        for W in list(range(1, 8)) + list(range(52, 131)):
            cache = api.make_token_cache(pages.shape[1], 1, block, D)
            q = api.cache_append_rotary(cache, k[:, :W], k[:, :W], pages, n, freqs, q=k[:, :W])
            c = cache["k"].view(torch.uint8)[:, 0].reshape(-1, D).view(torch.float8_e4m3fn)[:W].double()
            s = cache["k_scale"][:, 0].double().repeat_interleave(block)[:W, None]
            y, size = turn(k[0, :W], torch.arange(W, device="cuda"), freqs, "halves")
            tol = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * s[:, None]) * 1.001 + 2.0 ** -21 * size
            assert ((c * s - y[:, 0]).abs() <= tol[:, 0]).all(), (block, W)
            assert ((q[0].double() - y).abs() <= HALF[BF16] * 1.01 * y.abs() + 2.0 ** -20 * size).all(), (block, W)


def test_positions_far_and_negative(api):
    """Positions up to 2^30, frequencies of a caller's own (zero and negative ones among them)."""
    g = gen(2)
    for pairs in ("halves", "neighbours"):
        cache = api.make_token_cache(4, 2, 16, 64)
        pages = torch.arange(4, device="cuda", dtype=torch.int32).view(2, 2)
        zero = torch.zeros(2, device="cuda", dtype=torch.int32)
        x = torch.randn(2, 5, 8, 64, generator=g, device="cuda")
        positions = torch.tensor([[0, -1, 100_000, 2 ** 30, -2 ** 30], [1, 2, 131_071, 1_000_003, 77]], device="cuda", dtype=torch.int32)
        freqs = torch.randn(32, generator=g, device="cuda", dtype=torch.float64)
        freqs[3], freqs[4], freqs[5] = 0.0, 1e-9, -2.5
        check_rotary(api, cache, x[:, :, :2], x[:, :, 2:4], pages, zero, freqs, pairs, x[:, :, 4:], positions)


def test_no_turn_is_the_plain_append(api):
    """Frequencies of zero: what cache_append writes, bit by bit; queries unchanged."""
    g = gen(4)
    for dtype, D, block in ((BF16, 128, 64), (F32, 64, 48)):
        for W in (1, 7, 150):
            c = random_cache(api, g, 12, 2, block, D)
            d = {k: t.clone() for k, t in c.items()}
            pages = torch.arange(12, device="cuda", dtype=torch.int32).view(2, 6)
            n = torch.tensor([0, 50], device="cuda", dtype=torch.int32)
            x = torch.randn(2, W, 6, D, generator=g, device="cuda").to(dtype)
            q = api.cache_append_rotary(c, x[:, :, :2], x[:, :, 2:4], pages, n, torch.zeros(D // 2, device="cuda", dtype=torch.float64), q=x)
            api.cache_append(d, x[:, :, :2], x[:, :, 2:4], pages, n)
            assert torch.equal(q, x) and all(torch.equal(c[k].view(torch.uint8), d[k].view(torch.uint8)) for k in c)


def test_queries_in_place_and_without_keys_layouts(api):
    """Queries turned where they stand; layouts with strides of their own; calls without queries."""
    g = gen(5)
    for dtype in (BF16, F32):
        for pairs, rot in (("halves", 64), ("halves", 20), ("neighbours", 64)):
            x = torch.randn(3, 6, 4, 69, generator=g, device="cuda").to(dtype)
            q = x[..., 2:66]                             # rows on no 16-byte boundary
            kv = torch.randn(2, 3, 6, 64, generator=g, device="cuda").to(dtype).transpose(1, 2)[:, None]
            k, v = kv[0].transpose(1, 2), kv[1].transpose(1, 2)
            k, v = (torch.randn(3, 2, 6, 64, generator=g, device="cuda").to(dtype).transpose(1, 2) for _ in range(2))   # heads first
            pages = torch.arange(6, device="cuda", dtype=torch.int32).view(3, 2)
            n = torch.tensor([0, 3, 16], device="cuda", dtype=torch.int32)
            freqs = api.rotary_freqs(rot, 500.0)
            a, b = (api.make_token_cache(6, 2, 16, 64) for _ in range(2))
            apart = check_rotary(api, a, k, v, pages, n, freqs, pairs, q)
            rest = x.clone()
            r = api.cache_append_rotary(b, k, v, pages, n, freqs, pairs=pairs, q=q, out=q)
            assert r.data_ptr() == q.data_ptr() and torch.equal(q, apart)
            assert torch.equal(x[..., :2], rest[..., :2]) and torch.equal(x[..., 66:], rest[..., 66:])
            assert api.cache_append_rotary(b, k, v, pages, n, freqs, pairs=pairs) is None
            assert all(torch.equal(a[key].view(torch.uint8), b[key].view(torch.uint8)) for key in a)


def test_rotary_extreme_values_and_missing_pages(api):
    """An infinity's pair is two infinities (inf cos - x sin), codes of +-448, a NaN's two NaN; neither counts for the scale.
    Pages that do not exist."""
    from paper_2606_13426_gb300 import binding as B
    g = gen(6)
    cache = api.make_token_cache(4, 1, 16, 64)
    pages = torch.tensor([[0, 7], [1, -1], [2, 3]], device="cuda", dtype=torch.int32)
    n = torch.tensor([10, 16, 30], device="cuda", dtype=torch.int32)
    k = torch.randn(3, 8, 1, 64, generator=g, device="cuda")
    v = torch.randn(3, 8, 1, 64, generator=g, device="cuda")
    k[0, 1, 0, 5], k[0, 2, 0, 40] = INF, NAN
    status = torch.zeros(3, device="cuda", dtype=torch.int32)
    freqs = api.rotary_freqs(64)
    api.cache_append_rotary(cache, k, v, pages, n, freqs, status=status)
    assert status.tolist() == [B.SDV_STATUS_BAD_PAGE, B.SDV_STATUS_BAD_PAGE, B.SDV_STATUS_BAD_PAGE]   # the third's 33rd token on
    got = held(cache, pages, 0, 10, 6)[0]
    assert (got[1, 0, [5, 37]].abs() == 448 * cache["k_scale"][0, 0].double()).all()
    assert got[2, 0, [8, 40]].isnan().all() and int(got.isnan().sum()) == 2
    y, size = turn(k[0, :6], torch.arange(10, 16, device="cuda"), freqs, "halves")
    top = float(y[y.isfinite()].abs().max())
    assert float(cache["k_scale"][0, 0]) == max(1.0, 2.0 ** math.ceil(math.log2(top / 448)))    # (ten tokens were held at 1)
    fine = y.isfinite()
    assert ((got - y).abs()[fine] <= (2.0 ** -4 * 1.01 * y.abs() + 2.0 ** -9 * cache["k_scale"][0, 0].double())[fine]).all()


# ------------------------------------------------------------------------------ moving rows
def plain_keep(cache, path, pages, lengths):
    P, H, block, D = cache["k"].shape
    got = dict(k=cache["k"].double(), v=cache["v"].double().transpose(2, 3).contiguous(), k_scale=cache["k_scale"].double(),
               v_scale=cache["v_scale"].double())
    src = {a: t.clone() for a, t in got.items()}
    W = path.shape[1]
    for b in range(path.shape[0]):
        n, into = max(int(lengths[b]), 0), {}
        for j in range(W):
            i = int(path[b, j])
            if i < 0:
                break
            if i >= W or i == j:
                continue
            ends = []
            for at in (n + i, n + j):
                page = int(pages[b, at // block]) if at // block < pages.shape[1] else -1
                ends.append((page if 0 <= page < P else -1, at % block))
            if ends[0][0] >= 0 and ends[1][0] >= 0:
                into.setdefault(ends[1][0], []).append((ends[1][1],) + ends[0])
        for page, rows in into.items():
            for a in ("k", "v"):
                for h in range(H):
                    x = torch.stack([src[a][p, h, r] * src[a + "_scale"][p, h] for _, p, r in rows])
                    top = float(torch.where(x.isfinite(), x.abs(), 0.0).max())
                    was = float(src[a + "_scale"][page, h])
                    s = was
                    if top > 0:
                        least = 2.0 ** -126
                        while 448 * least < top:
                            least *= 2
                        s = least if least > abs(was) else was
                    if s != was:
                        got[a][page, h] = e4m3(got[a][page, h] * (was / s))
                        got[a + "_scale"][page, h] = s
                    for (to, _, _), y in zip(rows, x):
                        got[a][page, h, to] = e4m3(y / s)
    got["v"] = got["v"].transpose(2, 3)
    return got


def check_keep(api, cache, path, pages, lengths, status=None):
    ref = plain_keep(cache, path, pages, lengths)
    api.cache_keep(cache, path, pages, lengths, status=status)
    for a in ref:
        assert same(cache[a].double(), ref[a]), a


@pytest.mark.parametrize("B,W,H,D,block", [(1, 1, 1, 64, 16), (4, 8, 2, 128, 64), (9, 33, 3, 64, 48), (6, 64, 2, 128, 16), (5, 64, 1, 64, 128),
                                           (40, 20, 1, 128, 32)])
def test_keep(api, B, W, H, D, block):
    """Random codes, NaN among them, scales of 2^-6 to 2^2: paths of trees, and ones in any order."""
    g = gen(B + W + block)
    M = (2 * block + W) // block + 2
    cache = random_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    n = torch.randint(0, 2 * block, (B,), generator=g, device="cuda", dtype=torch.int32)
    path = torch.full((B, W), -1, dtype=torch.int32)
    for b in range(B):
        par = tree_of("tree", W, b)
        at = [W - 1 - b % max(1, W // 2)]
        while par[at[-1]] >= 0:
            at.append(par[at[-1]])
        path[b, :len(at)] = torch.tensor(at[::-1])
    check_keep(api, cache, path.cuda(), pages, n)
    any_order = torch.randint(-1, W, (B, W), generator=g, device="cuda", dtype=torch.int32)
    any_order[:, 0] = W - 1
    check_keep(api, cache, any_order, pages, n)
    check_keep(api, cache, torch.arange(W, device="cuda", dtype=torch.int32).expand(B, W).contiguous(), pages, n)
    back = torch.arange(W - 1, -1, -1, device="cuda", dtype=torch.int32).expand(B, W).contiguous()
    check_keep(api, cache, back, pages, n)


def test_keep_with_scales_of_a_callers_own(api):
    """Scales that are no powers of two, negative, zero, not finite; sizes far apart."""
    g = gen(7)
    cache = random_cache(api, g, 30, 2, 16, 64)
    for a in ("k_scale", "v_scale"):
        cache[a].mul_(2.0 ** torch.randint(-40, 40, (30, 2), generator=g, device="cuda"))
        cache[a][::7] *= -1
        cache[a][3] = 0
    pages = torch.randperm(30, generator=g, device="cuda").to(torch.int32).view(3, 10)
    n = torch.tensor([3, 40, 80], device="cuda", dtype=torch.int32)
    path = torch.tensor([[0, 5, 17, 33, 40] + [-1] * 59, [3, 30, 31, 60, 2] + [-1] * 59, [0, 1, 2, 50, 63] + [-1] * 59], device="cuda", dtype=torch.int32)
    check_keep(api, cache, path, pages, n)


def test_keep_bad_entries_and_pages(api):
    from paper_2606_13426_gb300 import binding as B
    g = gen(8)
    cache = random_cache(api, g, 12, 2, 16, 64)
    pages = torch.randperm(12, generator=g, device="cuda").to(torch.int32).view(3, 4)
    n = torch.tensor([10, 20, 50], device="cuda", dtype=torch.int32)
    path = torch.tensor([[0, 9, 12, 5, -3, 7] + [-1] * 6, [0, 3, 11, 6, 8, 10] + [-1] * 6, [1, 2, 4, 11, -1, -1] + [-1] * 6], device="cuda", dtype=torch.int32)
    pages[1, 1] = 77                                     # rows 0 to 11 of the second sequence lie in pages 1 and 2 of its table
    status = torch.zeros(3, device="cuda", dtype=torch.int32)
    check_keep(api, cache, path, pages, n, status)
    assert status.tolist() == [B.SDV_STATUS_BAD_TREE, B.SDV_STATUS_BAD_PAGE, 0]
    n.copy_(torch.tensor([2 ** 31 - 1, -5, 60], dtype=torch.int32))
    status.zero_()
    before = {a: t.clone() for a, t in cache.items()}
    api.cache_keep(cache, path, pages, n, status=status)
    assert int(status[0]) & B.SDV_STATUS_BAD_PAGE
    other = pages[0].long()
    assert all(torch.equal(cache[a].view(torch.uint8)[other], before[a].view(torch.uint8)[other]) for a in cache)


def test_cache_offsets_past_32_bits(api):
    H, block, D = 4, 64, 128
    P = (1 << 32) // (H * block * D) + 40
    g = gen(46)
    cache = api.make_token_cache(P, H, block, D)
    small = api.make_token_cache(8, H, block, D)
    pages = torch.arange(P - 8, P, device="cuda", dtype=torch.int32).view(2, 4)
    low = torch.arange(8, device="cuda", dtype=torch.int32).view(2, 4)
    n = torch.tensor([0, 60], device="cuda", dtype=torch.int32)
    k = torch.randn(2, 60, H, D, generator=g, device="cuda")
    path = torch.tensor([[0, 3, 9, 59] + [-1] * 56, [0, 1, 30, 40] + [-1] * 56], device="cuda", dtype=torch.int32)
    for c, p in ((cache, pages), (small, low)):
        api.cache_append_rotary(c, k, k.flip(1), p, n, api.rotary_freqs(D))
        api.cache_keep(c, path, p, n)
    for a in small:
        assert torch.equal(cache[a][P - 8:].view(torch.uint8), small[a].view(torch.uint8))
    assert not cache["k"][: P - 8].view(torch.uint8)[-64:].any() and not cache["k"][:8].view(torch.uint8).any()


def test_captured_and_on_another_stream(api):
    g = gen(9)
    base = random_cache(api, g, 40, 2, 16, 64)
    pages = torch.arange(36, device="cuda", dtype=torch.int32).view(3, 12)
    n = torch.tensor([100, 64, 150], device="cuda", dtype=torch.int32)
    x = torch.randn(3, 12, 8, 64, generator=g, device="cuda").to(BF16)
    path = torch.tensor([[0, 4, 9], [0, 1, 11], [0, 2, 3]], device="cuda", dtype=torch.int32)
    path = torch.cat([path, torch.full((3, 9), -1, device="cuda", dtype=torch.int32)], 1)
    freqs = api.rotary_freqs(64)
    cache = {a: t.clone() for a, t in base.items()}

    def step():
        q = api.cache_append_rotary(cache, x[:, :, :2], x[:, :, 2:4], pages, n, freqs, q=x[:, :, 4:])
        api.cache_keep(cache, path, pages, n)
        return q

    def reset():
        for a in base:
            cache[a].view(torch.uint8).copy_(base[a].view(torch.uint8))
    q = step()
    ref = {a: t.clone() for a, t in cache.items()}
    torch.cuda.synchronize()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q2 = step()
    side.synchronize()
    assert torch.equal(q, q2) and all(torch.equal(ref[a].view(torch.uint8), cache[a].view(torch.uint8)) for a in ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q3 = step()
    for _ in range(2):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, q3) and all(torch.equal(ref[a].view(torch.uint8), cache[a].view(torch.uint8)) for a in ref)


def test_refusals(api):
    from paper_2606_13426_gb300 import binding as B
    c = api.make_token_cache(4, 2, 16, 64)
    pt = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n = torch.ones(1, dtype=torch.int32, device="cuda")
    k = torch.zeros(1, 3, 2, 64, device="cuda")
    f = api.rotary_freqs(64)
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f.float())
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f, pairs="thirds")
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f, q=k.to(BF16))
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f, out=k)
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f, positions=torch.zeros(1, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        api.cache_append_rotary(c, k, k, pt, n, f.cpu())
    with pytest.raises(B.SDVError):
        api.cache_append_rotary(c, k, k, pt, n, api.rotary_freqs(66))
    with pytest.raises(B.SDVError):
        api.cache_append_rotary(c, k, k, pt, n, f[:0])
    with pytest.raises(ValueError):
        api.cache_keep(c, torch.zeros(1, 3, dtype=torch.int64, device="cuda"), pt, n)
    with pytest.raises(ValueError):
        api.cache_keep(c, torch.zeros(2, 3, dtype=torch.int32, device="cuda"), pt, n)
    with pytest.raises(B.SDVError):
        api.cache_keep(c, torch.zeros(1, 65, dtype=torch.int32, device="cuda"), pt, n)
