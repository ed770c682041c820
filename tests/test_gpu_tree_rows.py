"""The attention's kernels for many rows of a key head (more than a warp's tile, on the fifth-generation matrix unit) where
they can go wrong: tiles whose last warp is only partly filled, pages that are no power of two, NaN codes in every part of
a step, sequences of many steps.  Tolerances are those of test_gpu_tree_attend.
"""
import pytest
import torch

from test_gpu_tokens import BF16, F16, api, gen, make_cache  # noqa: F401
from test_gpu_tree_attend import HALF, LEAST, check_tree_as, plain_tree, tree_of, widened

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("W,H,G", [(60, 1, 3), (33, 2, 4), (50, 2, 4), (43, 1, 5), (26, 3, 10)])
def test_tiles_that_end_inside_a_warp(api, W, H, G, dtype):
    """Tiles of 90, 66, 100, 108 and 87 rows of 128: items that a run takes whole, and items that several runs share."""
    g = gen(61 + W)
    block, D = 32, 128
    for lengths in ([6000, 61, 700], [W + 17 * (b % 9) for b in range(100)]):
        B, M = len(lengths), max(lengths) // block + 1
        cache = make_cache(api, g, B * M, H, block, D)
        pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
        n = torch.tensor(lengths, device="cuda", dtype=torch.int32)
        q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(dtype)
        check_tree_as(api, q, cache, widened(pages), n, [tree_of("tree", W, b) for b in range(B)])


def row_tiles(q, cache, pages):
    """Tiles of rows of such a call: 0 where the kernels for few rows take it."""
    from paper_2606_13426_gb300 import binding as B
    return B.sdv_tree_attend_row_tiles(q.shape[0], q.shape[1], q.shape[2], cache["k"].shape[1], q.shape[3], cache["k"].shape[2], pages.shape[1])


def laid_out(api, g, lengths, H, block, D, spare=3):
    B, M = len(lengths), max(lengths) // block + 1
    cache = make_cache(api, g, B * M + spare, H, block, D)
    pages = torch.randperm(B * M + spare, generator=g, device="cuda")[:B * M].to(torch.int32).view(B, M)
    return cache, widened(pages), torch.tensor(lengths, device="cuda", dtype=torch.int32)


def check_result(r, q, cache, pages, lengths, par):
    """A result against 64 bits, as check_tree_as holds its own to them, but for the sums: 2^-15 for those of 64 steps, and 2^-24
    of a step's 128 terms and each of up to n / 32 steps after it."""
    D, n = q.shape[3], float(lengths.max())
    out, lse, mag, most = plain_tree(q, cache, pages, lengths, [q.shape[1]] * q.shape[0], par, D ** -0.5)
    sums = (128 + n / 32) * 2.0 ** -24
    E = (2 * D + 8) * 2.0 ** -24 * most
    tol = 2 * (E[..., None] + 2.0 ** -15 + sums) * mag + 1.01 * HALF[q.dtype] * out.abs() + LEAST[q.dtype]
    err = (r["out"].double() - out).abs()
    assert (err <= tol).all(), "output off by %g of its bound" % float((err / tol).max())
    err = (r["lse"].double() - lse).abs()
    assert (err <= E + 2.0 ** -19 + sums + 2.0 ** -22 * lse.abs()).all(), "lse off by %g" % float(err.max())


PAGES = [(block, D) for block in range(16, 129, 16) for D in (64, 128)]


@pytest.mark.parametrize("block,D", PAGES)
def test_every_size_of_pages(api, block, D):
    """Steps of 128, 96, 80 and 112 keys, of one page to eight; both types; a negative scale; scales far apart, of either sign
    and zero; pages that are not there."""
    from paper_2606_13426_gb300 import binding as B
    g = gen(71 + block + D)
    step = 128 // block * block
    for (W, H, G), dtype in (((64, 2, 2), BF16), ((60, 2, 3), F16)):
        cache, pages, n = laid_out(api, g, [W, W + step, 3 * step, 3 * step + 1, 17 * step - 5], H, block, D)
        q = torch.randn(len(n), W, H * G, D, generator=g, device="cuda").to(dtype)
        par = [tree_of("tree", W, b) for b in range(len(n))]
        assert row_tiles(q, cache, pages) == (W * G + 127) // 128
        check_tree_as(api, q, cache, pages, n, par)
        c = {a: t.clone() for a, t in cache.items()}
        k = 40 if dtype == BF16 else 8
        c["v_scale"] *= torch.exp2(torch.floor(k * (torch.rand(c["v_scale"].shape, generator=g, device="cuda") - 0.5)))
        c["v_scale"][::5] *= -1
        c["v_scale"][3::11] = 0
        c["k_scale"][1::4] *= -1
        counts = torch.tensor([W, 1, W // 2, 0, W - 1], device="cuda", dtype=torch.int32)
        check_tree_as(api, 4 * q, c, pages, n, par, counts, scale=-0.1)
        gone = pages.clone()
        gone[1, 0], gone[3, min(1, 3 * step // block)], gone[4, 1::3] = -1, cache["k"].shape[0], -1
        status = torch.zeros(len(n), device="cuda", dtype=torch.int32)
        check_tree_as(api, q, cache, gone, n, par, status=status)
        assert status.tolist() == [0, B.SDV_STATUS_BAD_PAGE, 0, B.SDV_STATUS_BAD_PAGE, B.SDV_STATUS_BAD_PAGE]


@pytest.mark.parametrize("block,D", PAGES)
def test_a_nan_code_in_every_part_of_a_step(api, block, D):
    """One NaN code in each (sequence, head): every chunk of a step, steps at the beginning, within and at the end of runs of
    several, the context and the tree.  The rows that see it are NaN, all others have the bits that they have without."""
    g = gen(81 + block + D)
    step = 128 // block * block
    W, H, G = 32, 8, 4
    lengths = [20 * step + 7, 18 * step, 23 * step - 1, 20 * step + 33, 19 * step + 1, 21 * step + step // 2]
    B, chunks = len(lengths), step // 16
    cache, pages, n = laid_out(api, g, lengths, H, block, D)
    par = [tree_of("tree", W, b) for b in range(B)]
    parents = torch.tensor(par, dtype=torch.int32, device="cuda")
    below = [[[False] * W for _ in range(W)] for _ in range(B)]     # [sequence][node][ancestor or itself]
    for b in range(B):
        for i in range(W):
            u = i
            while u >= 0:
                below[b][i][u] = True
                u = par[b][u]
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
    assert row_tiles(q, cache, pages) == 1
    units = sum(-(-x // step) for x in lengths) * H
    assert units > 5 * torch.cuda.get_device_properties(0).multi_processor_count        # runs of five steps and more
    base = api.tree_attend(q, cache, pages, n, parents)
    assert base["out"].isfinite().all() and base["lse"].isfinite().all()
    table = pages.cpu()
    for turn in range(4):
        for name in ("k", "v"):
            c = {a: t.clone() for a, t in cache.items()}
            codes = c[name].view(torch.uint8)
            want = torch.zeros(B, W, H * G, dtype=torch.bool)
            for b in range(B):
                for h in range(H):
                    i = b * H + h + turn * B * H
                    at = (7 * i + turn) % -(-lengths[b] // step) * step + i % chunks * 16 + (5 * i + turn) % 16
                    if turn == 3 and i % 2:                         # a node's
                        at = lengths[b] - 1 - (3 * i) % W
                    at = min(at, lengths[b] - 1)
                    page, row, d = int(table[b, at // block]), at % block, (11 * i + 3) % D
                    if name == "k":
                        codes[page, h, row, d] = 0x7f if i % 2 else 0xff
                    else:
                        codes[page, h, d, row] = 0xff if i % 2 else 0x7f
                    node = at - (lengths[b] - W)
                    for j in range(W):
                        want[b, j, h * G:(h + 1) * G] = node < 0 or below[b][j][node]
            r = api.tree_attend(q, c, pages, n, parents)
            want = want.cuda()
            assert torch.equal(r["lse"].isnan(), want) and torch.equal(r["out"].isnan(), want[..., None].expand_as(r["out"]))
            assert torch.equal(r["out"][~want], base["out"][~want]) and torch.equal(r["lse"][~want], base["lse"][~want])


def test_which_kernels_run(api):
    """Few rows go through cache_attend's kernels, many over a long table through their own, in tiles of up to 128."""
    from paper_2606_13426_gb300 import binding as B
    assert B.sdv_tree_attend_row_tiles(2, 4, 8, 8, 128, 64, 1000) == 0
    assert [B.sdv_tree_attend_row_tiles(32, W, 32, 8, 128, 64, 250) for W in (32, 33, 64)] == [1, 2, 2]


@pytest.mark.parametrize("W,H,G,D,B", [(64, 1, 8, 128, 40), (64, 1, 8, 64, 40), (32, 1, 4, 128, 152)])
def test_sums_do_not_lose_with_their_length(api, W, H, G, D, B):
    """Values that are all alike, so that an output is the ratio of two sums of the same probabilities, 2^-14 to either side of the
    middle between two f16 numbers: it rounds to the one on its side if it is within 2^-14, 6.1e-5, of the value.

    The matrix unit's sums are cut off: 5e-7 for a step of 128 keys, 3.2e-5 for the 64 that are summed there (without a limit
    these runs of 250 steps lose 1.6e-4).  Probabilities' halves lose 2^-22, the sums of probabilities, rounded to nearest, (128 +
    250) 2^-24 at most: 5.5e-5 altogether."""
    g = gen(91 + W + D)
    block, n = 64, 32000
    cache = make_cache(api, g, n // block, H, block, D)
    cache["v"].view(torch.uint8).fill_(0x38)             # 1
    pages = torch.arange(n // block, device="cuda", dtype=torch.int32).expand(B, -1).contiguous()
    lengths = torch.full((B,), n, device="cuda", dtype=torch.int32)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(F16)
    parents = torch.tensor(tree_of("tree", W), dtype=torch.int32, device="cuda").expand(B, W).contiguous()
    assert row_tiles(q, cache, pages) == W * G // 128
    for side, want in ((1, 1 + 2.0 ** -10), (-1, 1.0)):
        cache["v_scale"].fill_((1 + 2.0 ** -11) * (1 + side * 2.0 ** -14))
        r = api.tree_attend(q, cache, pages, lengths, parents)
        assert (r["out"] == want).all(), "%d of %d" % (int((r["out"] != want).sum()), r["out"].numel())


@pytest.mark.parametrize("growing", ["keys", "huge", "values"])
@pytest.mark.parametrize("D", [64, 128])
def test_references_that_move_over_many_steps(api, D, growing):
    """Runs of 157 steps, of which every 64 are put aside: scores that grow along the sequence, so that the rows' references pass
    what was put aside again and again; scores past 2^20, which get bases; value scales far apart."""
    g = gen(95 + D)
    W, G, B, block, n = 64, 8, 38, 32, 20000
    cache = make_cache(api, g, n // block, 1, block, D)
    at = torch.arange(n // block, device="cuda", dtype=torch.float32)[:, None] / (n // block)
    if growing == "keys":
        cache["k_scale"].copy_(0.05 + 4 * at)
    elif growing == "huge":
        cache["k_scale"].copy_(torch.exp2(torch.floor(24 * at)))
    else:
        cache["v_scale"].copy_(torch.exp2(torch.floor(40 * torch.rand(at.shape, generator=g, device="cuda") - 20)))
    one = torch.arange(n // block, device="cuda", dtype=torch.int32)[None]
    pages = one.expand(B, -1).contiguous()
    lengths = torch.full((B,), n, device="cuda", dtype=torch.int32)
    for dtype in (BF16, F16):
        if growing == "values" and dtype == F16:
            cache["v_scale"].clamp_(2.0 ** -6, 2.0 ** 5)
        q = torch.randn(1, W, G, D, generator=g, device="cuda").to(dtype)
        many = q.expand(B, -1, -1, -1).contiguous()
        assert row_tiles(many, cache, pages) == 4
        par = tree_of("tree", W)
        r = api.tree_attend(many, cache, pages, lengths, torch.tensor([par] * B, device="cuda", dtype=torch.int32))
        assert all(torch.equal(r[k], r[k][:1].expand_as(r[k])) for k in ("out", "lse"))     # each of them one run
        check_result({k: t[:1] for k, t in r.items()}, q, cache, one, lengths[:1], [par])


@pytest.mark.parametrize("W,D", [(2, 64), (2, 128), (8, 128)])
def test_sums_of_few_rows_do_not_lose_with_their_length(api, W, D):
    """As above for the kernels for few rows, a run of 1000 steps of 32 keys a warp: a step's products are summed by the matrix unit
    (1.3e-7), the steps rounded to nearest, within 1000 2^-24 = 6e-5 were they all one way, in fact within a hundredth of it."""
    g = gen(97 + W + D)
    B, H, G, block, n = torch.cuda.get_device_properties(0).multi_processor_count, 8, 4, 64, 32000
    cache = make_cache(api, g, n // block, H, block, D)
    cache["v"].view(torch.uint8).fill_(0x38)             # 1
    pages = torch.arange(n // block, device="cuda", dtype=torch.int32).expand(B, -1).contiguous()
    lengths = torch.full((B,), n, device="cuda", dtype=torch.int32)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(F16)
    parents = torch.tensor(tree_of("tree", W), dtype=torch.int32, device="cuda").expand(B, W).contiguous()
    assert row_tiles(q, cache, pages) == 0
    for side, want in ((1, 1 + 2.0 ** -10), (-1, 1.0)):
        cache["v_scale"].fill_((1 + 2.0 ** -11) * (1 + side * 2.0 ** -14))
        r = api.tree_attend(q, cache, pages, lengths, parents)
        assert (r["out"] == want).all(), "%d of %d" % (int((r["out"] != want).sum()), r["out"].numel())


@pytest.mark.parametrize("growing", ["keys", "huge", "values"])
@pytest.mark.parametrize("W,D", [(3, 64), (2, 128), (8, 128)])
def test_references_of_few_rows_that_move_over_many_steps(api, W, D, growing):
    """The same on the kernels for few rows, in runs of 625 steps of 32 keys."""
    g = gen(99 + W + D)
    B, H, G, block, n = torch.cuda.get_device_properties(0).multi_processor_count, 8, 4, 32, 20000
    cache = make_cache(api, g, n // block, H, block, D)
    at = torch.arange(n // block, device="cuda", dtype=torch.float32)[:, None] / (n // block)
    if growing == "keys":
        cache["k_scale"].copy_((0.05 + 4 * at).expand(-1, H))
    elif growing == "huge":
        cache["k_scale"].copy_(torch.exp2(torch.floor(24 * at)).expand(-1, H))
    one = torch.arange(n // block, device="cuda", dtype=torch.int32)[None]
    pages = one.expand(B, -1).contiguous()
    lengths = torch.full((B,), n, device="cuda", dtype=torch.int32)
    for dtype in (BF16, F16):
        if growing == "values":
            span = 40 if dtype == BF16 else 10
            cache["v_scale"].copy_(torch.exp2(torch.floor(span * torch.rand(at.shape[0], H, generator=g, device="cuda") - span / 2)))
        q = torch.randn(1, W, H * G, D, generator=g, device="cuda").to(dtype)
        many = q.expand(B, -1, -1, -1).contiguous()
        assert row_tiles(many, cache, pages) == 0
        par = tree_of("tree", W)
        r = api.tree_attend(many, cache, pages, lengths, torch.tensor([par] * B, device="cuda", dtype=torch.int32))
        assert all(torch.equal(r[k], r[k][:1].expand_as(r[k])) for k in ("out", "lse"))     # each item one warp's
        check_result({k: t[:1] for k, t in r.items()}, q, cache, one, lengths[:1], [par])


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("W,H,G,D", [(64, 2, 2, 128), (64, 2, 2, 64), (4, 2, 4, 128), (6, 2, 2, 64)])
def test_probabilities_have_22_bits(api, W, H, G, D, wide):
    """Scores without rounding errors (whole queries, keys and scales): f16 outputs are roundings of numbers within 2^-18 sum p |v|.

    A score is a whole number times scale / ln 2 in fp32, below 32: half a step of it, with the argument's own rounding, makes
    2^-19.5 of a probability; ex2 2^-22; its halves 2^-22; the sum of probabilities 2^-22 (pairs of 64 terms, few steps); what the matrix unit cuts off of
    the sum of products 5e-7, 2^-21, a step of 128 keys, runs have two steps here.  Together below 2^-18.4.  With eleven bits
    (one half alone), outputs are off by up to 2^-10 of them: the bound has to turn them down."""
    g = gen(101 + W + D)
    block, n = 32, 1500
    M = 200_000 // block if wide else n // block + 1
    cache = make_cache(api, g, 2 * (n // block + 1), H, block, D)
    cache["k"].copy_((torch.randint(-2, 3, cache["k"].shape, generator=g, device="cuda")).float().to(torch.float8_e4m3fn))
    cache["k_scale"].fill_(0.25)
    cache["v"].copy_((1 + torch.rand(cache["v"].shape, generator=g, device="cuda")).to(torch.float8_e4m3fn))
    cache["v_scale"].copy_(torch.exp2(torch.randint(-1, 2, cache["v_scale"].shape, generator=g, device="cuda").float()))
    pages = torch.full((2, M), -1, dtype=torch.int32, device="cuda")
    pages[:, :n // block + 1] = torch.arange(2 * (n // block + 1), device="cuda", dtype=torch.int32).view(2, -1)
    lengths = torch.tensor([n, 321], device="cuda", dtype=torch.int32)
    q = torch.randint(-2, 3, (2, W, H * G, D), generator=g, device="cuda").to(F16)
    assert (row_tiles(q, cache, pages) > 0) == (wide and W == 64)
    par = [tree_of("tree", W)] * 2
    scale = D ** -0.5
    out, _, mag, most = plain_tree(q, cache, pages[:, :n // block + 1], lengths, [W, W], par, scale)
    got = api.tree_attend(q, cache, pages, lengths, torch.tensor(par, device="cuda", dtype=torch.int32))["out"].double()
    low, high = [x.to(F16).double() for x in (out - 2.0 ** -18 * mag, out + 2.0 ** -18 * mag)]
    assert (low <= got).all() and (got <= high).all()
    # a row of the oracle's with probabilities of eleven bits, cut off below the row's largest
    at = torch.arange(n - W + 1, device="cuda")
    k = (cache["k"][pages[0, at // block].long(), 0, at % block].double() * 0.25)
    v = cache["v"][pages[0, at // block].long(), 0, :, at % block].double() * cache["v_scale"][pages[0, at // block].long(), 0].double()[:, None]
    p = torch.softmax(scale * (q[0, 0, :G].double() @ k.T), 1)
    assert ((p @ v - out[0, 0, :G]).abs() <= 1e-12).all()
    _, e = torch.frexp(p)
    cut = torch.floor(p * torch.exp2(11.0 - e)) * torch.exp2(e - 11.0)
    bad = (cut @ v).to(F16).double()
    assert not ((low[0, 0, :G] <= bad) & (bad <= high[0, 0, :G])).all()
