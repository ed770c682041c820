"""The attention over the 8-bit cache where one row's result must not hang on what other rows see, hold
or are scaled by: value scales far apart, pages behind the span, NaN codes, queries of very different
size.  Every row is compared with the 64-bit form of itself.

Tolerances: scores are within 2^-22 of the sum of their products' magnitudes and probabilities within
2^-20 of themselves, so that an output is within 2^-14 sum p |v| (of its own row) and its rounding.
"""
import pytest
import torch

from test_gpu_tokens import BF16, F16, NAN, api, gen, make_cache, near, plain_attend  # noqa: F401

pytestmark = pytest.mark.gpu

HALF = {BF16: 2.0 ** -8, F16: 2.0 ** -11}


def check_rows(api, q, cache, pages, lengths, counts=None, span=0, scale=None, **kw):
    """As check_attend, with 2^-14 for 2^-11 and nothing absolute but the output's own least step."""
    B, W, Hq, D = q.shape
    r = api.cache_attend(q, cache, pages, lengths, counts=counts, span=span, scale=scale, **kw)
    out, lse, mag = plain_attend(q, cache, pages, lengths, [W] * B if counts is None else counts, D ** -0.5 if scale is None else scale, span)
    least = 2.0 ** -132 if q.dtype == BF16 else 2.0 ** -25
    tol = 2.0 ** -14 * mag + 1.01 * HALF[q.dtype] * out.abs() + least
    err = (r["out"].double() - out).abs()
    assert (err <= tol).all(), "output off by %g of its bound" % float((err / tol).max())
    assert near(r["lse"], lse, 2e-5)
    return r




# ------------------------------------------------------------------------------ roundings
@pytest.mark.parametrize("W,G,D,n", [(1, 4, 128, 900), (9, 4, 128, 700), (5, 7, 64, 3000), (17, 1, 64, 65), (2, 2, 64, 9)])
def test_bf16_outputs_are_rounded_once(api, W, G, D, n):
    """An output is the rounding of a number within 2^-14 sum p |v| of the exact one."""
    g = gen(150 + n)
    cache = make_cache(api, g, 200, 2, 32, D)
    pages = torch.randperm(200, generator=g, device="cuda").to(torch.int32).view(2, 100)
    lengths = torch.tensor([n, n // 2], device="cuda", dtype=torch.int32)
    for sharp in (1.0, 3.0):
        q = (sharp * torch.randn(2, W, 2 * G, D, generator=g, device="cuda")).to(BF16)
        out, _, mag = plain_attend(q, cache, pages, lengths, [W, W], D ** -0.5, 0)
        got = api.cache_attend(q, cache, pages, lengths)["out"].double()
        tol = 2.0 ** -14 * mag
        # (through fp32, whose rounding is 2^-24 of it)
        low, high = ((out - tol).float().to(BF16).double(), (out + tol).float().to(BF16).double())
        assert (low <= got).all() and (got <= high).all()


# ------------------------------------------------------------------------------ value scales
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("k", [20, 27, 30, 40, 60, 100])
def test_a_page_that_a_row_does_not_see_may_have_any_value_scale(api, k, dtype):
    """17 tokens in pages of 16, two queries: the first sees one page, the second's page is 2^k larger."""
    g = gen(80 + k)
    cache = make_cache(api, g, 2, 1, 16, 64)
    lift = 0 if dtype == BF16 else 8                    # (f16 outputs: the large page's values below 2^16)
    cache["v_scale"][0] *= 2.0 ** -(k - lift)
    cache["v_scale"][1] *= 2.0 ** lift
    pages = torch.arange(2, device="cuda", dtype=torch.int32)[None]
    n = torch.tensor([17], device="cuda", dtype=torch.int32)
    q = torch.randn(1, 2, 2, 64, generator=g, device="cuda").to(dtype)
    if dtype == F16 and k > 30:                         # values below f16's least step: nothing to compare
        return
    r = check_rows(api, q, cache, pages, n)
    alone = api.cache_attend(q[:, :1], cache, pages, n - 1)
    a, b = r["out"][:, :1].double(), alone["out"].double()
    assert ((a - b).abs() <= 2 * HALF[dtype] * b.abs() + 2.0 ** -24 * (dtype == F16)).all() and near(r["lse"][:, :1], alone["lse"], 2e-5)


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (F16, 64)])
@pytest.mark.parametrize("k", [20, 30, 40, 80, 140])
def test_rows_whose_weight_lies_on_pages_of_small_values(api, k, dtype, D):
    """Sharp rows over pages whose value scales spread over 2^k, in runs of many steps and in sequences of a
    few; heads whose scales only grow, only fall and are mixed."""
    g = gen(90 + k + D)
    B, H, G, W, block = 5, 4, 2, 3, 32
    M = 640
    cache = make_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    e = torch.rand(B, M, H, generator=g, device="cuda")
    e[:, :, 0] = torch.linspace(0, 1, M, device="cuda")
    e[:, :, 1] = torch.linspace(1, 0, M, device="cuda")
    e[:, :, 2] = (e[:, :, 2] < 0.5).float()              # two sizes, side by side
    e = torch.floor(k * (e - (1.0 if dtype == F16 else 0.5)))
    cache["v_scale"][pages.long()] *= torch.exp2(e)
    cache["v_scale"][pages[:, ::7].long(), 3] *= -1
    cache["v_scale"][pages[:, 3::11].long(), 3] = 0
    n = torch.tensor([M * block - 5, 20000, 13000, 400, 31], device="cuda", dtype=torch.int32)
    for sharp in (1.0, 6.0, 20.0):
        q = (sharp * torch.randn(B, W, H * G, D, generator=g, device="cuda")).to(dtype)
        if dtype == F16:
            cache_ = dict(cache, v_scale=cache["v_scale"] * 2.0 ** 8)
            check_rows(api, q, cache_, pages, n)
        else:
            check_rows(api, q, cache, pages, n)


def test_pages_of_zeros_and_of_huge_values_beside_ordinary_ones(api):
    """Pages of zeros as they are appended (scale 2^-126) first, and a last page that only the later queries see, near
    fp32's end: the earlier queries' results are those without it."""
    g = gen(101)
    H, D, block = 2, 64, 16
    cache = api.make_token_cache(64, H, block, D)
    pages = torch.randperm(64, generator=g, device="cuda").to(torch.int32).view(1, 64)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = torch.randn(1, 900, H, D, generator=g, device="cuda")
    x[:, :100] = 0
    x[:, 300:340] = 0
    api.cache_append(cache, x, x, pages, none)
    q = (2 * torch.randn(1, 6, 4, D, generator=g, device="cuda")).to(BF16)
    n = none + 900
    check_rows(api, q, cache, pages, n)
    for huge in (1e20, 1e30, 3e38):
        y = torch.full((1, 3, H, D), huge, device="cuda")
        c = {k: v.clone() for k, v in cache.items()}
        last = torch.randn(1, 9, H, D, generator=g, device="cuda")       # up to a page's end: 909 = 56 * 16 + 13
        c2 = {k: v.clone() for k, v in c.items()}
        api.cache_append(c, last, last, pages, n)
        api.cache_append(c2, last, last, pages, n)
        api.cache_append(c, last[:, :3], last[:, :3], pages, n + 9)      # to 912
        api.cache_append(c2, last[:, :3], last[:, :3], pages, n + 9)
        api.cache_append(c, last[:, :3], y, pages, n + 12)
        api.cache_append(c2, last[:, :3], last[:, :3], pages, n + 12)
        a = api.cache_attend(q, c, pages, n + 15)                        # queries at 909 .. 914: three see the page at 912
        b = api.cache_attend(q, c2, pages, n + 15)
        u, v = a["out"][:, :3].double(), b["out"][:, :3].double()
        assert ((u - v).abs() <= 2 * HALF[BF16] * v.abs() + 2.0 ** -16).all(), huge
        assert near(a["lse"][:, :3], b["lse"][:, :3].double(), 2e-5)
        out, _, mag = plain_attend(q, c, pages, n + 15, [6], D ** -0.5, 0)
        live = mag < 3e38
        assert ((a["out"].double() - out).abs() <= 2.0 ** -14 * mag + 1.01 * 2.0 ** -8 * out.abs())[live].all()


# ------------------------------------------------------------------------------ pages behind the span
@pytest.mark.parametrize("block,n,span", [(16, 100, 48), (48, 1150, 1000), (80, 570, 321), (16, 3010, 2000)])
def test_pages_behind_the_span_are_not_looked_at(api, block, n, span):
    """A page whose last token lies before every query's span: its table entry may be anything, and so may its scales."""
    g = gen(110 + n)
    M = n // block + 1
    cache = make_cache(api, g, M + 1, 2, block, 64)
    pages = torch.arange(M, device="cuda", dtype=torch.int32)[None].contiguous()
    lengths = torch.tensor([n], device="cuda", dtype=torch.int32)
    for W in (1, 3):
        q = torch.randn(1, W, 4, 64, generator=g, device="cuda").to(BF16)
        first = n - W - span + 1                         # the first key that is seen
        assert first > block
        gone = first // block                            # pages wholly before it
        ref = check_rows(api, q, cache, pages, lengths, span=span)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        for entry in (-1, 1 << 30):
            freed = pages.clone()
            freed[0, :gone] = entry
            r = api.cache_attend(q, cache, freed, lengths, span=span, status=st)
            assert st.tolist() == [0]
            assert torch.equal(r["out"], ref["out"]) and torch.equal(r["lse"], ref["lse"])
        for size in (2.0 ** 100, NAN, 0.0, -1e30):       # another sequence has the page
            c = {k: v.clone() for k, v in cache.items()}
            c["v_scale"][M] = size
            c["k_scale"][M] = size
            lent = pages.clone()
            lent[0, :gone] = M
            r = api.cache_attend(q, c, lent, lengths, span=span)
            assert torch.equal(r["out"], ref["out"]) and torch.equal(r["lse"], ref["lse"]), size


# ------------------------------------------------------------------------------ NaN codes
@pytest.mark.parametrize("B,H,G,W,D,n", [(1, 1, 2, 1, 64, 5000), (2, 2, 4, 9, 128, 900), (40, 2, 1, 3, 64, 30), (3, 1, 5, 4, 64, 64),
                                         (300, 4, 1, 2, 128, 700)])
def test_a_nan_element_makes_the_rows_that_see_it_nan(api, B, H, G, W, D, n):
    """One element of one key or value, in a step inside the sequence and in the last ones: all of the output and lse of
    the rows that see it, nothing of the others."""
    g = gen(120 + B + n)
    block = 32
    M = n // block + 1
    cache = make_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    lengths = torch.full((B,), n, device="cuda", dtype=torch.int32)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
    ref = api.cache_attend(q, cache, pages, lengths)
    b, h = B // 2, H - 1
    for which in ("k", "v"):
        for at in sorted({0, n // 3, n - W - 1, n - W, n - 1}):
            d = (7 * at + 3) % D
            codes = cache[which].view(torch.uint8)
            page, row = int(pages[b, at // block]), at % block
            where = (page, h, row, d) if which == "k" else (page, h, d, row)
            was = int(codes[where])
            codes[where] = 0x7f if at % 2 else 0xff
            r = api.cache_attend(q, cache, pages, lengths)
            codes[where] = was
            sees = torch.zeros(B, W, H * G, dtype=torch.bool, device="cuda")
            sees[b, max(0, at - (n - W)):, h * G:(h + 1) * G] = True
            assert r["out"][sees].isnan().all() and r["lse"][sees].isnan().all(), (which, at)
            assert torch.equal(r["out"][~sees], ref["out"][~sees]) and torch.equal(r["lse"][~sees], ref["lse"][~sees]), (which, at)


# ------------------------------------------------------------------------------ large scores
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,G,W,n", [(64, 2, 2, 300), (128, 4, 9, 1000), (64, 1, 1, 20)])
@pytest.mark.parametrize("size", [2.0 ** 22, 2.0 ** 27, 2.0 ** 40, 2.0 ** 90])
def test_scores_of_any_size(api, D, G, W, n, size, dtype):
    """Scores up to 1e30, where one key stands out, where several are equal, far below 0, and beside
    ordinary ones (the second key head's): queries along one axis, so that the products are exact."""
    g = gen(130 + D)
    H, block = 2, 16
    M = n // block + 1
    cache = make_cache(api, g, M, H, block, D)
    codes = (20 * torch.randn(M, H, block, D, generator=g, device="cuda")).clamp(-200, 200)
    codes[..., 0] = codes[..., 0].clamp(-20, 20)
    codes[M // 3, :, 5, 0] = 448
    codes[M // 2, :, 3, 0] = codes[M // 4, :, 9, 0] = -448
    cache["k"].copy_(codes.to(torch.float8_e4m3fn))
    cache["k_scale"].fill_(2.0 ** -4)
    cache["k_scale"][M // 2 + 1:] = 2.0 ** -6
    cache["v_scale"][::2] *= 2.0 ** 9
    pages = torch.arange(M, device="cuda", dtype=torch.int32)[None]
    lengths = torch.tensor([n], device="cuda", dtype=torch.int32)
    q = torch.zeros(1, W, H * G, D, device="cuda")
    q[..., 0] = 1.0
    q[:, :, G:] = 0.25 * torch.randn(1, W, G, D, generator=g, device="cuda").to(BF16).float()
    q[:, :, G:, 0] = 0
    for sign in (1.0, -1.0):
        z = q.clone()
        z[:, :, :G] *= sign
        z = z.to(dtype)
        if dtype == BF16:
            big = z.clone()
            big[:, :, :G] *= size
            check_rows(api, big, cache, pages, lengths)
        c = dict(cache, k_scale=cache["k_scale"].clone())
        c["k_scale"][:, 0] *= size
        check_rows(api, z, c, pages, lengths)
        if n > 100:                                       # the large ones after ordinary ones, and before
            for part in (slice(0, M // 4), slice(M // 4, M)):
                c = dict(cache, k_scale=cache["k_scale"].clone())
                c["k_scale"][part, 0] *= size
                check_rows(api, z, c, pages, lengths)


# ------------------------------------------------------------------------------ queries
@pytest.mark.parametrize("D,G,W", [(64, 2, 2), (128, 4, 9), (64, 1, 1)])
def test_queries_of_very_different_size_side_by_side(api, D, G, W):
    """A large query in the same call leaves the others what they are.  (It is along one axis, where one key stands
    out, so that its own softmax is decided.)"""
    g = gen(130 + D)
    H, block, n = 2, 16, 300
    cache = make_cache(api, g, 20, H, block, D)
    codes = (20 * torch.randn(20, H, block, D, generator=g, device="cuda")).clamp(-200, 200)
    codes[..., 0] = codes[..., 0].clamp(-50, 50)
    codes[3, :, 5, 0] = 448
    cache["k"].copy_(codes.to(torch.float8_e4m3fn))
    cache["k_scale"].fill_(2.0 ** -4)
    pages = torch.arange(20, device="cuda", dtype=torch.int32)[None]
    lengths = torch.tensor([n], device="cuda", dtype=torch.int32)
    q = torch.randn(1, W, H * G, D, generator=g, device="cuda")
    for size in (2.0 ** 10, 2.0 ** 30, 2.0 ** 60, 2.0 ** 90):
        z = q.clone()
        z[0, W - 1, 0] = 0
        z[0, W - 1, 0, 0] = size
        check_rows(api, z.to(BF16), cache, pages, lengths)
    z = q.clone()
    z[0, 0] *= 2.0 ** -40                                # and small ones: all but flat
    check_rows(api, z.to(BF16), cache, pages, lengths)


@pytest.mark.parametrize("below", [20, 26, 29, 31])
def test_small_elements_of_a_query_count(api, below):
    """Elements 2^-below of a row's largest, all eight of their bits, where the largest meets keys of zero."""
    g = gen(140 + below)
    D = 64
    cache = make_cache(api, g, 4, 1, 32, D)
    codes = cache["k"].float()
    codes[..., 0] = 0
    cache["k"].copy_(codes.to(torch.float8_e4m3fn))
    pages = torch.arange(4, device="cuda", dtype=torch.int32)[None]
    lengths = torch.tensor([100], device="cuda", dtype=torch.int32)
    q = (1 + torch.rand(1, 2, 2, D, generator=g, device="cuda")) * 2.0 ** -below
    q = q * torch.where(torch.rand(1, 2, 2, D, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    q[..., 0] = 1.0
    check_rows(api, q.to(BF16), cache, pages, lengths, scale=2.0 ** below * 0.5)


# ------------------------------------------------------------------------------ prompts
@pytest.mark.parametrize("B,W,H,G,D,span", [(2, 100, 2, 4, 128, 0), (1, 700, 2, 2, 64, 0), (3, 257, 1, 8, 64, 100), (1, 600, 1, 1, 128, 33)])
def test_windows_of_whole_prompts(api, B, W, H, G, D, span):
    """Windows far longer than a row tile: prompts from nothing, prompts behind cached tokens, shorter ones than
    the window; each row against its own reference."""
    g = gen(160 + W)
    block = 64
    M = (W + 300) // block + 1
    cache = make_cache(api, g, B * M, H, block, D)
    pages = torch.randperm(B * M, generator=g, device="cuda").to(torch.int32).view(B, M)
    q = torch.randn(B, W, H * G, D, generator=g, device="cuda").to(BF16)
    n = torch.full((B,), W, device="cuda", dtype=torch.int32)
    check_rows(api, q, cache, pages, n, span=span)
    n += torch.randint(0, 300, (B,), generator=g, device="cuda", dtype=torch.int32)
    counts = torch.randint(1, W + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    check_rows(api, q, cache, pages, n, counts, span=span)
