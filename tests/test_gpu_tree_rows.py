"""The attention's kernels for many rows of a key head (more than a warp's tile, on the fifth-generation matrix unit) where
they can go wrong: tiles whose last warp is only partly filled, pages that are no power of two, NaN codes in every part of
a step, sequences of many steps.  Tolerances are those of test_gpu_tree_attend.
"""
import pytest
import torch

from test_gpu_tokens import BF16, F16, api, gen, make_cache  # noqa: F401
from test_gpu_tree_attend import check_tree_as, tree_of, widened

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
