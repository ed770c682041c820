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
