"""The attention over the 8-bit cache, each output against the 64-bit form of its own row.

Tolerances: scores are within 2^-22 of the sum of their products' magnitudes and probabilities within
2^-20 of themselves, so that an output is within 2^-14 sum p |v| (of its own row) and its rounding.
"""
import pytest
import torch

from test_gpu_tokens import BF16, api, gen, make_cache, plain_attend  # noqa: F401

pytestmark = pytest.mark.gpu


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
