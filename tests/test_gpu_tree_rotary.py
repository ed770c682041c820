"""The position rotation where its angles can go wrong: frequencies of either sign and any size at far positions."""
import math
import random
from fractions import Fraction

import pytest
import torch

from test_gpu_tokens import F32, api, gen  # noqa: F401

pytestmark = pytest.mark.gpu

TWO_PI = 2 * Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


def exact_angle(pos, f):
    """pos f modulo a turn, as the nearest float."""
    x = pos * Fraction(f)
    return float(x - math.floor(x / TWO_PI + Fraction(1, 2)) * TWO_PI)


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_far_positions_and_frequencies_of_either_sign(api, pairs):
    """Queries (1, 0) become (cos, sin) of the angle.  The argument, an eighth of a turn at most, is rounded twice, 2^-23 of it; the
    series and its roundings add 2^-24: 2^-22.5 of 1.  The angle itself is off by pos (2^-52 |f| + 2^-61) and a step of 2^-33 turns."""
    rng = random.Random(5)
    D, W, block = 128, 32, 32
    size = [10.0 ** rng.uniform(-12, 0.5) for _ in range(48)] + [1e-9 * (1 + k / 16) for k in range(16)]
    freqs = [s if k % 2 else -s for k, s in enumerate(size)]
    far = [2 ** 31 - 1 - rng.randrange(10 ** 6) for _ in range(W // 2)] + [rng.randrange(2 ** 20) for _ in range(W // 2 - 2)] + [0, -2 ** 31]
    cache = api.make_token_cache(1, 1, block, D)
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k = torch.zeros(1, W, 1, D, device="cuda")
    q = torch.zeros(1, W, 1, D, device="cuda")
    a, b = (slice(0, D // 2), slice(D // 2, D)) if pairs == "halves" else (slice(0, D, 2), slice(1, D, 2))
    q[..., a] = 1
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    out = api.cache_append_rotary(cache, k, k, table, lengths, f, pairs=pairs, q=q,
                                  positions=torch.tensor([far], dtype=torch.int32, device="cuda"))[0, :, 0].double().cpu()
    for w, pos in enumerate(far):
        for i, x in enumerate(freqs):
            t = exact_angle(pos, x)
            tol = 2.0 ** -22.5 + abs(pos) * (2.0 ** -52 * abs(x) + 2.0 ** -61) + 2 * math.pi * 2.0 ** -33
            assert abs(out[w, a][i] - math.cos(t)) <= tol and abs(out[w, b][i] - math.sin(t)) <= tol, (pos, x)
