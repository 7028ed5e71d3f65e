"""What an angle is off by: positions and frequencies whose product is so large that this is all that shows, against integers of 200 bits."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2510_05373_amd as kv

pytestmark = pytest.mark.gpu
ONE = 1 << 200


def arctan_inverse(x):
    term = total = ONE // x
    n, sign = 3, -1
    while term:
        term //= x * x
        total += sign * (term // n)
        n, sign = n + 2, -sign
    return total


TWO_PI = Fraction(8 * (4 * arctan_inverse(5) - arctan_inverse(239)), ONE)


# Turns are p (f c), c = 1 / (2 pi) in binary64, 0.56 of 2^-53 off relative to itself; two products, 2^-53 each: 2.56 * 2^-53 of them, and to second
# order nothing; reduced exactly.  So an angle is off by less than 2^-51 p f; sine and cosine besides by what the series and
# its argument in binary32 leave, 8 * 2^-24 as derived in bounded_reference.py.
@pytest.mark.parametrize("channels, interleaved", [(128, False), (128, True), (36, False)])
def test_an_angle_is_exact_to_its_bound(channels, interleaved):
    rng = np.random.default_rng(channels + interleaved)
    freq = rng.choice([-1.0, 1.0], channels // 2) * 10.0 ** rng.uniform(-3.0, 3.0, channels // 2)
    plan, cache, T = kv.KVLincRotary(freq, interleaved=interleaved), kv.KVLincCache(1, 1, 1, 128), 64
    first = 2 ** 31 - 1
    depth = rng.integers(0, 2 ** 31, T).astype(np.int32)
    x = torch.zeros(1, 1, T, 128, device="cuda")
    real = np.arange(0, channels, 2) if interleaved else np.arange(channels // 2)
    other = real + 1 if interleaved else real + channels // 2
    x[..., real] = 1.0
    y = cache.rotary(plan, x, first=torch.tensor([first], dtype=torch.int32, device="cuda"), depth=torch.tensor(depth[None], device="cuda"), counted=False,
                     dtype=torch.float32)[0][0, 0].double().cpu().numpy()
    for t in range(T):
        p = first + int(depth[t])
        for i, f in enumerate(freq):
            turns = p * Fraction(float(f)) / TWO_PI
            a = float((turns - round(turns)) * TWO_PI)  # (in binary64 only when it is small)
            tol = 2.0 ** -51 * abs(p * f) + 8 * 2.0 ** -24
            assert abs(y[t, real[i]] - np.cos(a)) <= tol and abs(y[t, other[i]] - np.sin(a)) <= tol, (t, i, p, f)
