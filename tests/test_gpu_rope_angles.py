"""slimattn_rope_*: sines and cosines at positions over the whole range of int32, against rational arithmetic.

A pair (1, 0) without a norm turns into (cos t, sin t), back into (cos t, -sin t): one product with 1, one sum with 0, nothing rounded behind the sine and cosine.
Tolerance, in steps of h = 2^-25: the reduced angle (at most pi/4) is rounded to 32 bits, h; a sum's last rounding (values up to 1), h; the roundings inside, of the
square (2^-24 of it, halved by the cosine's term, a sixth in the sine's), the cubic's product and the inner sums, below h; the first Taylor term left out,
2e-9 < h / 8.  Together below 4 h = 2^-23."""
from fractions import Fraction
import math

import numpy as np
import pytest
import torch

from paper_2509_26246_amd import harness as H

pytestmark = pytest.mark.gpu
PI = Fraction(31415926535897932384626433832795028841971693993751058209749446, 10 ** 61)   # to 61 decimals


def _cos_sin(pos, freq):
    """In 64 bits, of the exact product reduced by quarter turns."""
    t = Fraction(pos) * Fraction(freq)
    k = round(t / (PI / 2))
    a = float(t - k * PI / 2)
    c, s = math.cos(a), math.sin(a)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[k % 4]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("lo,hi", [(0.9, 1.0), (1e-6, 0.1), (1.0, 50.0)])
def test_far_positions_are_as_exact_as_near_ones(lo, hi, adjacent):
    T, d = 24, 128
    r = np.random.default_rng(1)
    pos = np.concatenate([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 1 << 24, 123456789], r.integers(2 ** 30, 2 ** 31, 8), -r.integers(2 ** 30, 2 ** 31, 4),
                          r.integers(0, 2 ** 17, 4)]).astype(np.int32)
    freq = r.uniform(lo, hi, d // 2).astype(np.float32)
    want = torch.tensor([[_cos_sin(int(p), float(f)) for f in freq] for p in pos], dtype=torch.float64)      # [T, pairs, 2]
    x = torch.zeros(T, 1, d)
    x[..., 0:d:2 if adjacent else 1][..., :d // 2] = 1
    pairs = (lambda y: y.reshape(T, d // 2, 2)) if adjacent else (lambda y: y.reshape(T, 2, d // 2).transpose(1, 2))
    rot = H.Rotary(1, 0, d, torch.float32, torch.from_numpy(freq).cuda(), adjacent=adjacent)
    x, dpos, y, g = x.cuda(), torch.from_numpy(pos).cuda(), torch.empty(T, 1, d, device="cuda"), torch.empty(T, 1, d, device="cuda")
    rot.forward(x, None, dpos, y, None)
    rot.backward(x, None, dpos, x, None, g, None)
    for got, sign in ((y, 1.0), (g, -1.0)):
        err = (pairs(got.double().cpu()) - want * torch.tensor([1.0, sign])).abs().max()
        assert err <= 2.0 ** -23, f"{float(err):.2e}"
