"""Rotary angles of positions over the whole int32 range, against frequencies of 50 digits."""
import decimal

import numpy as np
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("theta,half", [(1e6, 64), (1e4, 32), (5e5, 24)])
def test_far_positions(theta, half):
    pos = [0, 1, -1, 12345, 1 << 20, -(1 << 24) + 3, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31]
    with decimal.localcontext() as ctx:
        ctx.prec = 50
        pi = decimal.Decimal("3.14159265358979323846264338327950288419716939937510")
        freq = [decimal.Decimal(theta) ** (decimal.Decimal(-i) / half) / (2 * pi) for i in range(half)]
        turn = np.array([[float(decimal.Decimal(p) * f % 1) for f in freq] for p in pos])
        w = np.array([[abs(float(decimal.Decimal(p) * f)) for f in freq] for p in pos])
    d = 128 if half > 32 else 64
    x = torch.zeros((len(pos), 1, d), device=DEV)
    x[..., :half] = 1.0                         # (1, 0) in every pair: out is (cos, sin)
    y, _ = vc.viscache_mrope(vc.make_rope((half,), theta), torch.tensor([pos], dtype=torch.int32, device=DEV), x)
    y = y[:, 0].double().cpu().numpy()
    # the phase: a frequency within 2^-45 of itself, 2^-32 turn cut off, rounded to 24 bits (2^-26
    # turn); cosine and sine 2 ulp
    tol = 2 * np.pi * (w * 2.0 ** -45 + 2.0 ** -32 + 2.0 ** -26) + 2.0 ** -22
    assert (np.abs(y[:, :half] - np.cos(2 * np.pi * turn)) <= tol).all()
    assert (np.abs(y[:, half:2 * half] - np.sin(2 * np.pi * turn)) <= tol).all()
