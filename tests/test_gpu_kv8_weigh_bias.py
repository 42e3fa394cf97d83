"""The mean error of viscache_kv8_weigh: what the tensor cores cut off a score is made up for, in each
kernel, type and head size."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _mean_error(dtype, d, rows, n_req, along, scale, spread, L=1024, Hkv=2, G=4, page=64, seed=0):
    """(sum of the weights' errors over their sum, mean score of a term, mean distance of a term's score to its lse)"""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device=DEV, generator=g, dtype=torch.float64)
    n = n_req * L // page
    k_scale = torch.full((n, Hkv), 2.0 ** -6, device=DEV)
    codes = torch.from_numpy(kv8.encode((rand(n, Hkv, page, d) * 64).cpu().numpy())).to(DEV)
    keys = torch.from_numpy(kv8.VALUE.astype(np.float64)).to(DEV)[codes.long()] / 64
    keys = keys.view(n_req, L // page, Hkv, page, d).transpose(1, 2).reshape(n_req, Hkv, L, d)
    s = d ** -0.5 if scale == 0.0 else float(np.float32(scale))
    q = rand(n_req, rows, Hkv, G, d) * ((1.0 if along else spread) / (s * math.sqrt(d)))
    if along:                                   # each row along a key: its largest term grows over all of its dimensions
        t = torch.randint(0, L, (n_req, rows, Hkv, G), device=DEV, generator=g)
        for h in range(Hkv):
            q[:, :, h] += keys[torch.arange(n_req, device=DEV)[:, None, None], h, t[:, :, h]] * (3.0 * spread / (s * d))
    q = q.to(dtype)
    x = torch.einsum("rmgjd,rgtd->rmgjt", q.double(), keys) * s
    lse = torch.logsumexp(x, -1).float()
    p = torch.exp(x - lse.double()[..., None])
    want = p.sum((1, 3))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    cache = vc.Kv8Cache(codes, torch.zeros_like(codes), k_scale, torch.zeros_like(k_scale))
    step = vc.Kv8Step(torch.arange(n, dtype=torch.int32, device=DEV).view(n_req, -1), i32([L] * n_req),
                      i32([rows * r for r in range(n_req + 1)]), rows * n_req)
    w = torch.zeros(n, Hkv, page, device=DEV)
    vc.viscache_kv8_weigh(cache, step, q.reshape(rows * n_req, Hkv * G, d), lse.view(rows * n_req, Hkv * G), w, scale,
                          causal=False)
    got = w.double().view(n_req, L // page, Hkv, page).transpose(1, 2).reshape(n_req, Hkv, L)
    total = want.sum()
    return (((got - want).sum() / total).item(), ((p * x).sum() / total).item(),
            ((p * (lse.double()[..., None] - x).abs()).sum() / total).item())


@pytest.mark.parametrize("along", [False, True], ids=["any", "along a key"])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,n_req", [(2, 64), (256, 8)], ids=["few", "many"])
def test_scores_are_not_short_on_average(rows, n_req, d, dtype, along):
    for scale in (0.0, 0.07):
        error, score, away = _mean_error(dtype, d, rows, n_req, along, scale, 5.0)
        # a factor is off by half an ulp at most (2^-24 of the score, or, where lse's goes with it, of a score's distance
        # to its lse); cuts lie within 0.6 of the middle of their range (few rows of fp32: 0.9); the exponentials' 2^-22
        # and the roundings of sums go either way: a tenth of that
        cut = 0.9 if dtype == F32 and rows == 2 else 0.6
        factor = score if rows == 2 else away
        assert abs(error) <= 2.0 ** -24 * (cut * score + factor) + 0.1 * 2.0 ** -22, (error, score, away)
