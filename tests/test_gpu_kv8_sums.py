"""fp32 sums of the few-rows attention kernel over the 8-bit paged cache, over long contexts and
full batches."""
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV
from tests.test_gpu_kv8_values import runs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq", [4, 48], ids=["1 row", "12 rows"])
@pytest.mark.parametrize("d", [64, 128])
def test_fp32_sums_over_long_contexts(Hq, d):
    # 256 units of about 157 tiles on every SM, values around 1: a warp adds up more than a hundred
    # chunks.  Scores below 4 (log2) summed over 2 d / 16 steps cut off at 2^-23: 2^-19 at most;
    # exponentials and two parts 2^-21; a chunk's product cut off twice at 2^-23, sums rounded to
    # nearest: under 2^-18 of the output's norm together
    n_req, Hkv, page, n = 64, 4, 128, 20000
    g = torch.Generator(DEV).manual_seed(7)
    pages = -(-n // page)
    codes = []
    for mean in (0.0, 1.0):
        x = torch.randn((pages * n_req, Hkv, page, d), generator=g, device=DEV, dtype=BF) * 0.25 + mean
        codes.append((x * 128).to(torch.float8_e4m3fn).view(torch.uint8))
        del x
    scale = torch.full((pages * n_req, Hkv), 2.0 ** -7, device=DEV)
    cache = vc.Kv8Cache(*codes, scale, scale)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    table = torch.randperm(pages * n_req, generator=g, device=DEV).to(torch.int32).view(n_req, pages)
    step = vc.Kv8Step(table, i32([n] * n_req), i32(list(range(n_req + 1))), n_req)
    q = torch.randn((n_req, Hq, d), generator=g, device=DEV)
    with runs("kv8_attn"):
        out = vc.viscache_kv8_attention(cache, step, q)
    G = Hq // Hkv
    for r in range(0, n_req, 7):
        for h in range(Hkv):
            Kd, Vd = (c[table[r].long(), h].view(torch.float8_e4m3fn).double().mul_(2.0 ** -7).view(-1, d)[:n] for c in codes)
            x = q[r, h * G:(h + 1) * G].double() @ Kd.T * d ** -0.5
            ref = torch.softmax(x, 1) @ Vd
            err = (out[r, h * G:(h + 1) * G].double() - ref).norm() / ref.norm()
            assert err <= 2.0 ** -18, float(err)
