"""Finite values near the types' largest stay finite in the 8-bit cache."""
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV, F32, Pool, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_finite_values_read_back_finite(dtype):
    top = torch.finfo(dtype).max
    pool = Pool([40], 1, 16, 64)
    K, V = _rand((40, 1, 64), 1, dtype), _rand((40, 1, 64), 2, dtype)
    K[3, 0, :4] = torch.tensor([top, -top, 3.2e38, -3.3e38]).to(dtype)
    K[17, 0, 0] = top
    K[17, 0, 1] = float("inf")                  # (this one is not)
    V[35, 0, 9] = -top
    pool.append([39], [39], K[:39], V[:39])
    pool.check()
    pool.append([40], [1], K[39:], V[39:])
    pool.check()
    for out_type in (BF, F32):
        k, v = vc.viscache_kv8_read(pool.cache, pool.step([40], [40]), out_type)
        assert torch.isfinite(v).all()
        assert torch.equal(~torch.isfinite(k).cpu(), ~torch.isfinite(K))
        # 4 bits of a number between 240 and 256 steps of 2^120: within 1/16
        got, want = k.float().cpu(), K.float()
        big = torch.isfinite(want) & (want.abs() > 1e38)
        assert ((got - want).abs()[big] <= want.abs()[big] / 16 * 1.001).all()
