"""Rows of viscache_kv8_weigh whose lse is -inf add nothing: in both kernels, at scales whose factor of
lse rounds either way."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv8_weigh import Case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 90], ids=["few", "many"])
@pytest.mark.parametrize("d,scale", [(64, None), (128, None), (64, 0.07), (128, 96 ** -0.5), (128, 0.125)])
def test_lse_of_minus_infinity_adds_nothing(d, scale, rows, dtype):
    c = Case([333, 90], [rows, rows], 6, 1, d, 64, dtype, scale=scale)
    rng = np.random.default_rng(5)
    c.lse[rng.random(c.lse.shape) < 0.2] = -np.inf
    c.lse[1] = -np.inf
    assert np.isfinite(c.want()).all()
    c.check()
    c.lse[:] = -np.inf
    c.check()
