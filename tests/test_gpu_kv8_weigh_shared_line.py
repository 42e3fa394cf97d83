"""GPU parity of viscache_kv8_weigh where requests with more rows than tokens share the line of
steps with others (more units than blocks): tests/test_kv8_line.py checks the sharing itself."""
import numpy as np
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8_weigh import Case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("batch", [([20] * 24, [64] * 24), ([90] * 23 + [20], [64] * 24), ([20] + [90] * 39, [64] * 40),
                                   ([500, 40, 0, 13] * 10, [60, 100, 9, 70] * 10)], ids=["all", "last", "first", "mixed"])
def test_more_rows_than_tokens_on_a_shared_line(batch, dtype):
    c = Case(*batch, 64, 8, 64, 16, dtype)
    c.check()
    dead = ~np.isfinite(c.lse)                  # rows that are no tokens add nothing whatever their lse says
    c.lse[dead] = -3.0
    c.check()
