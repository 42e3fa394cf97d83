"""A key that is not finite with the attention's own lse: NaN goes to the tokens of the rows that see it
and of no other KV head or request."""
import numpy as np
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8_weigh import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 9, 60])
def test_attention_s_lse_of_a_key_that_is_not_finite(rows, dtype):
    c = Case([90, 70], [rows, rows], 4, 2, 64, 16, dtype)
    c.codes[c.table[0, 2], 1, 5] = 0x7F             # token 37 of head 1 of the first request: its last row sees it
    cache, step, q, lse, w = c.device()
    vc.viscache_kv8_attention(cache, step, q, lse=lse)
    c.lse = lse.cpu().numpy()
    assert np.isnan(c.lse[rows - 1, 2:]).all() and np.isfinite(c.lse[:, :2]).all() and np.isfinite(c.lse[rows:]).all()
    got = vc.viscache_kv8_weigh(cache, step, q, lse, w).cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = c.want()
    t = np.arange(90)
    assert np.isnan(got[c.table[0][t // 16], 1, t % 16]).all()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    # as in the operator's own tests: the score's parts and sums, 2^-15 of a sum of positive terms
    assert (np.abs(got[ok] - want[ok]) <= 2.0 ** -15 * np.abs(want[ok]) + 1e-30).all()
