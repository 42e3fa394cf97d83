"""Rows of viscache_kv8_weigh that are no tokens (more rows than tokens, a padded batch) add nothing,
whatever their queries and their lse hold."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv8_weigh import Case

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows", [[6, 10], [90, 140]], ids=["few", "many"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_rows_that_are_no_tokens_may_hold_anything(value, rows, causal, dtype):
    lens = [3, 7] if rows[0] < 50 else [20, 33]
    c = Case(lens, rows, 4, 2, 64, 16, dtype, causal)
    at = 0
    for x, m in zip(lens, rows):
        c.q[at:at + m - x] = value
        c.lse[at:at + m - x] = value
        at += m
    assert np.isfinite(c.want()).all()
    c.check()
