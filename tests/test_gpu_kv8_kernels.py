"""Attention over the 8-bit paged cache: units split over many blocks, on each kernel by name (a
table's width alone does not say which kernel a call with long contexts takes)."""
import pytest

from tests.test_gpu_kv8 import BF, F32, _filled
from tests.test_gpu_kv8_chunks import check
from tests.test_gpu_kv8_values import runs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,lens,rows,Hq,page,d,dtype,wide", [
    ("kv8_attn", [20000, 3001], [4, 3], 4, 64, 128, BF, False),
    ("kv8_attn", [20000, 3001], [4, 3], 4, 64, 128, F32, False),
    ("kv8_attn", [20000, 3001], [2, 2], 4, 16, 64, F32, True),
    ("kv8_attn", [9000], [16], 2, 16, 64, F32, False),
    ("kv8_attn_tc1", [20000, 3001], [30, 17], 4, 64, 128, BF, False),
    ("kv8_attn_tc1", [20000, 3001], [40, 17], 4, 64, 128, F32, False),
    ("kv8_attn_tc1", [9000], [300], 2, 16, 64, F32, True),
    ("kv8_attn_tc1", [9000], [300], 1, 128, 128, BF, False),
    ("kv8_attn_tc2", [20000], [300], 4, 64, 128, BF, True),
    ("kv8_attn_tc2", [9000], [600], 2, 16, 64, BF, True)], ids=str)
def test_units_split_over_blocks(kernel, lens, rows, Hq, page, d, dtype, wide):
    pool = _filled(lens, 1, page, d)
    with runs(kernel):
        check(pool, lens, rows, Hq, True, wide, sample=3, dtype=dtype)
