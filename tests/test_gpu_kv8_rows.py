"""Attention over the 8-bit paged cache: what query rows with a wide channel keep of their other
values.  Scores are read off the log-sum-exp."""
import numpy as np
import pytest

from oracle import kv8
from tests.test_gpu_kv8 import BF, DEV, F32, _rand
from tests.test_gpu_kv8_values import FORMS as ALL
from tests.test_gpu_kv8_values import _call, _pool

pytestmark = pytest.mark.gpu
FORMS = [f for f in ALL if f[5] == 1]


def _wide_rows(form, d, width):
    """A call whose rows have one channel `width` times as large as the others, which no key has:
    the log-sum-exps, the reference's, and the scores' size without that channel."""
    m, Hq, dtype = form[1:4]
    n = 300
    K, V = _rand((n, d), 1, F32), _rand((n, d), 2, F32)
    K[..., 5] = 0.0
    q = _rand((m, Hq, d), 3, dtype)
    q[..., 5] = width
    pool = _pool(form, 32, d, K, V)
    _, lse = _call(form, pool, n, q.to(DEV))
    Kd, Vd = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
    ref, size, low = (np.empty((m, Hq)) for _ in range(3))
    for i in range(m):
        k = n - m + i + 1
        for j in range(Hq):
            x = q[i:i + 1, j].double().numpy()
            ref[i, j] = kv8.attention(x, Kd[:k], Vd[:k], None, d ** -0.5)[1][0]
            size[i, j] = (np.abs(x) @ np.abs(Kd[:k]).T * d ** -0.5).max()
            small = np.where(np.abs(x) < 2.0 ** -13 * width, 1.0, 0.0)
            low[i, j] = (small @ np.abs(Kd[:k]).T * d ** -0.5).max()
    return np.abs(lse[0, :, 0].double().cpu().numpy() - ref), np.abs(ref), size, low


@pytest.mark.parametrize("form", [f for f in FORMS if f[3] == F32], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_fp32_rows_with_a_wide_channel(form, d):
    # two fp16 parts hold 22 bits of a value down to 2^-17 of its row's largest (2^14 at least); sums
    # and scalings as elsewhere
    err, ref, size, _ = _wide_rows(form, d, 4096.0)
    assert (err <= size * (d / 8 + 8) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * ref).all(), float(err.max())


@pytest.mark.parametrize("form", [f for f in FORMS if f[3] == BF], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("width", [128.0, 1024.0])
def test_bf16_rows_with_a_wide_channel(form, d, width):
    # values down to 2^-13 of their row's largest are exact, those below within 2^-21 of it
    err, ref, size, low = _wide_rows(form, d, width)
    tol = size * (d / 16 + 6) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * ref + low * 2.0 ** -21 * width
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("form", FORMS, ids=str)
def test_tiny_rows_over_large_keys(form):
    # rows of 2^-122 and keys of 2^124: ordinary scores
    m, Hq, dtype = form[1:4]
    n, d = 300, 64
    K, V = _rand((n, d), 1, F32, 2.0 ** 124), _rand((n, d), 2, F32)
    q = _rand((m, Hq, d), 3, F32, 2.0 ** -122).to(dtype)
    pool = _pool(form, 32, d, K, V)
    _, lse = _call(form, pool, n, q.to(DEV))
    Kd, Vd = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
    for i in (0, m - 1):
        k = n - m + i + 1
        x = q[i, :1].double().numpy()
        ref = kv8.attention(x, Kd[:k], Vd[:k], None, d ** -0.5)[1][0]
        size = (np.abs(x) @ np.abs(Kd[:k]).T * d ** -0.5).max()
        # sums and scalings as elsewhere; the scaling's factor, 2^-126 of a row times a page's scale,
        # may be a number below the normal ones: within 2^-12
        assert abs(float(lse[0, i, 0, 0]) - ref) <= size * ((d / 8 + 8) * 2.0 ** -23 + 2.0 ** -12) + 2.0 ** -20 + 2.0 ** -22 * abs(ref)
