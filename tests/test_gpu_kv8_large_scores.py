"""Attention over the 8-bit paged cache: scores in the millions, of which fp32 keeps a quarter."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV, F32, _rand
from tests.test_gpu_kv8_values import FORMS as ALL
from tests.test_gpu_kv8_values import _pool, runs
from tests.test_gpu_kv8_chunks import _step

pytestmark = pytest.mark.gpu
FORMS = [f for f in ALL if f[5] == 1]
UNIT = 0.6931472                                # times log2(e) in fp32: 1


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("size", [1.0, 2.0 ** -4, 2.0 ** -20, 2.0 ** 12])
def test_scores_of_2_to_the_21(form, size):
    # one token at 2^21 (log2 units), one 8 above it in a later tile and in a page of another V scale,
    # the rest far below
    kernel, m, Hq, dtype = form[:4]
    assert np.float32(UNIT) * np.float32(np.log2(np.e)) == 1.0
    n, d, a, b = 700, 64, 40, 300
    K, V = torch.zeros(n, d), _rand((n, d), 2, F32)
    V[b // 16 * 16:b // 16 * 16 + 16] *= size
    K[:, 0] = 1024.0
    K[a, 0] = K[b, 0] = 2048.0
    K[b, 1] = 32.0
    q = torch.zeros((m, Hq, d))
    q[..., 0], q[..., 1] = 1024.0, 0.25
    pool = _pool(form, 16, d, K, V)
    step = _step(pool, [n], [m], form[4])
    with runs(kernel):
        out = vc.viscache_kv8_attention(pool.cache, step, q.to(dtype).to(DEV), UNIT, True)
    Kd, Vd = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
    x = Kd @ q[0, 0].double().numpy()
    assert x[b] - x[a] == 8.0 and x[a] == 2.0 ** 21 and np.delete(x, [a, b]).max() <= 2.0 ** 20
    ref = (Vd[b] + 2.0 ** -8 * Vd[a]) / (1 + 2.0 ** -8)
    # probabilities to fp16 (2^-11) or two of them, the output's rounding
    rel = (2.0 ** -11 if dtype == BF else 2.0 ** -20)
    tol = rel * (np.abs(Vd[b]) + 2.0 ** -8 * np.abs(Vd[a])) + torch.finfo(dtype).eps / 2 * np.abs(ref) * (1 + rel)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert (err <= tol).all(), float((err / tol).max())
