"""Attention over the 8-bit paged cache where values are far apart: pages of V of very different
size, seen and unseen, query rows with a channel far above the others, and long sums.  Every
case says which kernel it is for and checks that it ran there."""
import contextlib

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV, F32, Pool, _rand
from tests.test_gpu_kv8_chunks import _run, _step

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def runs(kernel):
    vc.viscache_profile_enable(True)
    try:
        yield
        torch.cuda.synchronize()
        assert list(vc.viscache_profile_read()) == [kernel]
    finally:
        vc.viscache_profile_enable(False)


# kernel, rows of a request, query heads a KV head, type, wide table, requests: one, or 40 (with the
# same pages, and 4 KV heads with the same rows), so that a warp of the few-rows kernel takes several chunks
FORMS = [("kv8_attn", 5, 1, BF, False, 1), ("kv8_attn", 5, 1, BF, False, 40), ("kv8_attn", 14, 1, BF, False, 40),
         ("kv8_attn", 6, 4, F32, False, 1), ("kv8_attn", 6, 4, F32, False, 40), ("kv8_attn", 4, 2, F32, False, 40),
         ("kv8_attn_tc1", 90, 2, BF, True, 1), ("kv8_attn_tc1", 90, 2, F32, True, 1),
         ("kv8_attn_tc2", 150, 4, BF, True, 1)]


def _pool(form, page, d, K, V):
    """A request's K, V [n][d] in a pool with as many KV heads as the form has."""
    n, Hkv = K.shape[0], 4 if form[5] > 1 else 1
    pool = Pool([n], Hkv, page, d)
    pool.append([n], [n], *(x[:, None].expand(n, Hkv, d).contiguous() for x in (K, V)))
    return pool


def _call(form, pool, n, q):
    """q [m][heads of a KV head][d] in every request and KV head: out, lse [requests][m][KV heads][heads]."""
    kernel, m, G, dtype, wide, n_req = form
    step = _step(pool, [n], [m], wide)
    if n_req > 1:
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        step = vc.Kv8Step(step.tensors[0].repeat(n_req, 1), i32([n] * n_req), i32([m * r for r in range(n_req + 1)]),
                          m * n_req)
    with runs(kernel):
        out, lse = _run(pool, step, q.repeat(n_req, pool.Hkv, 1), True)
    return out.view(n_req, m, pool.Hkv, G, -1), lse.view(n_req, m, pool.Hkv, G)


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("page,d", [(16, 128), (64, 64)])
@pytest.mark.parametrize("big", [2.0 ** 20, 2.0 ** 30, 2.0 ** 90])
def test_a_large_value_reaches_no_row_that_does_not_see_its_page(form, page, d, big):
    # the last page holds a value of 2^20 and more: rows of the pages before give the same bits
    m, Hq, dtype = form[1:4]
    first, n = 704, 707                               # the last page's first token, in the middle of a tile
    K, V = _rand((n, d), 1, F32), _rand((n, d), 2, F32)
    q = _rand((m, Hq, d), 3, dtype).to(DEV)
    outs = []
    for x in (1.0, big):
        W = V.clone()
        W[first, 7] = x
        outs.append(_call(form, _pool(form, page, d, K, W), n, q))
    before = torch.arange(n - m, n, device=DEV) < first
    assert before.any() and not before.all()
    for a, b in zip(*outs):
        assert torch.equal(a[:, before], b[:, before])
    assert not torch.equal(outs[0][0], outs[1][0])


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("page,d", [(16, 128), (32, 64)])
@pytest.mark.parametrize("at", [(0, 32), (416, 448)], ids=str)
def test_large_values_without_weight_cost_the_others_nothing(form, page, d, at):
    # pages whose values are 2^26 times the others' and whose keys score 2^-100: their
    # contribution is 2^-74 of the others', which keep the precision of a call without them
    m, Hq, dtype = form[1:4]
    n = 700
    K, V = _rand((n, d), 1, F32), _rand((n, d), 2, F32)
    q = _rand((m, Hq, d), 3, dtype)
    q[..., 0] = 8.0
    K[..., 0] = 0.0
    V[at[0]:at[1]] *= 2.0 ** 26
    K[at[0]:at[1], 0] = -12.5 * d ** 0.5              # (a score of about -100 nats)
    pool = _pool(form, page, d, K, V)
    out, lse = _call(form, pool, n, q.to(DEV))
    Kd, Vd = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
    small = np.ones(n, bool)
    small[at[0]:at[1]] = False
    vmax = np.abs(Vd[small]).max()
    for i in sorted({0, m // 2, m - 1}):
        k = n - m + i + 1
        for j in range(Hq):
            qq = q[i:i + 1, j].double().numpy()
            ref, lref, absv = kv8.attention(qq, Kd[:k], Vd[:k], None, d ** -0.5)
            # scores: fp32 sums of d / 16 steps (twice that for two parts), scalings; probabilities to
            # fp16 (2^-11; fp32 calls twice fp16: 2^-21), what is left to the smallest of them (2^-28
            # and 2^-36 of the largest contribution a key); sums over k / 16 steps; the output's rounding
            size = (np.abs(qq[:, 1:]) @ np.abs(Kd[:k, 1:]).T * d ** -0.5).max()
            E = size * (d / 8 + 8) * 2.0 ** -23 + 2.0 ** -21
            rel = 2 * E + (2.0 ** -11 if dtype == BF else 2.0 ** -21) + (k / 8 + 40) * 2.0 ** -23
            tol = rel * absv + (1 + rel) * torch.finfo(dtype).eps / 2 * np.abs(ref) \
                + k * (2.0 ** -28 if dtype == BF else 2.0 ** -36) * vmax
            err = np.abs(out[:, i, :, j].double().cpu().numpy() - ref[0])
            assert (err <= tol[0]).all(), (i, j, float((err / tol[0]).max()))
            zerr = np.abs(lse[:, i, :, j].double().cpu().numpy() - lref[0])
            assert (zerr <= E + (k / 128 + 40) * 2.0 ** -23 + 2.0 ** -22 * abs(lref[0])).all()


@pytest.mark.parametrize("form", FORMS, ids=str)
def test_tiny_and_zero_pages_of_values_keep_their_weight(form):
    # V pages of 0, of 2^-120 and one of 2^100 beside ordinary ones: every token counts in the normaliser
    m, Hq, dtype = form[1:4]
    n, d = 400, 64
    K, V = _rand((n, d), 1, F32, 0.3), _rand((n, d), 2, F32)
    for j in range(0, n, 16):
        V[j:j + 16] *= (1.0, 0.0, 2.0 ** -120, 1.0, 2.0 ** 100 if j == 64 else 1.0)[j // 16 % 5]
    for scale in (1.0, 2.0 ** -100, 2.0 ** 20):
        pool = _pool(form, 16, d, K, V * scale)
        q = _rand((m, Hq, d), 3, dtype)
        out, lse = _call(form, pool, n, q.to(DEV))
        Kd, Vd = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
        for i in (0, m - 1):
            k = n - m + i + 1
            qq = q[i, :1].double().numpy()
            ref, lref, absv = kv8.attention(qq, Kd[:k], Vd[:k], None, d ** -0.5)
            # (as above, with sizes below 4)
            E = 4 * (d / 8 + 8) * 2.0 ** -23 + 2.0 ** -21
            rel = 2 * E + (2.0 ** -11 if dtype == BF else 2.0 ** -21) + (k / 8 + 40) * 2.0 ** -23
            vmax = np.abs(Vd[:k]).max()
            tol = rel * absv + (1 + rel) * torch.finfo(dtype).eps / 2 * np.abs(ref) \
                + k * (2.0 ** -28 if dtype == BF else 2.0 ** -36) * vmax + 2.0 ** -126
            err = np.abs(out[:, i, :, 0].double().cpu().numpy() - ref[0])
            assert (err <= tol[0]).all(), (scale, i, float((err / tol[0]).max()))
            zerr = np.abs(lse[:, i, :, 0].double().cpu().numpy() - lref[0])
            assert (zerr <= E + (k / 128 + 40) * 2.0 ** -23 + 2.0 ** -22 * abs(lref[0])).all()
