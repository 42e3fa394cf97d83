"""GPU parity of attention over the 8-bit paged cache with many query rows a request, against
the float64 oracle on sampled rows, and against fp32 rows of the same values.  The block
table's width stands for the lengths where a call chooses between its kernels, so every
case runs on both: with the table as wide as its pages, and much wider."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV, Pool, _filled, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[False, True], ids=["narrow", "wide"])
def wide(request):
    return request.param


def _step(pool, lens, rows, wide):
    step = pool.step(lens, rows)
    if not wide:
        return step
    # entries past a request's pages are not read: no page has this number
    table = torch.full((len(lens), 400000 // pool.page), -7, dtype=torch.int32, device=DEV)
    table[:, :pool.table.shape[1]] = step.tensors[0]
    return vc.Kv8Step(table, step.tensors[1], step.tensors[2], step.n_rows)


def test_every_kernel_runs():
    pool = _filled([300, 40], 1, 64, 128)
    q = _rand((40, 4, 128), 1, BF).to(DEV)
    big = _rand((600, 8, 128), 1, BF).to(DEV)
    pools = (pool, [300, 40], [20, 20]), (_filled([700], 1, 64, 128), [700], [600])
    for (p, lens, rows), x, is_wide, name in ((pools[0], q, False, "kv8_attn"), (pools[0], q, True, "kv8_attn_tc1"),
                                              (pools[0], q.float(), False, "kv8_attn"),
                                              (pools[0], q.float(), True, "kv8_attn_tc1"),
                                              (pools[1], big, True, "kv8_attn_tc2"),
                                              (pools[1], big.float(), True, "kv8_attn_tc1")):
        vc.viscache_profile_enable(True)
        try:
            _run(p, _step(p, lens, rows, is_wide), x, True)
            assert list(vc.viscache_profile_read()) == [name]
        finally:
            vc.viscache_profile_enable(False)


def _run(pool, step, q, causal, scale=0.0):
    total, Hq, d = q.shape
    lse = torch.full((total, Hq), float("nan"), device=DEV)
    out = torch.full((total, Hq, d), float("nan"), dtype=q.dtype, device=DEV)
    ws = torch.empty(vc.viscache_kv8_workspace_size(total, Hq, pool.Hkv, d), dtype=torch.uint8, device=DEV)
    ws.fill_(0xA5)
    vc.viscache_kv8_attention(pool.cache, step, q, scale, causal, out, lse, ws)
    assert vc.prunekv_get_status(ws) == vc.VC_OK
    return out, lse


def check(pool, lens, rows, Hq, causal, wide, scale=0.0, qscale=1.5, sample=7, seed=60, dtype=BF):
    """Rows of the call against the oracle: a few of each request, the first, the last and those
    at row-tile ends among them."""
    Hkv, d, G = pool.Hkv, pool.d, Hq // pool.Hkv
    q = _rand((sum(rows), Hq + Hkv, d), seed, dtype, qscale)
    out, lse = _run(pool, _step(pool, lens, rows, wide), q.to(DEV)[:, :Hq], causal, scale)
    got, z = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(got).all()
    sc = scale if scale > 0 else 1.0 / np.sqrt(d)
    q64 = q[:, :Hq].double().numpy()
    rng = np.random.default_rng(seed)
    at = 0
    for r, (n, m) in enumerate(zip(lens, rows)):
        pick = sorted({0, m - 1, 128 // G, 256 // G} | set(rng.integers(0, m, sample).tolist())) if m else []
        pick = [i for i in pick if i < m]
        for g in range(Hkv if pick else 0):
            K = kv8.gather(pool.codes[0], pool.scale[0], pool.table[r], n, g)
            V = kv8.gather(pool.codes[1], pool.scale[1], pool.table[r], n, g)
            vmax = np.abs(V).max(initial=0.0)
            for j in range(g * G, (g + 1) * G):
                for i in pick:
                    k = n if not causal else min(n, max(0, n - m + i + 1))
                    qq = q64[at + i:at + i + 1, j]
                    ref, lref, absv = kv8.attention(qq, K[:k], V[:k], None, sc)
                    # scores: d / 16 fp32 sums of products, scalings; probabilities to fp16
                    # (2^-11), those below 2^-17 of the reference to 2^-28 of it; sums over k / 16
                    # product steps; the output's rounding
                    size = (np.abs(qq) @ np.abs(K[:k]).T * sc).max(initial=0.0)
                    if dtype == BF:
                        E = size * (d / 16 + 6) * 2.0 ** -23 + 2.0 ** -21
                        rel = 2 * E + 2.0 ** -11 + (k / 16 + 40) * 2.0 ** -23
                        tol = rel * absv + (1 + rel) * 2.0 ** -8 * np.abs(ref) + k * 2.0 ** -28 * vmax
                    else:
                        # fp32 rows: two fp16 parts of rows and probabilities (2^-22 each), so
                        # twice the product steps; a probability's second part ends at 2^-25 of
                        # 2^12 (2^-37 a key), a value's fp16 number at 2^-25 of its tile's scale
                        # (under 2^-32 of the largest value)
                        E = size * (d / 8 + 8) * 2.0 ** -23 + 2.0 ** -21
                        rel = 2 * E + 2.0 ** -21 + (k / 8 + 40) * 2.0 ** -23
                        tol = rel * absv + (1 + rel) * 2.0 ** -24 * np.abs(ref) + (k * 2.0 ** -36 + 2.0 ** -32) * vmax
                    err = np.abs(got[at + i, j] - ref[0])
                    assert (err <= tol[0]).all(), (r, i, j, float((err - tol[0]).max()), float(err.max()))
                    if k == 0:
                        assert np.isneginf(z[at + i, j])
                    else:
                        ltol = E + (k / 128 + 40) * 2.0 ** -23 + 2.0 ** -22 * abs(lref[0])
                        assert abs(z[at + i, j] - lref[0]) <= ltol
        at += m
    return out, lse


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(28, 4, 128, 64), (8, 4, 64, 16), (16, 1, 64, 128), (2, 2, 128, 32),
                                           (24, 1, 128, 16)])
def test_chunks_match_oracle(Hq, Hkv, d, page, causal, wide, dtype):
    # one and two row tiles of a unit, units that end inside them, requests without rows, all of
    # whose tokens are rows, with more rows than tokens
    lens, rows = [700, 40, 300, 60, 0, 513], [129, 0, 300, 77, 65, 400]
    check(_filled(lens, Hkv, page, d), lens, rows, Hq, causal, wide, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_long_chunks_match_oracle(wide, dtype):
    # at least 512 packed rows a request on average: units of 256 rows in the wide case, whole and
    # partial ones, a request without rows, rows without tokens
    lens, rows = [1500, 40, 700, 513], [300, 0, 259, 700]
    check(_filled(lens, 2, 64, 128), lens, rows, 8, True, wide, sample=4, dtype=dtype)
    lens, rows = [2900, 3], [330, 3]
    check(_filled(lens, 1, 16, 64), lens, rows, 16, False, wide, sample=4, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_units_split_over_blocks(wide, dtype):
    # few units and long contexts: every unit's tiles lie on many blocks
    lens, rows = [20000, 3001], [40, 17]
    check(_filled(lens, 1, 64, 128), lens, rows, 4, True, wide, dtype=dtype)
    lens, rows = [9000], [300]
    check(_filled(lens, 1, 16, 64), lens, rows, 2, True, wide, sample=3, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_more_units_than_blocks(wide, dtype):
    rng = np.random.default_rng(8)
    rows = rng.integers(1, 150, 40).tolist()
    lens = [m + int(x) for m, x in zip(rows, rng.integers(0, 300, 40))]
    check(_filled(lens, 4, 32, 128), lens, rows, 8, True, wide, sample=2, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_rising_maxima_and_scales(wide, dtype):
    # scores that rise by hundreds along the tokens and V pages of growing size: O is rescaled
    # again and again; then the other way round
    n = 1200
    for flip in (False, True):
        pool = Pool([n], 1, 16, 128)
        K, V = _rand((n, 1, 128), 1, torch.float32), _rand((n, 1, 128), 2, torch.float32)
        size = torch.linspace(0.2, 6.0, n)[:, None, None]
        grow = 2.0 ** torch.div(torch.arange(n), 100, rounding_mode="floor")[:, None, None]
        K, V = K * (size.flip(0) if flip else size), V * (grow.flip(0) if flip else grow)
        pool.append([n], [n], K, V)
        for rows in (90, 130):                  # 360 and 520 rows of the KV head
            check(pool, [n], [rows], 4, True, wide, scale=0.5, dtype=dtype)
            check(pool, [n], [rows], 4, True, wide, qscale=1e-20, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_zero_pages_and_zero_rows(wide, dtype):
    pool = Pool([400], 2, 16, 64)
    K, V = _rand((400, 2, 64), 1, torch.float32), _rand((400, 2, 64), 2, torch.float32)
    K[0:160] = 0
    V[128:272] = 0
    K[320:] = 0
    pool.append([400], [400], K, V)
    for rows in (100, 260):                     # 200 and 520 rows of a KV head
        check(pool, [400], [rows], 4, True, wide, dtype=dtype)
        check(pool, [400], [rows], 4, True, wide, qscale=0.0, dtype=dtype)


def test_paths_agree_and_calls_repeat(wide):
    # the same rows through the many-rows path (one call) and the few-rows path (fp32 rows)
    lens, rows = [900, 333], [200, 150]
    pool = _filled(lens, 2, 64, 128)
    q = _rand((350, 8, 128), 5, BF).to(DEV)
    a, la = _run(pool, _step(pool, lens, rows, wide), q, True)
    b, lb = _run(pool, _step(pool, lens, rows, wide), q, True)
    assert torch.equal(a, b) and torch.equal(la, lb)
    f, lf = _run(pool, _step(pool, lens, rows, wide), q.float(), True)
    # within the output's rounding and the fp16 probabilities' (2^-11 of sum p |V| <= max |V|),
    # and the scores' error: sums of up to size = sum |q| |k| * scale, as in check()
    K, V = (np.abs(kv8.VALUE[c]) * x[..., None, None] for c, x in zip(pool.codes, pool.scale))
    vmax, kmax = np.nanmax(V[V < 1e6]), np.nanmax(K[K < 1e6])
    E = float(q.float().abs().sum(-1).max()) * kmax / 128 ** 0.5 * 14 * 2.0 ** -23
    assert ((a.float() - f).abs() <= 2.0 ** -8 * f.abs() + (2.0 ** -10 + 4 * E) * vmax).all()
    assert ((la - lf).abs() <= 2 * E + 1e-5).all()


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_rows_keep_their_precision_over_long_contexts(wide, d):
    # as a whole: exponentials within 2^-22, their exponents (up to 2^4) within 2^-21, scores of
    # size 2^3 summed within 2^-22 of them, the sum of a few tiles cut off at 2^-26 a step
    # (2^-20 for 64), fp32 sums of the rest: under 2^-18 of the output's norm together
    n, m = 20000, 40
    pool = _filled([n], 1, 64, d)
    q = _rand((m, 4, d), 9, torch.float32)
    out, _ = _run(pool, _step(pool, [n], [m], wide), q.to(DEV), False)
    K, V = (kv8.gather(c, s, pool.table[0], n, 0) for c, s in zip(pool.codes, pool.scale))
    ref = kv8.attention(q.double().numpy().reshape(m * 4, d), K, V, None, d ** -0.5)[0].reshape(m, 4, d)
    err = np.linalg.norm(out.double().cpu().numpy() - ref) / np.linalg.norm(ref)
    assert err <= 2.0 ** -18, err


@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page,n,m", [(8, 2, 128, 64, 900, 300), (4, 1, 64, 16, 500, 500), (2, 2, 128, 128, 260, 5),
                                               (32, 2, 128, 32, 700, 90), (4, 2, 64, 32, 6000, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(Hq, Hkv, d, page, n, m, dtype, wide):
    # keys and values of tokens that are not finite: rows before them are what they would be without
    # them, and a row that sees one is NaN: everywhere for a key, in the value's dimensions for a value
    K, V = (_rand((n, Hkv, d), k, torch.float32, 2.0) for k in (1, 2))
    bad = K.clone(), V.clone()
    first_k, first_v, second_v = n - m // 2, n - m // 3 - 1, n - 2
    bad[0][first_k, 0, 3] = float("inf")
    bad[1][first_v, Hkv - 1, 5] = float("nan")
    bad[1][second_v, Hkv - 1, d - 1] = float("-inf")
    # (finite stand-ins that leave the pages' scales as they are)
    K[first_k, 0, 3] = V[first_v, Hkv - 1, 5] = V[second_v, Hkv - 1, d - 1] = 0.0
    q = _rand((m, Hq, d), 3, dtype).to(DEV)
    outs = []
    for k, v in ((K, V), bad):
        pool = Pool([n], Hkv, page, d)
        pool.append([n], [n], k, v)
        pool.check()
        outs.append(_run(pool, _step(pool, [n], [m], wide), q, True))
    (out, lse), (got, zgot) = outs
    G, own = Hq // Hkv, torch.arange(n - m, n, device=DEV)
    want, zwant = out.clone(), lse.clone()
    sees = own >= first_k
    want[sees, :G], zwant[sees, :G] = float("nan"), float("nan")
    want[own >= first_v, (Hkv - 1) * G:, 5] = float("nan")
    want[own >= second_v, (Hkv - 1) * G:, d - 1] = float("nan")
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isnan(zgot), torch.isnan(zwant))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert torch.equal(torch.nan_to_num(zgot), torch.nan_to_num(zwant))
