"""GPU parity of the 8-bit paged cache: written (codes and scales bit for bit against the
oracle), read back, and attended over (against float64 on the oracle's values)."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2608_24063_gb300 import synth
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _rand(shape, key, dtype, scale=1.0):
    n = int(np.prod(shape))
    return synth._round(synth.normal(key, 0, max(n, 1), "cpu")[:n].view(*shape) * scale, dtype)


class Pool:
    """A cache on the device and its oracle copy: pages in a shuffled order, garbage (NaN codes,
    huge scales) in everything that was never written."""

    def __init__(self, caps, Hkv, page, d, seed=1, spare=2):
        need = [-(-c // page) for c in caps]
        n = sum(need) + spare
        order = np.random.default_rng(seed).permutation(n)
        self.table = np.zeros((len(caps), max(1, max(need))), np.int32)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = order[at:at + k]
            at += k
        self.codes = [np.full((n, Hkv, page, d), 0x7F, np.uint8) for _ in range(2)]
        self.scale = [np.full((n, Hkv), 2.0 ** 60, np.float32) for _ in range(2)]
        t = [torch.from_numpy(x.copy()).to(DEV) for x in self.codes + self.scale]
        self.cache = vc.Kv8Cache(*t)
        self.page, self.Hkv, self.d = page, Hkv, d

    def step(self, lens, rows):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        start = np.concatenate([[0], np.cumsum(rows)])
        return vc.Kv8Step(torch.from_numpy(self.table).to(DEV), i32(list(lens)), i32(start.tolist()), int(start[-1]))

    def append(self, lens, rows, K, V):
        """On the device and in the oracle's copy."""
        vc.viscache_kv8_append(self.cache, self.step(lens, rows), K.to(DEV), V.to(DEV))
        for i, x in enumerate((K, V)):
            kv8.append(self.codes[i], self.scale[i], self.table, lens, rows, x.double().numpy())

    def check(self):
        torch.cuda.synchronize()
        k, v, ks, vs = (t.cpu().numpy() for t in self.cache.tensors)
        np.testing.assert_array_equal(ks, self.scale[0])
        np.testing.assert_array_equal(vs, self.scale[1])
        for got, want in ((k, self.codes[0]), (v, self.codes[1])):
            same = got == want
            same |= ((got & 127) == 127) & ((want & 127) == 127)       # NaN of either sign
            assert same.all(), "%d codes differ" % (~same).sum()


SHAPES = [(16, 64, BF), (16, 128, F32), (32, 128, BF), (32, 64, F32), (64, 128, BF), (64, 64, BF), (128, 128, F32),
          (128, 128, BF), (128, 64, F32)]


@pytest.mark.parametrize("page,d,dtype", SHAPES, ids=str)
def test_append_matches_oracle(page, d, dtype):
    # requests of 0, 1, page - 1, page, page + 1 and many tokens, then steps that start inside
    # pages, with growing and with shrinking values
    first = [0, 1, page - 1, page, page + 1, 3 * page + 5, 2]
    pool = Pool([x + 2 * page + 9 for x in first], 3, page, d)
    K, V = _rand((sum(first), 3, d), 1, dtype), _rand((sum(first), 3, d), 2, dtype)
    K[..., ::7] *= 12
    pool.append(first, first, K, V)
    pool.check()
    lens = list(first)
    for key, (rows, scale) in enumerate([([1] * 7, 1.0), ([0, 2, 1, page, 3, page + 1, 0], 40.0), ([1] * 7, 0.01)]):
        lens = [x + m for x, m in zip(lens, rows)]
        K = _rand((sum(rows), 3, d), 10 + key, dtype, scale)
        V = _rand((sum(rows), 3, d), 20 + key, dtype, scale * 0.1)
        pool.append(lens, rows, K, V)
        pool.check()


def test_append_many_requests():
    # more requests than a warp counts at once, one row each
    n = 700
    rng = np.random.default_rng(5)
    old = rng.integers(0, 40, n).tolist()
    pool = Pool([x + 1 for x in old], 1, 16, 64)
    pool.append(old, old, _rand((sum(old), 1, 64), 3, BF), _rand((sum(old), 1, 64), 4, BF))
    rows = (rng.random(n) < 0.8).astype(int).tolist()
    pool.append([x + m for x, m in zip(old, rows)], rows, _rand((sum(rows), 1, 64), 5, BF, 3.0),
                _rand((sum(rows), 1, 64), 6, BF, 0.3))
    pool.check()


def test_append_special_values():
    d, page = 64, 16
    pool = Pool([40], 2, page, d)
    K, V = _rand((33, 2, d), 1, F32), _rand((33, 2, d), 2, F32)
    K[0, 0, :4] = torch.tensor([float("nan"), float("inf"), float("-inf"), 3.4e38])
    K[16:32] = 0.0                              # a page of zeros
    K[32, 1] = 1e-42                            # below the smallest scale
    V[3] = 1e-38
    V[20, :, ::2] = -448.0 * 2.0 ** 100
    pool.append([33], [33], K, V)
    pool.check()
    pool.append([35], [2], _rand((2, 2, d), 3, F32, 1e-44), _rand((2, 2, d), 4, F32, 2.0 ** 90))
    pool.check()


def test_append_is_idempotent_and_strided_rows_are_read_in_place():
    Hkv, d, page = 2, 128, 32
    pool = Pool([200], Hkv, page, d)
    K0, V0 = _rand((41, Hkv, d), 1, BF), _rand((41, Hkv, d), 2, BF)
    pool.append([41], [41], K0, V0)
    # rows as the compression pass leaves them, [Hkv][B][d], and a slice of a fused projection
    block = _rand((Hkv, 57, d), 3, BF, 9.0)
    fused = _rand((57, 3 * Hkv, d), 4, BF)
    K, V = block.transpose(0, 1), fused[:, 2 * Hkv:]
    for i, x in enumerate((K, V)):
        kv8.append(pool.codes[i], pool.scale[i], pool.table, [98], [57], x.double().numpy())
    step = pool.step([98], [57])
    Kd, Vd = block.to(DEV).transpose(0, 1), fused.to(DEV)[:, 2 * Hkv:]
    for _ in range(2):
        vc.viscache_kv8_append(pool.cache, step, Kd, Vd)
        pool.check()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("page,d", [(16, 128), (64, 64), (128, 128)])
def test_read_matches_oracle(page, d, dtype):
    lens = [0, 1, page + 3, 5 * page, 17]
    pool = Pool(lens, 2, page, d)
    pool.append(lens, lens, _rand((sum(lens), 2, d), 1, F32, 5.0), _rand((sum(lens), 2, d), 2, F32))
    for rows in (lens, [0, 1, 5, page + 2, 16]):
        K, V = vc.viscache_kv8_read(pool.cache, pool.step(lens, rows), dtype)
        torch.cuda.synchronize()
        for got, codes, scale in ((K, pool.codes[0], pool.scale[0]), (V, pool.codes[1], pool.scale[1])):
            want = np.concatenate([np.stack([kv8.gather(codes, scale, pool.table[r], n, g)[n - m:]
                                             for g in range(2)], 1) for r, (n, m) in enumerate(zip(lens, rows))])
            assert torch.equal(got.cpu(), torch.from_numpy(want).to(dtype))


def _attend_case(pool, lens, rows, Hq, dtype, causal, scale=0.0, qscale=1.5, seed=50, strided=False):
    """The call's outputs against the oracle on the cache's own values."""
    Hkv, d, G = pool.Hkv, pool.d, Hq // pool.Hkv
    total = sum(rows)
    q = _rand((total, Hq + (Hkv if strided else 0), d), seed, dtype, qscale)
    qd = q.to(DEV)[:, :Hq]
    lse = torch.full((total, Hq), float("nan"), device=DEV)
    out = torch.full((total, Hq, d), float("nan"), dtype=dtype, device=DEV)
    ws = torch.empty(vc.viscache_kv8_workspace_size(total, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), qd, scale, causal, out, lse, ws)
    assert vc.prunekv_get_status(ws) == vc.VC_OK
    got, z = out.double().cpu().numpy(), lse.double().cpu().numpy()
    sc = scale if scale > 0 else 1.0 / np.sqrt(d)
    q64 = q[:, :Hq].double().numpy()
    at = 0
    for r, (n, m) in enumerate(zip(lens, rows)):
        for g in range(Hkv):
            K = kv8.gather(pool.codes[0], pool.scale[0], pool.table[r], n, g)
            V = kv8.gather(pool.codes[1], pool.scale[1], pool.table[r], n, g)
            for j in range(g * G, (g + 1) * G):
                qq = q64[at:at + m, j]
                ref, lref, absv = kv8.attention(qq, K, V, n - m if causal else None, sc)
                # scores: fp32 sums of d exact products, each partial sum within 2^-23 of the
                # largest (d / 16 + 2 of them), a second fp16 part of fp32 rows within 2^-22,
                # and the scalings; a probability's relative error is that of its exponent,
                # twice (numerator and normaliser)
                size = (np.abs(qq) @ np.abs(K).T * sc).max(initial=0.0)
                E = size * (d / 16 + 6) * 2.0 ** -23 + 2.0 ** -21
                # probabilities to fp16 (2^-11) or two fp16 parts (2^-21); sums over n tokens,
                # 16 a product step, eight warps
                rel = 2 * E + (2.0 ** -11 if dtype == BF else 2.0 ** -21) + (n / 128 + 40) * 2.0 ** -23
                # the output's rounding: half the spacing of the type
                tol = rel * absv + (1 + rel) * torch.finfo(dtype).eps / 2 * np.abs(ref)
                # and what the largest value's fixed point leaves to the small ones
                tol = tol + 2.0 ** -24 * np.abs(V).max(initial=0.0)
                err = np.abs(got[at:at + m, j] - ref)
                assert (err <= tol).all(), (r, j, float((err - tol).max()), float(err.max()))
                live = np.isfinite(lref)
                np.testing.assert_array_equal(np.isneginf(z[at:at + m, j]), ~live)
                ltol = E + (n / 128 + 40) * 2.0 ** -23 + 2.0 ** -22 * np.abs(lref[live])
                assert (np.abs(z[at:at + m, j][live] - lref[live]) <= ltol).all()
                assert (got[at:at + m, j][~live] == 0).all()
        at += m
    return out, lse


def _filled(lens, Hkv, page, d, seed=1):
    pool = Pool(lens, Hkv, page, d, seed)
    K, V = _rand((sum(lens), Hkv, d), seed + 1, F32), _rand((sum(lens), Hkv, d), seed + 2, F32)
    K[..., ::33] *= 10
    at = 0
    for n in lens:
        if n:
            V[at] *= 0.01                       # the first token a sink with small values
        at += n
    pool.append(lens, lens, K, V)
    return pool


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(28, 4, 128, 64), (8, 4, 64, 16), (8, 1, 128, 128), (3, 3, 64, 32),
                                           (16, 1, 64, 64), (48, 2, 128, 16)])
def test_decode_step_matches_oracle(Hq, Hkv, d, page, dtype):
    # one row a request; lengths of 0, 1, ends inside pages and tiles, several tiles
    lens = [1, 0, 15, 16, 127, 128, 129, 700]
    pool = _filled(lens, Hkv, page, d)
    _attend_case(pool, lens, [1] * len(lens), Hq, dtype, True)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(7, 1, 128, 32), (8, 4, 64, 16), (4, 4, 128, 64)])
def test_chunks_match_oracle(Hq, Hkv, d, page, causal, dtype):
    # rows that fill and overrun row tiles; a request without rows, one whose rows are all its
    # tokens, one with more rows than tokens, one empty
    lens, rows = [300, 40, 33, 5, 0, 190], [17, 0, 33, 9, 3, 40]
    pool = _filled(lens, Hkv, page, d)
    _attend_case(pool, lens, rows, Hq, dtype, causal, strided=True)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_long_context_split_over_blocks(dtype):
    # one request's tiles over every block, and a ragged pair whose pieces meet inside blocks
    for lens in ([40000], [9000, 20011]):
        pool = _filled(lens, 1, 64, 128)
        _attend_case(pool, lens, [1] * len(lens), 5, dtype, True)


def test_many_short_requests():
    rng = np.random.default_rng(2)
    lens = rng.integers(0, 60, 300).tolist()
    pool = _filled(lens, 1, 16, 64)
    _attend_case(pool, lens, [1] * 300, 2, BF, True)


def test_scales_far_apart_and_extreme_scores():
    # pages whose values differ by 2^12 in size, scores of hundreds, an explicit scale
    lens = [400]
    pool = Pool(lens, 1, 16, 128)
    K, V = _rand((400, 1, 128), 1, F32), _rand((400, 1, 128), 2, F32)
    for j in range(0, 400, 16):
        V[j:j + 16] *= 2.0 ** ((j // 16) % 13 - 6)
    pool.append(lens, lens, K * 3, V)
    for dtype in (BF, F32):
        _attend_case(pool, lens, [3], 4, dtype, True, scale=1.0, qscale=1.0)
        _attend_case(pool, lens, [3], 4, dtype, True, qscale=1e-30)
        _attend_case(pool, lens, [3], 4, dtype, True, qscale=1e-6)


def test_nan_rows_stay_their_own():
    # a NaN query row gives NaN there and nowhere else
    lens, rows = [200, 90], [4, 1]
    pool = _filled(lens, 2, 16, 64)
    q = _rand((5, 4, 64), 9, BF).to(DEV)
    ref = vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q)
    q[2, 1, 5] = float("nan")
    got = vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q)
    assert torch.isnan(got[2, 1]).all()
    got[2, 1] = ref[2, 1]
    assert torch.equal(got, ref)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_same_call_same_bits_on_any_stream_and_in_a_graph(dtype):
    lens, rows = [5000, 333, 64], [1, 5, 2]
    pool = _filled(lens, 2, 32, 128)
    q = _rand((8, 8, 128), 4, dtype).to(DEV)
    step = pool.step(lens, rows)
    ws = torch.empty(vc.viscache_kv8_workspace_size(8, 8, 2, 128), dtype=torch.uint8, device=DEV)
    a = vc.viscache_kv8_attention(pool.cache, step, q, ws=ws)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b = vc.viscache_kv8_attention(pool.cache, step, q, ws=ws, stream=st)
    st.synchronize()
    assert torch.equal(a, b)
    # a captured call replayed with other lengths than it was captured with
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vc.viscache_kv8_attention(pool.cache, step, q, out=out, ws=ws)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, a)
    step.tensors[1].copy_(torch.tensor([1234, 7, 60], dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    want = vc.viscache_kv8_attention(pool.cache, pool.step([1234, 7, 60], rows), q)
    assert torch.equal(out, want)


def test_bad_device_arrays_are_reported_and_skipped():
    lens, rows = [100, 50], [2, 3]
    pool = _filled(lens, 2, 16, 64)
    before = [t.clone() for t in pool.cache.tensors]
    q, kv = _rand((5, 4, 64), 1, BF).to(DEV), _rand((5, 2, 64), 2, BF).to(DEV)
    ws = torch.empty(vc.viscache_kv8_workspace_size(5, 4, 2, 64), dtype=torch.uint8, device=DEV)
    good = vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q)

    def spoil(which, index, value):
        s = pool.step(lens, rows)
        s.tensors[which].view(-1)[index] = value
        return s

    width = pool.table.shape[1]
    for s in (spoil(0, width + 3, 1 << 20), spoil(0, width + 3, -1), spoil(1, 1, -5), spoil(1, 1, 10000),
              spoil(2, 2, 4000), spoil(2, 1, -7)):
        got = vc.viscache_kv8_attention(pool.cache, s, q, ws=ws)
        assert vc.prunekv_get_status(ws) == vc.VC_ERR_DEVICE_INDEX
        if s.tensors[2][1] == 2:
            assert torch.equal(got[:2], good[:2])             # the other request is untouched
        vc.viscache_kv8_read(pool.cache, s, ws=ws)
        assert vc.prunekv_get_status(ws) == vc.VC_ERR_DEVICE_INDEX
    # append: nothing of the pool changes where the page does not exist
    s = spoil(0, width + 3, 1 << 20)
    s.tensors[2].copy_(torch.tensor([0, 0, 2], dtype=torch.int32))      # only request 1 has rows, on page 3
    vc.viscache_kv8_append(pool.cache, s, kv, kv, ws=ws)
    assert vc.prunekv_get_status(ws) == vc.VC_ERR_DEVICE_INDEX
    for t, b in zip(pool.cache.tensors, before):
        assert torch.equal(t, b)
    # and the next good call clears the status
    vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q, ws=ws)
    assert vc.prunekv_get_status(ws) == vc.VC_OK


def test_more_rows_than_tokens_are_not_written():
    pool = Pool([20], 1, 16, 64)
    K, V = _rand((9, 1, 64), 1, BF), _rand((9, 1, 64), 2, BF)
    pool.append([4], [9], K, V)                  # tokens are the last four rows
    pool.check()
    out = torch.full((9, 1, 64), 7.0, dtype=BF, device=DEV)
    vc.viscache_kv8_read(pool.cache, pool.step([4], [9]), out=(out, out.clone()))
    assert (out[:5] == 7).all()


def test_rows_past_the_step_are_left_alone():
    # a padded batch: the row arrays hold more rows than the requests own
    lens, rows = [30, 40], [1, 2]
    pool = _filled(lens, 2, 16, 64)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = vc.Kv8Step(torch.from_numpy(pool.table).to(DEV), i32(lens), i32([0, 1, 3]), 6)
    q = _rand((6, 4, 64), 3, BF).to(DEV)
    out = torch.full((6, 4, 64), 9.0, dtype=BF, device=DEV)
    vc.viscache_kv8_attention(pool.cache, step, q, out=out)
    assert (out[3:] == 9).all()
    assert torch.equal(out[:3], vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q[:3].contiguous()))


def test_binding_refuses():
    pool = _filled([10], 2, 16, 64)
    step = pool.step([10], [2])
    q, kv = torch.zeros((2, 4, 64), dtype=BF, device=DEV), torch.zeros((2, 2, 64), dtype=BF, device=DEV)
    for bad in (dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(out=q.float()), dict(lse=q[..., 0])):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_kv8_attention(pool.cache, step, **{**dict(q=q), **bad})
    for K, V in ((kv[:1], kv), (kv, kv[:, :1]), (kv, kv.float()), (kv.cpu(), kv)):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_kv8_append(pool.cache, step, K, V)
    with pytest.raises(vc.VisCacheError):
        vc.viscache_kv8_read(pool.cache, step, out=(kv[:1], kv))
    with pytest.raises(TypeError):
        vc.viscache_kv8_attention(pool.cache, step, q.half())


@pytest.mark.parametrize("n,Hq,Hkv,top", [(33, 4, 1, 900), (38, 8, 4, 700), (150, 16, 1, 300), (160, 2, 1, 2000),
                                          (161, 2, 1, 500), (64, 3, 3, 1500)])
def test_more_requests_than_a_warps_lanes(n, Hq, Hkv, top):
    # units around the number of SMs, some requests empty, some without rows
    rng = np.random.default_rng(n)
    lens = rng.integers(0, top, n).tolist()
    rows = (rng.random(n) < 0.9).astype(int).tolist()
    pool = _filled(lens, Hkv, 32, 64)
    _attend_case(pool, lens, rows, Hq, BF, True)
    _attend_case(pool, lens, [3 * m for m in rows], Hq, F32, True)
