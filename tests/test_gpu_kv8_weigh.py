"""GPU parity of the attention added up for each cached token (viscache_kv8_weigh) against the
float64 oracle: few and many rows, ragged batches, padding, masks that leave rows empty."""
import numpy as np
import pytest
import torch

from oracle import kv8
from oracle import step as ostep
from paper_2608_24063_gb300 import synth
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _rand(shape, key, dtype, scale=1.0):
    n = int(np.prod(shape))
    return synth._round(synth.normal(key, 0, max(n, 1), "cpu")[:n].view(*shape) * scale, dtype)


class Case:
    """A pool in shuffled pages with NaN codes where nothing was written, a step's rows and their lse
    in float64 from the oracle's values."""

    def __init__(self, lens, rows, Hq, Hkv, d, page, dtype, causal=True, seed=1, capacity=0, scale=None, spread=0.7):
        self.lens, self.rows, self.Hq, self.Hkv, self.d, self.page = lens, rows, Hq, Hkv, d, page
        self.causal, self.scale, self.dtype = causal, scale, dtype
        rng = np.random.default_rng(seed)
        need = [-(-max(x, 0) // page) for x in lens]
        n = sum(need) + 2
        order = rng.permutation(n)
        self.table = np.zeros((len(lens), max([1, capacity] + need)), np.int32)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = order[at:at + k]
            at += k
        K = rng.standard_normal((n, Hkv, page, d)) * np.exp2(spread * rng.standard_normal((n, Hkv, 1, 1)))
        K[..., ::50] *= 6.0
        self.k_scale = np.array([[kv8.scale_of(np.abs(K[p, g]).max()) for g in range(Hkv)] for p in range(n)], np.float32)
        self.codes = kv8.encode(K / self.k_scale[:, :, None, None])
        for r, x in enumerate(lens):
            if x % page:
                self.codes[self.table[r, x // page], :, x % page:] = 0x7F
        self.weights = (rng.random((n, Hkv, page)) ** 2 * 4).astype(np.float32)
        self.q = _rand((sum(rows), Hq, d), seed, dtype)
        self.lse = self.row_lse().astype(np.float32)

    def row_lse(self):
        out = np.full((sum(self.rows), self.Hq), -np.inf)
        s = 1.0 / np.sqrt(self.d) if self.scale is None else self.scale
        G, at = self.Hq // self.Hkv, 0
        K = kv8.VALUE[self.codes] * self.k_scale[:, :, None, None].astype(np.float64)
        for r, (length, m) in enumerate(zip(self.lens, self.rows)):
            t = np.arange(max(length, 0))
            for g in range(self.Hkv if length > 0 else 0):
                k = K[self.table[r][t // self.page], g, t % self.page]
                for i in range(m):
                    sees = length - m + i + 1 if self.causal else length
                    if sees <= 0 or i < m - length:
                        continue
                    x = k[:sees] @ self.q[at + i, g * G:(g + 1) * G].double().numpy().T * s
                    top = x.max(0)
                    out[at + i, g * G:(g + 1) * G] = np.log(np.exp(x - top).sum(0)) + top
            at += m
        return out

    def want(self):
        return ostep.weigh(self.codes, self.k_scale, self.table, self.lens, self.rows, self.q.double().numpy(),
                           self.lse.astype(np.float64), self.weights, self.scale, self.causal)

    def device(self):
        d = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        codes = d(self.codes)
        self.cache = vc.Kv8Cache(codes, torch.zeros_like(codes), d(self.k_scale), torch.zeros_like(d(self.k_scale)))
        start = np.concatenate([[0], np.cumsum(self.rows)]).tolist()
        self.step = vc.Kv8Step(d(self.table), i32(list(self.lens)), i32(start), start[-1])
        return self.cache, self.step, self.q.to(DEV), d(self.lse), d(self.weights)

    def run(self, **kw):
        cache, step, q, lse, w = self.device()
        ws = torch.empty(vc.viscache_kv8_workspace_size(step.n_rows, self.Hq, self.Hkv, self.d), dtype=torch.uint8,
                         device=DEV)
        out = vc.viscache_kv8_weigh(cache, step, q, lse, w, 0.0 if self.scale is None else self.scale, self.causal,
                                    ws=ws, **kw)
        assert vc.prunekv_get_status(ws) == vc.VC_OK
        return out.cpu().numpy()

    def check(self, got=None):
        got = self.run() if got is None else got
        want = self.want()
        untouched = np.ones(want.shape, bool)
        for r, (x, m) in enumerate(zip(self.lens, self.rows)):
            if m:
                t = np.arange(x)
                untouched[self.table[r][t // self.page], :, t % self.page] = False
        assert np.array_equal(got[untouched], self.weights[untouched])
        # a term's exponent: a score of up to 40 in fp32 with the scale's rounding and the sums' cuts (2^-21 of it), ex2's
        # 2^-22; rows as fp16 or e4m3 + e5m2 parts 2^-21 of the score's largest term; sums of positive terms in fp32
        tol = 2.0 ** -15 * np.abs(want) + 1e-30
        err = np.abs(got - want)
        assert (err <= tol).all(), (err / np.maximum(np.abs(want), 1e-30)).max()


FEW = [  # lens, rows, Hq, Hkv, d, page
    ([1], [1], 1, 1, 64, 16), ([777], [1], 28, 4, 128, 64), ([1, 2, 15, 16, 17, 33, 0], [1] * 7, 8, 2, 64, 16),
    ([300, 129, 64], [1, 2, 1], 16, 2, 128, 32), ([500, 0, 131], [5, 0, 3], 8, 4, 64, 128),
    ([40, 3], [7, 1], 6, 2, 128, 16), ([260], [1], 16, 1, 64, 32), ([513, 640], [1, 1], 64, 8, 128, 64)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", FEW, ids=str)
def test_few_rows(case, causal, dtype):
    Case(*case, dtype, causal).check()


MANY = [([200], [200], 4, 2, 64, 16), ([333, 65], [90, 65], 6, 1, 128, 64), ([1000], [37], 28, 4, 128, 32),
        ([140, 0, 513, 256], [140, 0, 3, 100], 8, 2, 64, 128), ([700], [300], 2, 2, 128, 16),
        ([129, 385, 770], [20, 1, 64], 16, 2, 128, 64)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", MANY, ids=str)
def test_many_rows(case, causal, dtype):
    Case(*case, dtype, causal).check()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", [([300, 90], [2, 1], 160, 1, 64, 16), ([200], [130], 128, 1, 64, 64), ([500], [70], 65, 1, 128, 32)],
                         ids=str)
def test_wide_groups(case, dtype):
    # query heads of a group: more than a step of the many-rows kernel holds, as many as it holds, just over half
    Case(*case, dtype).check()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows", [16, 17, 33, 64, 65, 80])
def test_rows_around_the_kernels_borders(rows, dtype):
    Case([150, 333], [rows, rows], 1, 1, 128, 16, dtype).check()


@pytest.mark.parametrize("causal", [True, False])
def test_more_rows_than_tokens(causal):
    # the surplus first rows are no tokens: they add nothing, whatever their lse says
    for rows in ([6, 40], [90, 140]):
        c = Case([3, 20], rows, 4, 2, 64, 16, F32, causal)
        c.check()
        dead = ~np.isfinite(c.lse)
        c.lse[dead] = -3.0
        c.check()


def test_rows_that_see_nothing_add_nothing():
    c = Case([40, 50], [2, 3], 4, 2, 64, 16, BF)
    c.lse[1] = -np.inf
    c.check()


@pytest.mark.parametrize("rows", [1, 9, 60])
def test_a_key_that_is_not_finite(rows):
    c = Case([90], [rows], 4, 2, 64, 16, BF)
    want = c.want()
    c.codes[c.table[0, 2], 1, 5] = 0x7F             # token 37 of head 1; its rows' lse would be NaN: taken without it
    got = c.run()
    p = c.table[0, 2]
    # row i sees tokens up to 90 - rows + i: with 60 rows token 37 is seen by the rows from 7 on
    assert np.isnan(got[p, 1, 5])
    got[p, 1, 5] = want[p, 1, 5]
    assert np.allclose(got, want, rtol=2.0 ** -15)


def test_scale_and_repeatability_and_streams():
    c = Case([900, 260], [3, 2], 16, 2, 128, 64, BF, scale=0.05, capacity=40)
    c.check()
    st = torch.cuda.Stream()
    a = c.run()
    cache, step, q, lse, w = c.device()
    st.wait_stream(torch.cuda.current_stream())
    vc.viscache_kv8_weigh(cache, step, q, lse, w, 0.05, stream=st)
    st.synchronize()
    assert np.array_equal(a, w.cpu().numpy())


def test_many_requests():
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 60, 700).tolist()
    rows = (rng.random(700) < 0.7).astype(int).tolist()
    Case(lens, rows, 2, 1, 64, 16, BF).check()


@pytest.mark.parametrize("rows", [1, 48])
def test_captured_and_replayed_with_new_lengths(rows):
    lens = [200, 150, 90]
    c = Case(lens, [rows] * 3, 8, 2, 128, 16, BF, capacity=16)
    cache, step, q, lse, w = c.device()
    w0 = w.clone()
    ws = torch.empty(vc.viscache_kv8_workspace_size(step.n_rows, 8, 2, 128), dtype=torch.uint8, device=DEV)
    vc.viscache_kv8_weigh(cache, step, q, lse, w, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vc.viscache_kv8_weigh(cache, step, q, lse, w, ws=ws)
    for new in ([190, 60, 90], [48, 149, 61]):
        step.tensors[1].copy_(torch.tensor(new, dtype=torch.int32))
        c.lens = new
        c.lse = c.row_lse().astype(np.float32)
        lse.copy_(torch.from_numpy(c.lse))
        for _ in range(2):
            w.copy_(w0)
            g.replay()
            torch.cuda.synchronize()
            assert vc.prunekv_get_status(ws) == vc.VC_OK
            c.check(w.cpu().numpy())


@pytest.mark.parametrize("rows", [1, 40])
def test_bad_device_arrays_are_reported_and_skipped(rows):
    c = Case([100, 80], [rows, rows], 4, 2, 64, 16, F32)
    good = c.run()
    cache, step, q, lse, w = c.device()
    ws = torch.empty(vc.viscache_kv8_workspace_size(step.n_rows, 4, 2, 64), dtype=torch.uint8, device=DEV)
    table = step.tensors[0]
    table[0, 2] = 10 ** 6
    vc.viscache_kv8_weigh(cache, step, q, lse, w, ws=ws)
    assert vc.prunekv_get_status(ws) == vc.VC_ERR_DEVICE_INDEX
    got = w.cpu().numpy()
    p = c.table[0, 2]
    assert np.array_equal(got[p], c.weights[p])
    rest = np.arange(len(got)) != p
    assert np.array_equal(got[rest], good[rest])
    for i, value in ((1, -5), (1, 10 ** 6), (2, -1), (2, 10 ** 6)):
        _, step, _, _, w = c.device()
        step.tensors[i][0] = value
        vc.viscache_kv8_weigh(cache, step, q, lse, w, ws=ws)
        assert vc.prunekv_get_status(ws) == vc.VC_ERR_DEVICE_INDEX


def test_binding_refuses():
    c = Case([40], [2], 4, 2, 64, 16, F32)
    cache, step, q, lse, w = c.device()
    good = dict(cache=cache, step=step, q=q, lse=lse, weights=w)
    vc.viscache_kv8_weigh(**good)
    for kw in (dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(q=q[:, :3]), dict(lse=lse[:1]), dict(lse=lse.double()),
               dict(weights=w[:1]), dict(weights=w.bfloat16()), dict(weights=w.transpose(1, 2)), dict(weights=w.cpu()),
               dict(scale=-1.0), dict(ws=torch.empty(100, dtype=torch.uint8, device=DEV))):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_kv8_weigh(**{**good, **kw})
