"""GPU parity of eviction by weight (viscache_kv8_evict) against the oracle: what stays, codes,
scales and weights bit for bit, and everything that is not to be touched."""
import numpy as np
import pytest
import torch

from oracle import kv8
from oracle import step as ostep
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    """Pools in shuffled pages, weights, and what is in slots that hold no token; the oracle's copy."""

    def __init__(self, lens, keep, Hkv, d, page, sink=0, recent=0, seed=1, spread=2.0, extra=0, max_keep=None):
        rng = np.random.default_rng(seed)
        need = [-(-x // page) for x in lens]
        n = sum(need) + 2
        order = rng.permutation(n)
        self.table = np.zeros((len(lens), max([1] + need) + extra), np.int32)
        at = 0
        for r, k in enumerate(need):
            self.table[r, :k] = order[at:at + k]
            at += k
        self.codes, self.scale = [], []
        for i in range(2):
            x = rng.standard_normal((n, Hkv, page, d)) * np.exp2(spread * rng.standard_normal((n, Hkv, 1, 1)))
            x *= np.exp2(rng.integers(-6, 3, (n, Hkv, page, 1)))
            s = np.array([[kv8.scale_of(np.abs(x[p, g]).max()) for g in range(Hkv)] for p in range(n)], np.float32)
            self.codes.append(kv8.encode(x / s[:, :, None, None]))
            self.scale.append(s)
        self.weights = np.exp2(3 * rng.standard_normal((n, Hkv, page))).astype(np.float32)
        self.lens, self.keep, self.Hkv, self.sink, self.recent = lens, keep, Hkv, sink, recent
        self.kept = np.full((len(lens), Hkv, max_keep or max(max(keep), 1)), -7, np.int32)

    def device(self):
        d = lambda x: torch.from_numpy(x.copy()).to(DEV)
        i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device=DEV)
        n = len(self.lens)
        self.cache = vc.Kv8Cache(d(self.codes[0]), d(self.codes[1]), d(self.scale[0]), d(self.scale[1]))
        self.step = vc.Kv8Step(d(self.table), i32(self.lens), i32(range(n + 1)), n)
        return dict(cache=self.cache, step=self.step, weights=d(self.weights), keep=i32(self.keep),
                    max_keep=self.kept.shape[2], sink=self.sink, recent=self.recent, kept=d(self.kept),
                    new_lens=torch.full((n,), -9, dtype=torch.int32, device=DEV),
                    ws=torch.empty(vc.viscache_kv8_evict_workspace_size(n, self.Hkv), dtype=torch.uint8, device=DEV))

    def oracle(self):
        return ostep.evict(self.codes, self.scale, self.table, self.lens, self.weights, self.keep, self.sink,
                           self.recent, self.kept)

    def compare(self, a, lens):
        k, v, ks, vs = (t.cpu().numpy() for t in a["cache"].tensors)
        assert a["new_lens"].tolist() == lens
        np.testing.assert_array_equal(a["kept"].cpu().numpy(), self.kept)
        np.testing.assert_array_equal(a["weights"].cpu().numpy(), self.weights)
        np.testing.assert_array_equal(ks, self.scale[0])
        np.testing.assert_array_equal(vs, self.scale[1])
        for got, want in ((k, self.codes[0]), (v, self.codes[1])):
            same = (got == want) | (((got & 127) == 127) & ((want & 127) == 127))
            assert same.all(), "%d codes differ" % (~same).sum()

    def check(self, **kw):
        a = {**self.device(), **kw}
        vc.viscache_kv8_evict(**a)
        assert vc.prunekv_get_status(a["ws"]) == vc.VC_OK
        self.compare(a, self.oracle())
        return a


CASES = [  # lens, keep, Hkv, d, page, sink, recent
    ([1], [1], 1, 64, 16, 0, 0), ([2], [1], 1, 64, 16, 0, 0), ([2], [1], 3, 128, 128, 1, 16),
    ([65, 0, 64, 63, 1], [64] * 5, 2, 128, 64, 4, 16), ([300, 17, 16, 15], [16] * 4, 4, 64, 16, 1, 4),
    ([1000, 700, 333], [250, 699, 40], 3, 128, 32, 4, 64), ([513], [512], 2, 64, 128, 0, 128),
    ([2500, 40], [1300, 0], 2, 128, 16, 0, 0), ([900, 900], [30, 800], 5, 64, 32, 40, 100),
    ([5000], [4100], 1, 128, 64, 4, 1000), ([5000], [4100], 2, 64, 16, 0, 16)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_matches_oracle(case):
    Case(*case).check()


def test_weights_of_all_kinds():
    # ties by place, infinities, NaN behind everything, zeros of both signs, negative numbers
    c = Case([400, 400], [150, 390], 3, 64, 32, 2, 5, max_keep=395)
    rng = np.random.default_rng(4)
    kinds = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, 1.0, -2.0, 1e-42, 3e38], np.float32)
    c.weights = rng.choice(kinds, c.weights.shape)
    c.check()
    c = Case([700], [300], 2, 64, 16)
    c.weights[:] = 0.0                          # all alike: the first stay, nothing moves
    a = c.check()
    assert a["kept"][0, 0].tolist() == list(range(300))


def test_values_of_all_kinds():
    # NaN codes, pages of zeros with any scale, the largest and the smallest scales
    c = Case([640], [300], 2, 64, 32, 3, 7, seed=5)
    rng = np.random.default_rng(6)
    for codes, scale in zip(c.codes, c.scale):
        codes[rng.random(codes.shape) < 0.01] = 0x7F
        codes[2] &= 0x80                        # zeros of both signs ...
        scale[2] = 2.0 ** 100                   # ... under a scale that means nothing
        codes[4] = 0
        scale[4] = 0.0
        scale[5] = 2.0 ** 120
        codes[5] = np.where((codes[5] & 127) > 0x77, 0x77, codes[5])    # 240 * 2^120 at most
        scale[6] = 2.0 ** -126
    c.check()


def test_long_requests_and_few_kept():
    # more tokens than the keys held in shared memory
    Case([30000, 24577, 24576], [500, 60, 24000], 1, 64, 128, 4, 64).check()


def test_lengths_in_place_and_again():
    c = Case([333, 90, 200], [100, 100, 100], 2, 128, 32, 4, 16)
    a = c.device()
    a["new_lens"] = a["step"].tensors[1]
    vc.viscache_kv8_evict(**a)
    c.compare(a, c.oracle())
    # what is within its budget stays as it is
    c.lens = [100, 90, 100]
    before = [t.clone() for t in a["cache"].tensors]
    vc.viscache_kv8_evict(**a)
    assert all(torch.equal(x, y) for x, y in zip(before, a["cache"].tensors))
    c.oracle()
    c.compare(a, [100, 90, 100])


def test_side_stream_and_repeatability():
    kw = dict(lens=[900, 1200, 77], keep=[300, 200, 50], Hkv=4, d=128, page=64, sink=4, recent=32)
    c, st = Case(**kw), torch.cuda.Stream()
    a, b = c.device(), c.device()
    st.wait_stream(torch.cuda.current_stream())
    vc.viscache_kv8_evict(**a, stream=st)
    st.synchronize()
    vc.viscache_kv8_evict(**b)
    c.compare(a, c.oracle())
    assert torch.equal(a["kept"], b["kept"])
    assert all(torch.equal(x, y) for x, y in zip(a["cache"].tensors, b["cache"].tensors))


def test_captured_and_replayed_with_new_lengths():
    first = Case([400, 300], [100, 90], 2, 64, 16, 2, 8, extra=6)
    a = first.device()
    keep = [t.clone() for t in a["cache"].tensors] + [a["weights"].clone(), a["kept"].clone()]
    vc.viscache_kv8_evict(**a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vc.viscache_kv8_evict(**a)
    for lens, budget in (([390, 299], [95, 100]), ([17, 250], [16, 16])):
        for t, old in zip(list(a["cache"].tensors) + [a["weights"], a["kept"]], keep):
            t.copy_(old)
        a["step"].tensors[1].copy_(torch.tensor(lens, dtype=torch.int32))
        a["keep"].copy_(torch.tensor(budget, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        assert vc.prunekv_get_status(a["ws"]) == vc.VC_OK
        c = Case([400, 300], [100, 90], 2, 64, 16, 2, 8, extra=6)
        c.lens, c.keep = lens, budget
        c.compare(a, c.oracle())


def test_bad_device_arrays_are_reported_and_the_request_left_alone():
    c = Case([200, 150], [60, 60], 2, 64, 16, 2, 8)
    a = c.device()
    a["step"].tensors[0][0, 3] = 10 ** 6
    vc.viscache_kv8_evict(**a)
    assert vc.prunekv_get_status(a["ws"]) == vc.VC_ERR_DEVICE_INDEX
    table = c.table[0].copy()
    c.lens = [0, 150]
    c.oracle()
    c.compare(a, [200, 60])
    for name, value in (("keep", -1), ("keep", 61), ("lens", -1), ("lens", 10 ** 6)):
        c = Case([200, 150], [60, 60], 2, 64, 16, 2, 8)
        a = c.device()
        (a["keep"] if name == "keep" else a["step"].tensors[1])[1] = value
        vc.viscache_kv8_evict(**a)
        assert vc.prunekv_get_status(a["ws"]) == vc.VC_ERR_DEVICE_INDEX
        assert a["new_lens"].tolist() == [60, {"keep-1": 0, "keep61": 60, "lens-1": 0, "lens1000000": 60}[name + str(value)]]


def test_binding_refuses():
    c = Case([40], [20], 2, 64, 16)
    good = c.device()
    vc.viscache_kv8_evict(**good)
    w = good["weights"]
    for kw in (dict(weights=w[:1]), dict(weights=w.double()), dict(weights=w.cpu()), dict(keep=good["keep"].long()),
               dict(keep=torch.zeros(2, dtype=torch.int32, device=DEV)), dict(kept=good["kept"][:, :1]),
               dict(max_keep=21), dict(max_keep=0), dict(new_lens=good["new_lens"].long()), dict(sink=-1), dict(recent=-1),
               dict(ws=torch.empty(100, dtype=torch.uint8, device=DEV))):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_kv8_evict(**{**good, **kw})
