"""GPU parity of viscache_sample against the float64 oracle: tokens equal, log probabilities close."""
import math

import numpy as np
import pytest
import torch

from oracle import step as ostep
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _logits(rows, vocab, dtype, seed, spread=2.5, best=20):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, vocab)) * spread
    for r in range(rows):
        i = rng.integers(0, vocab, min(best, vocab))
        x[r, i] += rng.uniform(4, 10, len(i))
    return torch.from_numpy(x).to(dtype)


def _check(x, u, T, k=None, p=None, m=None, device=None):
    d = lambda v, dt: None if v is None else torch.tensor(v, dtype=dt, device=DEV)
    n = x.shape[0]
    token, logprob = vc.viscache_sample(x.to(DEV) if device is None else device, d(u, F32), d(T, F32),
                                        d(k, torch.int32), d(p, F32), d(m, F32))
    token, logprob = token.tolist(), logprob.tolist()
    f = lambda v, r, none: none if v is None else float(np.float32(v[r]))
    for r in range(n):
        want = ostep.sample(x[r].double().numpy(), f(u, r, 0), f(T, r, 0), 0 if k is None else k[r], f(p, r, 1.0),
                            f(m, r, 0.0))
        assert token[r] == want[0], (r, token[r], want)
        # logf and the rounding of a number of up to 60: 2^-24 of it, a few ulp of the logarithm
        if math.isnan(want[1]):
            assert math.isnan(logprob[r])
        else:
            assert abs(logprob[r] - want[1]) <= 2.0 ** -21 * max(abs(want[1]), 2.0 ** -3), (r, logprob[r], want)
    return token


FILTERS = {"none": (None, None, None), "k": (50, None, None), "p": (None, 0.9, None), "m": (None, None, 0.02),
           "kp": (200, 0.8, None), "kpm": (50, 0.95, 0.02), "pm": (None, 0.99, 1e-4), "k1": (1, None, None),
           "p0": (None, 0.0, None), "m1": (None, None, 1.0), "wide": (10 ** 9, 0.9999, 1e-30)}


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 100, 1000, 4097, 32000, 50001, 131072])
@pytest.mark.parametrize("name", FILTERS)
def test_matches_oracle(name, vocab, dtype):
    rows = 5
    k, p, m = FILTERS[name]
    rng = np.random.default_rng(vocab)
    x = _logits(rows, vocab, dtype, vocab + len(name))
    fill = lambda v: None if v is None else [v] * rows
    _check(x, [0.0, 0.25, 0.999999] + rng.random(2).tolist(), [1.0, 0.5, 1.5, 0.05, 7.0], fill(k), fill(p), fill(m))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_rows_with_settings_of_their_own(dtype):
    n, rng = 61, np.random.default_rng(2)
    x = _logits(n, 3001, dtype, 3)
    T = rng.choice([0.0, -1.0, 0.3, 1.0, 2.0, 1e-3, 1e4], n).tolist()
    k = rng.choice([0, -5, 1, 2, 40, 2999, 3001, 5000], n).tolist()
    p = rng.choice([-1.0, 0.0, 0.1, 0.5, 0.95, 1.0, 2.0], n).tolist()
    m = rng.choice([-1.0, 0.0, 0.01, 0.3, 1.0, 3.0], n).tolist()
    _check(x, rng.random(n).tolist(), T, k, p, m)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_ties_are_cut_by_index(dtype):
    # few different logits: every cut falls among equal ones
    rng = np.random.default_rng(5)
    for vocab in (64, 5000, 40000):
        x = torch.from_numpy(rng.integers(0, 4, (8, vocab)) * 0.5).to(dtype)
        x[7] = 1.25                              # all alike
        u = rng.random(8).tolist()
        _check(x, u, [1.0] * 8, k=[1, 3, vocab // 8, vocab // 2, vocab - 1, 17, 1000, vocab // 3])
        _check(x, u, [0.7] * 8, p=[0.01, 0.2, 0.33, 0.5, 0.61, 0.75, 0.9, 0.5])
        _check(x, u, [0.7] * 8, k=[vocab // 2] * 8, p=[0.01, 0.2, 0.33, 0.5, 0.61, 0.75, 0.9, 0.5])
        _check(x, u, [0.0] * 8)


def test_logits_that_are_not_numbers():
    inf, nan = math.inf, math.nan
    x = torch.randn(8, 300)
    x[0, ::2] = -inf                            # masked
    x[1, :] = -inf                              # nothing left
    x[2, :] = nan
    x[3, 5:9] = nan
    x[4, [7, 90, 200]] = inf                    # these share everything
    x[5, :] = -inf
    x[5, 250] = -3.0e38                         # one left
    x[6, 0] = 3.0e38
    x[6, 1] = -3.0e38
    x[7, :299] = -inf
    for T in (1.0, 0.0, math.inf, math.nan, 1e-40):
        _check(x, [0.5] * 8, [T] * 8)
        _check(x, [0.9] * 8, [T] * 8, k=[2] * 8, p=[0.9] * 8, m=[0.1] * 8)


def test_numbers_outside_their_range():
    x = _logits(6, 500, F32, 9)
    _check(x, [-1.0, math.nan, 1.0, 1.5, math.inf, 0.0], [1.0] * 6)
    _check(x, [0.3] * 6, [1.0] * 6, p=[math.nan] * 6, m=[math.nan] * 6)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_strides_and_alignment(dtype):
    # rows that start at any element, with numbers around them that must not be seen
    wide = torch.full((9, 1300), 1e30, dtype=dtype)
    for off in range(0, 9):
        wide[:, off:off + 1237] = _logits(9, 1237, dtype, off)
        dev = wide.to(DEV)[:, off:off + 1237]
        _check(wide[:, off:off + 1237], [0.1 * i for i in range(9)], [1.0] * 9, k=[900] * 9, p=[0.97] * 9, device=dev)
        wide[:] = 1e30
    odd = _logits(7, 333, dtype, 4)             # dense rows of an odd length
    _check(odd, [0.3] * 7, [1.0] * 7, p=[0.9] * 7)


def test_flat_rows_of_the_largest_vocabulary():
    # every token about as likely: borders 2^-18 apart, the ones of a fine random number among them
    V = 262144
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.standard_normal((4, V)) * 0.1).float()
    _check(x, rng.random(4).tolist(), [1.0] * 4)
    _check(x, rng.random(4).tolist(), [1.0] * 4, p=[0.37] * 4)
    _check(x, rng.random(4).tolist(), [1.0] * 4, k=[200000] * 4, p=[0.9] * 4)


def test_tokens_at_the_end_of_what_is_counted():
    # thousands of tokens 2^-63.97 of the best, where a weight is nothing: they are on no list
    x = torch.full((4, 9000), -63.97 * math.log(2.0))
    x[:, 17] = 0.0
    x[:, 4000:4500] = -1.5
    _check(x, [0.001, 0.3, 0.9, 0.999], [1.0] * 4, p=[0.99999, 0.9999999, 0.5, 0.99])
    _check(x, [0.001, 0.3, 0.9, 0.999], [1.0] * 4, k=[1, 500, 501, 8000], p=[0.99999, 1.0, 0.5, 0.99])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1500, 262144])
def test_lists_of_every_length(vocab, dtype):
    # what top-k keeps is put in order: lengths around each power of two, with ties, drawn at both ends and between
    ks = [k for n in (2, 4, 32, 64, 128, 256, 512, 1024) for k in (n - 1, n, n + 1)]
    u = np.random.default_rng(9).random(len(ks))
    u[::5], u[1::5] = 0.0, 0.9999999
    x = _logits(len(ks), vocab, dtype, 10, spread=1.0)
    if dtype == F32:
        x[::2] = (x[::2] * 16).round() / 16
    _check(x, u.tolist(), [1.0, 8.0] * (len(ks) // 2), ks)
    _check(x, u.tolist(), [1.0, 8.0] * (len(ks) // 2), ks, [0.97, 0.5, 0.9999] * (len(ks) // 3))


@pytest.mark.parametrize("p", [None, 0.9])
def test_long_rows_of_every_range(p):
    # rows long enough for the weights of bf16 logits to be looked up: signs, ranges and temperatures of every kind
    vocab, rng = 131072, np.random.default_rng(12)
    base = rng.standard_normal(vocab)
    rows = [base * 3, -np.abs(base) - 5, base * 1e-3, base * 1e-20, np.abs(base) * 100, base * 0 - 7, base * 1e30,
            base * 0.01 + 50, base.copy(), base.copy(), base * 3 - 60, np.abs(base) * 1e-39, base * 3, base * 3]
    rows[8][rng.random(vocab) < 0.9] = -math.inf
    rows[9][rng.random(vocab) < 0.9] = float(torch.finfo(BF).min)
    T = [1.0, 0.7, 1e-3, 3e-21, 40.0, 1.0, 1e30, 0.02, 1.3, 1.3, 2.0, 1e-39, 1e5, 1e38]
    x = torch.from_numpy(np.stack(rows)).to(BF)
    n = len(rows)
    _check(x, rng.random(n).tolist(), T, None, None if p is None else [p] * n)
    _check(x, rng.random(n).tolist(), T, None, None if p is None else [p] * n, [1e-5] * n)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_temperatures_below_the_least(dtype):
    # a positive temperature below 2^-127 counts as 2^-127: logits of that size tell them apart
    x = (torch.randn(12, 300, dtype=torch.float64, generator=torch.Generator().manual_seed(6)) * 1e-38).to(dtype)
    T = [1e-45, 1e-42, 1e-39, 4e-39, 5.8e-39, 2.0 ** -127, 6e-39, 1e-38, 1e-37, 1e-45, 1e-40, 2.0 ** -126]
    _check(x, [(i + 0.5) / 12 for i in range(12)], T)
    _check(x, [(i + 0.5) / 12 for i in range(12)], T, p=[0.8] * 12)


def test_the_share_of_each_token():
    # u walks over [0, 1): how often a token comes is its probability, to one step
    x = torch.tensor([[1.0, 0.0, -1.0, 2.0, 0.5]])
    n = 4096
    u = ((torch.arange(n) + 0.5) / n).to(DEV)
    token, _ = vc.viscache_sample(x.expand(n, 5).contiguous().to(DEV), u, torch.ones(n, device=DEV))
    want = torch.softmax(x[0].double(), 0) * n
    assert ((torch.bincount(token.cpu(), minlength=5) - want).abs() <= 1.0).all()


def test_streams_graphs_and_optional_outputs():
    x, u = _logits(40, 9000, BF, 1).to(DEV), torch.rand(40, device=DEV)
    T, p = torch.full((40,), 0.8, device=DEV), torch.full((40,), 0.9, device=DEV)
    a = vc.viscache_sample(x, u, T, top_p=p)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b = vc.viscache_sample(x, u, T, top_p=p, stream=st)
    st.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    token, logprob = torch.empty_like(a[0]), torch.empty_like(a[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vc.viscache_sample(x, u, T, top_p=p, token=token, logprob=logprob)
    u.uniform_()
    x.copy_(_logits(40, 9000, BF, 7))
    g.replay()
    torch.cuda.synchronize()
    c = vc.viscache_sample(x, u, T, top_p=p)
    assert torch.equal(c[0], token) and torch.equal(c[1], logprob) and not torch.equal(a[0], token)
    vc.viscache_sample(x[:0], u[:0], T[:0])


def test_binding_refuses():
    x, one = torch.zeros((4, 100), device=DEV), torch.ones(4, device=DEV)
    good = dict(logits=x, u=one, temperature=one)
    vc.viscache_sample(**good)
    for kw in (dict(logits=x[0]), dict(logits=x.t()), dict(logits=x.cpu()), dict(u=one[:3]), dict(u=one.double()),
               dict(temperature=one.cpu()), dict(top_k=one), dict(top_p=one.bfloat16()), dict(min_p=one[None]),
               dict(token=one), dict(logprob=one.int()), dict(u=None), dict(temperature=None)):
        with pytest.raises((vc.VisCacheError, AttributeError)):
            vc.viscache_sample(**{**good, **kw})
    with pytest.raises(TypeError):
        vc.viscache_sample(**{**good, "logits": x.half()})
