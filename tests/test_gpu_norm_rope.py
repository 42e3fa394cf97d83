"""GPU parity of heads normed and rotated in one pass, and of the gradient, against the float64
oracle; the gradient against differences too."""
import numpy as np
import pytest
import torch

from oracle import step as ostep
from paper_2608_24063_gb300 import synth
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def _rand(shape, key, dtype):
    return synth._round(synth.normal(key, 0, int(np.prod(shape)), "cpu").view(*shape), dtype)


# rows, Hq, Hkv, d, sections, order, pairing: the smallest, odd rows, rotated parts of a head, no key heads,
# more heads than a block works on at once, more rows than the gradient's blocks
CASES = [(1, 1, 1, 64, (8,), "sectioned", "halves"), (1, 28, 4, 128, (16, 24, 24), "sectioned", "halves"),
         (37, 8, 4, 64, (12, 10, 10), "interleaved", "adjacent"), (130, 3, 1, 128, (24, 20, 20), "interleaved", "halves"),
         (33, 9, 3, 128, (8, 4, 4), "sectioned", "halves"), (9, 5, 0, 64, (4, 2, 1, 1), "sectioned", "adjacent"),
         (2600, 3, 2, 64, (12, 10, 10), "sectioned", "adjacent"), (77, 64, 8, 128, (16, 24, 24), "interleaved", "halves")]


def _inputs(case, dtype):
    rows, Hq, Hkv, d, sec, order, pairing = case
    x = _rand((rows, Hq + 2 * Hkv, d), 11 + rows, torch.float32)
    x *= torch.exp2(torch.arange(Hq + 2 * Hkv).float() % 7 - 3)[:, None]
    w = 1.0 + 0.3 * _rand((2, d), 5, torch.float32)
    pos = np.random.default_rng(rows).integers(-4000, 1 << 17, (len(sec), rows)).astype(np.int32)
    rope = vc.make_rope(sec, 1e6, interleaved=order == "interleaved", adjacent=pairing == "adjacent")
    return synth._round(x, dtype), synth._round(w, dtype), pos, rope


def _close(got, want, size, dtype):
    """Within the sums' 2^-20 of `size` (d terms of 2^-24, rsqrt's 2 ulp, the angle's 2^-25 turn and sincospi: under
    2^-20 together), and half a step of the type."""
    got = got.double().cpu().numpy()
    tol = 2.0 ** -19 * size + (2.0 ** -8 * np.abs(want) if dtype == BF else 0.0)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.abs(got - want)[bad].max(), bad.sum())


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward_matches_oracle(case, dtype):
    rows, Hq, Hkv, d, sec, order, pairing = case
    x, w, pos, rope = _inputs(case, dtype)
    xd, wd = x.to(DEV), w.to(DEV)
    q, k = xd[:, :Hq], xd[:, Hq:Hq + Hkv]            # slices of a fused projection
    qo, ko = vc.viscache_norm_mrope(rope, torch.from_numpy(pos).to(DEV), q, k if Hkv else None, wd[0],
                                    wd[1] if Hkv else None, EPS)
    for got, lo, hi, i in ((qo, 0, Hq, 0), (ko, Hq, Hq + Hkv, 1)):
        if got is not None:
            want = ostep.norm_mrope(x[:, lo:hi].double().numpy(), w[i].double().numpy(), pos.astype(np.int64), sec, 1e6,
                                    EPS, order, pairing)
            _close(got, want, np.abs(want).max(-1, keepdims=True), dtype)
    assert torch.equal(xd.cpu(), x)
    # in place, and again: the same bits
    vc.viscache_norm_mrope(rope, torch.from_numpy(pos).to(DEV), q, k if Hkv else None, wd[0], wd[1] if Hkv else None,
                           EPS, q_out=q, k_out=k if Hkv else None)
    assert torch.equal(q, qo) and (ko is None or torch.equal(k, ko))
    assert torch.equal(xd[:, Hq + Hkv:].cpu(), x[:, Hq + Hkv:])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient_matches_oracle(case, dtype):
    rows, Hq, Hkv, d, sec, order, pairing = case
    x, w, pos, rope = _inputs(case, dtype)
    dy = _rand((rows, Hq + Hkv, d), 91, dtype)
    xd, wd, yd = x.to(DEV), w.to(DEV), dy.to(DEV)
    posd = torch.from_numpy(pos).to(DEV)
    q, k = xd[:, :Hq], xd[:, Hq:Hq + Hkv] if Hkv else None
    args = (rope, posd, q, k, yd[:, :Hq], yd[:, Hq:] if Hkv else None, wd[0], wd[1] if Hkv else None, EPS)
    got = vc.viscache_norm_mrope_grad(*args)
    again = vc.viscache_norm_mrope_grad(*args)
    for g, lo, hi, i in ((0, 0, Hq, 0), (1, Hq, Hq + Hkv, 1)):
        if got[g] is None:
            continue
        X, Y, W = x[:, lo:hi].double().numpy(), dy[:, lo:hi].double().numpy(), w[i].double().numpy()
        dx, dw = ostep.norm_mrope_grad(X, Y, W, pos.astype(np.int64), sec, 1e6, EPS, order, pairing)
        # dx's terms are r h and r n mean(h n): their size is r's times the largest |h| (mean |n| <= 1)
        r = 1.0 / np.sqrt((X * X).mean(-1, keepdims=True) + EPS)
        n = np.abs(X * r).max(-1, keepdims=True)
        size = r * np.abs(W).max() * np.abs(Y).max(-1, keepdims=True) * 1.5 * (1.0 + n)
        _close(got[g], dx, size, dtype)
        # the sum's terms: each within 2^-20, added up in fp32 in pieces
        total = (np.abs(Y).max(-1, keepdims=True) * 1.5 * np.abs(X * r)).sum((0, 1))
        err = np.abs(got[g + 2].double().cpu().numpy() - dw)
        assert (err <= 2.0 ** -19 * (total + 1e-9)).all(), (err / total).max()
        assert torch.equal(got[g], again[g]) and torch.equal(got[g + 2], again[g + 2])
    # in place over the outputs' gradients, then over the inputs
    a, b = yd.clone(), xd.clone()
    vc.viscache_norm_mrope_grad(rope, posd, q, k, a[:, :Hq], a[:, Hq:] if Hkv else None, *args[6:],
                                q_grad=a[:, :Hq], k_grad=a[:, Hq:] if Hkv else None)
    vc.viscache_norm_mrope_grad(rope, posd, b[:, :Hq], b[:, Hq:Hq + Hkv] if Hkv else None, *args[4:],
                                q_grad=b[:, :Hq], k_grad=b[:, Hq:Hq + Hkv] if Hkv else None)
    assert torch.equal(a[:, :Hq], got[0]) and torch.equal(b[:, :Hq], got[0])
    if Hkv:
        assert torch.equal(a[:, Hq:], got[1]) and torch.equal(b[:, Hq:Hq + Hkv], got[1])
    assert torch.equal(b[:, Hq + Hkv:].cpu(), x[:, Hq + Hkv:])


def test_gradient_against_differences():
    rows, H, d, sec = 21, 5, 64, (12, 10, 10)
    x, dy = _rand((rows, H, d), 31, F32), _rand((rows, H, d), 32, F32)
    w = 1.0 + 0.3 * _rand((d,), 33, F32)
    pos = np.random.default_rng(8).integers(0, 9000, (3, rows)).astype(np.int32)
    rope = vc.make_rope(sec, 1e4, interleaved=True)
    dx, _, dw, _ = vc.viscache_norm_mrope_grad(rope, torch.from_numpy(pos).to(DEV), x.to(DEV), None, dy.to(DEV), None,
                                               w.to(DEV), None, EPS)
    X, W, Y = x.double().numpy(), w.double().numpy(), dy.double().numpy()
    loss = lambda a, b: (ostep.norm_mrope(a, b, pos, sec, 1e4, EPS, "interleaved") * Y).sum()
    rng = np.random.default_rng(9)
    v, u = rng.standard_normal(X.shape), rng.standard_normal(d)
    h = 1e-4
    diff = (loss(X + h * v, W + h * u) - loss(X - h * v, W - h * u)) / (2 * h)
    got = (dx.double().cpu().numpy() * v).sum() + (dw.double().cpu().numpy() * u).sum()
    # each of 6720 values of dx within 2^-19 of about 10, of 64 of dw within 2^-19 of 200 (a random direction adds their
    # roots), and the differences' own h^2 times third derivatives
    assert abs(got - diff) <= 2.0 ** -19 * 10 * np.abs(v).sum() + 1e-6 * abs(diff)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_rows_of_any_size(dtype):
    # zeros, the smallest and the largest numbers of the type, infinities and NaN in heads of their own
    d = 128
    x = torch.zeros(6, 2, d)
    x[1] = _rand((2, d), 3, F32) * 2.0 ** -60
    x[2] = _rand((2, d), 4, F32) * 2.0 ** 123
    x[3] = _rand((2, d), 5, F32)
    x[3, 0, 7] = float("inf")
    x[4] = _rand((2, d), 6, F32)
    x[4, 1, 9] = float("nan")
    x[5] = _rand((2, d), 7, F32) * 2.0 ** -5
    x = synth._round(x, dtype)
    w = torch.ones(d, dtype=dtype)
    pos = np.zeros((1, 6), np.int32)
    rope = vc.make_rope((32,), 1e4)                          # half of a head's values are normed alone
    y, _ = vc.viscache_norm_mrope(rope, torch.from_numpy(pos).to(DEV), x.to(DEV), None, w.to(DEV), None, EPS)
    with np.errstate(over="ignore"):
        want = ostep.norm_mrope(x.double().numpy(), np.ones(d), pos, (32,), 1e4, EPS)
    y = y.double().cpu().numpy()
    ok = np.isfinite(x.double().numpy()).all(-1)
    assert np.isfinite(y[ok]).all()
    tol = (2.0 ** -8 if dtype == BF else 2.0 ** -20) * np.abs(want[ok]).max(-1, keepdims=True) + 1e-30
    assert (np.abs(y[ok] - want[ok]) <= tol).all()
    assert np.isnan(y[3, 0, 7]) and np.isnan(y[4, 1, 9])


def test_gradient_of_large_rows():
    d = 64
    x = _rand((3, 2, d), 4, F32) * torch.tensor([1.0, 2.0 ** 66, 2.0 ** 110])[:, None, None]
    dy = _rand((3, 2, d), 5, F32)
    w = 1.0 + 0.3 * _rand((d,), 6, F32)
    pos = np.arange(3, dtype=np.int32)[None]
    rope = vc.make_rope((32,), 1e4)
    dx, _, dw, _ = vc.viscache_norm_mrope_grad(rope, torch.from_numpy(pos).to(DEV), x.to(DEV), None, dy.to(DEV), None,
                                               w.to(DEV), None, EPS)
    want, ww = ostep.norm_mrope_grad(x.double().numpy(), dy.double().numpy(), w.double().numpy(), pos, (32,), 1e4, EPS)
    err = np.abs(dx.double().cpu().numpy() - want)
    assert (err <= 2.0 ** -18 * np.abs(want).max(-1, keepdims=True)).all()
    assert (np.abs(dw.double().cpu().numpy() - ww) <= 2.0 ** -18 * 24).all()     # 6 terms of at most about 4


def test_no_rows_and_a_side_stream():
    rope = vc.make_rope((32,), 1e4)
    w = torch.ones(64, device=DEV)
    none = torch.empty((0, 2, 64), device=DEV)
    pos = torch.empty((1, 0), dtype=torch.int32, device=DEV)
    out = vc.viscache_norm_mrope_grad(rope, pos, none, none, none, none, w, w)
    assert not out[2].any() and not out[3].any()
    vc.viscache_norm_mrope(rope, pos, none, none, w, w)
    x = _rand((300, 6, 64), 77, BF).to(DEV)
    pos = torch.arange(300, dtype=torch.int32, device=DEV)[None]
    w = w.bfloat16()
    a, _ = vc.viscache_norm_mrope(rope, pos, x, None, w, None)
    ga = vc.viscache_norm_mrope_grad(rope, pos, x, None, a, None, w, None)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b, _ = vc.viscache_norm_mrope(rope, pos, x, None, w, None, stream=st)
    gb = vc.viscache_norm_mrope_grad(rope, pos, x, None, b, None, w, None, stream=st)
    st.synchronize()
    assert torch.equal(a, b) and torch.equal(ga[0], gb[0]) and torch.equal(ga[2], gb[2])


def test_captured_and_replayed_with_new_rows():
    rope = vc.make_rope((16, 24, 24), 1e6)
    w = (1.0 + 0.3 * _rand((2, 128), 5, F32)).bfloat16().to(DEV)
    x, dy = _rand((40, 10, 128), 1, BF).to(DEV), _rand((40, 8, 128), 2, BF).to(DEV)
    pos = torch.arange(120, dtype=torch.int32, device=DEV).view(3, 40)
    ws = torch.empty(vc.viscache_norm_mrope_grad_workspace_size(40, 6, 2, 128), dtype=torch.uint8, device=DEV)
    grads = [torch.empty_like(x[:, :6].contiguous()), torch.empty_like(x[:, :2].contiguous()),
             torch.empty(128, device=DEV), torch.empty(128, device=DEV)]
    outs = [torch.empty_like(g) for g in grads[:2]]

    def call():
        vc.viscache_norm_mrope(rope, pos, x[:, :6], x[:, 6:8], w[0], w[1], q_out=outs[0], k_out=outs[1])
        vc.viscache_norm_mrope_grad(rope, pos, x[:, :6], x[:, 6:8], dy[:, :6], dy[:, 6:], w[0], w[1], q_grad=grads[0],
                                    k_grad=grads[1], q_weight_grad=grads[2], k_weight_grad=grads[3], ws=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    x.copy_(_rand((40, 10, 128), 7, BF))
    pos.add_(900)
    g.replay()
    torch.cuda.synchronize()
    seen = [t.clone() for t in outs + grads]
    call()
    assert all(torch.equal(a, b) for a, b in zip(seen, outs + grads))


def test_binding_refuses():
    x, w = torch.zeros((4, 2, 64), device=DEV), torch.ones(64, device=DEV)
    pos = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    rope = vc.make_rope((32,), 1e4)
    good = dict(rope=rope, positions=pos, q=x, k=x, q_weight=w, k_weight=w)
    vc.viscache_norm_mrope(**good)
    bad = (dict(positions=pos.long()), dict(positions=pos[:, :3]), dict(q=x.transpose(1, 2)), dict(k=x[:3]),
           dict(k=x.bfloat16()), dict(q_weight=w[:32]), dict(q_weight=w.bfloat16()), dict(k_weight=None), dict(eps=0.0),
           dict(eps=float("nan")), dict(q_out=x.bfloat16()), dict(q_weight=w.cpu()))
    for kw in bad:
        with pytest.raises(vc.VisCacheError):
            vc.viscache_norm_mrope(**{**good, **kw})
    good.update(q_out_grad=x, k_out_grad=x)
    vc.viscache_norm_mrope_grad(**good)
    for kw in bad[:-2] + (dict(q_out_grad=x[:3]), dict(k_out_grad=None), dict(q_weight_grad=w.bfloat16()),
                          dict(k_weight_grad=w[:32]), dict(q_grad=x.bfloat16()),
                          dict(ws=torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_norm_mrope_grad(**{**good, **kw})
