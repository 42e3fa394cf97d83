"""GPU parity of the rotary positions with several axes against the float64 oracle, the
inverse as gradient, strided rows and rows rotated in place."""
import numpy as np
import pytest
import torch

from oracle import rope as orope
from paper_2608_24063_gb300 import synth
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rand(shape, key, dtype):
    return synth._round(synth.normal(key, 0, int(np.prod(shape)), "cpu").view(*shape), dtype)


def _tol(x, dtype):
    # The angle is off by at most 2^-25 turn (the phase's top 32 bits as fp32) plus sincospif's
    # 2 ulp; with the products, under 2^-20 of the pair's length.  bf16 adds half an ulp.
    size = np.abs(x).max()
    return 2.0 ** -19 * size + (2.0 ** -8 * size * 1.5 if dtype == torch.bfloat16 else 0.0)


CASES = [(1, 28, 4, 128, (16, 24, 24), "sectioned", "halves"), (37, 8, 4, 64, (12, 10, 10), "interleaved", "adjacent"),
         (130, 3, 1, 128, (24, 20, 20), "interleaved", "halves"), (5, 2, 2, 64, (32,), "sectioned", "adjacent"),
         (33, 9, 3, 128, (8, 4, 4), "sectioned", "halves"), (9, 1, 0, 64, (4, 2, 1, 1), "sectioned", "adjacent")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("inverse", [False, True])
def test_matches_oracle(case, dtype, inverse):
    rows, Hq, Hkv, d, sec, order, pairing = case
    x = _rand((rows, Hq + 2 * Hkv, d), 11 + rows, dtype)
    rng = np.random.default_rng(rows)
    pos = rng.integers(-(1 << 20), 1 << 20, (len(sec), rows)).astype(np.int32)
    pos[:, 0] = 0
    pos[0, -1] = 2 ** 31 - 1 if rows > 1 else 7
    desc = vc.make_rope(sec, 1e6, interleaved=order == "interleaved", adjacent=pairing == "adjacent")
    xd = x.to(DEV)
    q, k = xd[:, :Hq], xd[:, Hq:Hq + Hkv]           # slices of a fused projection
    qo, ko = vc.viscache_mrope(desc, torch.from_numpy(pos).to(DEV), q, k if Hkv else None, inverse=inverse)
    torch.cuda.synchronize()
    ref = orope.rotate(x.double().numpy(), pos.astype(np.int64), sec, 1e6, order, pairing, inverse)
    # frequencies are good to 2^-47, which position 2^31 - 1 turns into 2^-16 turn
    far = 2.0 ** -13 * np.abs(ref).max()
    for got, want in ((qo, ref[:, :Hq]), (ko, ref[:, Hq:Hq + Hkv])):
        if got is not None:
            err = np.abs(got.double().cpu().numpy() - want)
            assert err[:-1].max(initial=0.0) <= _tol(want, dtype)
            assert err[-1].max() <= _tol(want, dtype) + far
    assert torch.equal(xd.cpu(), x)


@pytest.mark.parametrize("adjacent", [False, True])
def test_in_place_equals_out_of_place(adjacent):
    x = _rand((65, 40, 128), 5, torch.bfloat16).to(DEV)
    pos = torch.arange(3 * 65, dtype=torch.int32, device=DEV).view(3, 65)
    desc = vc.make_rope((16, 24, 24), 1e6, adjacent=adjacent)
    q, k = x[:, :28], x[:, 28:32]
    qo, ko = vc.viscache_mrope(desc, pos, q, k)
    rest = x[:, 32:].clone()
    vc.viscache_mrope(desc, pos, q, k, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(x[:, 32:], rest)


def test_inverse_is_the_gradient():
    # <rotate(x), g> = <x, inverse(g)>: exact for the linear map, and against differences of
    # the oracle's forward form in a random direction
    rows, H, d, sec = 21, 5, 64, (12, 10, 10)
    x, g = _rand((rows, H, d), 31, torch.float32), _rand((rows, H, d), 32, torch.float32)
    pos = np.random.default_rng(8).integers(0, 9000, (3, rows)).astype(np.int32)
    desc = vc.make_rope(sec, 1e4, interleaved=True)
    gx, _ = vc.viscache_mrope(desc, torch.from_numpy(pos).to(DEV), g.to(DEV), inverse=True)
    gx = gx.double().cpu().numpy()
    fwd = lambda v: (orope.rotate(v, pos, sec, 1e4, "interleaved") * g.double().numpy()).sum()
    v = np.random.default_rng(9).standard_normal(x.shape)
    h = 1e-3
    diff = (fwd(x.double().numpy() + h * v) - fwd(x.double().numpy() - h * v)) / (2 * h)
    # each of gx's values within 2^-20 of its pair: the sum within that times the sum of |v| |g|
    assert abs((gx * v).sum() - diff) <= 2.0 ** -19 * 4 * np.abs(v).sum()


def test_side_stream_and_repeatability():
    x = _rand((300, 36, 128), 77, torch.bfloat16).to(DEV)
    pos = torch.arange(900, dtype=torch.int32, device=DEV).view(3, 300)
    desc = vc.make_rope((16, 24, 24), 1e6)
    a, _ = vc.viscache_mrope(desc, pos, x)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b, _ = vc.viscache_mrope(desc, pos, x, stream=st)
    st.synchronize()
    assert torch.equal(a, b)


def test_binding_refuses():
    x = torch.zeros((4, 2, 64), device=DEV)
    pos = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    desc = vc.make_rope((32,), 1e4)
    for kw in (dict(positions=pos.long()), dict(positions=pos[:, :3]), dict(q=x.transpose(1, 2)), dict(q=x.cpu()),
               dict(k=x[:3]), dict(k=x.bfloat16()), dict(q_out=x.bfloat16())):
        args = dict(positions=pos, q=x)
        args.update(kw)
        with pytest.raises(vc.VisCacheError):
            vc.viscache_mrope(desc, **args)
    with pytest.raises(TypeError):
        vc.viscache_mrope(desc, pos, x.half())
