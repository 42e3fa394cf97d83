"""Pins for oracle.kv8 (8-bit paged cache) and oracle.rope (rotary positions with several
axes), and the refusals of their entry points, which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv8, rope
from paper_2608_24063_gb300 import viscache as vc


def test_every_code_survives_a_round_trip():
    c = np.array([b for b in range(256) if b & 127 != 127], np.uint8)
    np.testing.assert_array_equal(kv8.encode(kv8.VALUE[c]), c)
    assert kv8.VALUE[0x7E] == 448.0 and kv8.VALUE[1] == 2.0 ** -9 and kv8.VALUE[8] == 2.0 ** -6


def test_encode_agrees_with_torch_everywhere_between_codes():
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.05, 0.05, 20001),
                        (kv8._POS[1:] + kv8._POS[:-1]) / 2]).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = kv8.encode(x.astype(np.float64))
    np.testing.assert_array_equal(kv8.VALUE[got], kv8.VALUE[t])


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (1.75, -8), (1.7500001, -7), (1.0, -8), (2.0, -7),
                                    (2.0 ** -130, -126), (3.0e38, 120)])
def test_scale_is_the_least_power_of_two_that_holds_amax(amax, e):
    assert kv8.scale_of(float(amax)) == 2.0 ** e


def test_growing_scale_reencodes_older_tokens():
    codes, scale = np.zeros((1, 1, 4, 2), np.uint8), np.zeros((1, 1), np.float32)
    kv8.append(codes, scale, [[0]], [1], [1], np.array([[[1.0, -0.5]]]))
    assert scale[0, 0] == 2.0 ** -8
    kv8.append(codes, scale, [[0]], [2], [1], np.array([[[100.0, 3.0]]]))
    assert scale[0, 0] == 2.0 ** -2
    # 100 / scale = 400 lies halfway between the codes 384 and 416: to the even one
    np.testing.assert_array_equal(kv8.gather(codes, scale, [0], 2, 0), [[1.0, -0.5], [96.0, 3.0]])


def test_attention_rows_see_their_tokens():
    rng = np.random.default_rng(3)
    q, K, V = rng.standard_normal((3, 8)), rng.standard_normal((2, 8)), rng.standard_normal((2, 8))
    out, lse, _ = kv8.attention(q, K, V, -1, 0.5)          # three rows, two tokens: row 0 sees none
    assert (out[0] == 0).all() and lse[0] == -np.inf
    np.testing.assert_allclose(out[1], V[0])
    full, _, _ = kv8.attention(q, K, V, None, 0.5)
    np.testing.assert_allclose(out[2], full[2])


def test_rope_is_a_rotation_and_its_inverse_undoes_it():
    rng = np.random.default_rng(4)
    x, pos = rng.standard_normal((5, 3, 64)), rng.integers(-50, 5000, (3, 5))
    for order in ("sectioned", "interleaved"):
        for pairing in ("halves", "adjacent"):
            y = rope.rotate(x, pos, (8, 4, 4), 1e4, order, pairing)
            np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
            np.testing.assert_array_equal(y[..., 32:], x[..., 32:])
            np.testing.assert_allclose(rope.rotate(y, pos, (8, 4, 4), 1e4, order, pairing, True), x, atol=1e-12)


def test_rope_scores_depend_on_distance_alone():
    rng = np.random.default_rng(5)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    dots = []
    for shift in (0, 7, 1000):
        a = rope.rotate(q, np.array([[9 + shift], [4 + shift]]), (4, 4), 100.0)
        b = rope.rotate(k, np.array([[2 + shift], [3 + shift]]), (4, 4), 100.0)
        dots.append(float((a * b).sum()))
    np.testing.assert_allclose(dots, dots[0])


def test_interleaved_axes():
    assert rope.axes_of((4, 2, 2), "interleaved") == [0, 1, 2, 0, 1, 2, 0, 0]
    assert rope.axes_of((2, 3, 3), "interleaved") == [0, 1, 2, 0, 1, 2, 0, 1]      # axis 2 has two that fit
    assert rope.axes_of((4, 2, 2), "sectioned") == [0, 0, 0, 0, 1, 1, 2, 2]


# ---- refusals, before any device work

P = 256            # a made-up 256-byte aligned address: nothing is launched


def _rope(rope_desc=None, positions=P, dtype=vc.VC_BF16, rows=4, Hq=2, Hkv=1, d=64, q=P, qs=192, k=P, ks=192,
          qo=P, qos=128, ko=P, kos=64):
    r = rope_desc if rope_desc is not None else vc.make_rope((8, 12, 12), 1e6)
    return vc.lib().viscache_mrope(r, positions, dtype, rows, Hq, Hkv, d, q, qs, k, ks, 0, qo, qos, ko, kos, None)


@pytest.mark.parametrize("bad", [
    dict(positions=None), dict(dtype=2), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(Hq=-1), dict(Hkv=5000),
    dict(d=96), dict(q=None), dict(q=P + 8), dict(qs=120), dict(qs=132), dict(k=None), dict(ks=60), dict(qo=None),
    dict(qos=100), dict(ko=P + 2), dict(kos=68)])
def test_mrope_refuses(bad):
    assert _rope(**bad) == vc.VC_ERR_INVALID_ARG


@pytest.mark.parametrize("desc", [
    vc.make_rope((8, 12, 11), 1e6), vc.make_rope((40,), 1e6), vc.make_rope((8,), 0.5),
    vc.make_rope((8,), float("inf")), vc.make_rope((8,), float("nan")), vc.make_rope((-8, 16), 1e4),
    vc.vc_rope(0, (ctypes.c_int32 * 4)(), 0, 0, 1e4), vc.vc_rope(5, (ctypes.c_int32 * 4)(8), 0, 0, 1e4),
    vc.vc_rope(1, (ctypes.c_int32 * 4)(8), 2, 0, 1e4), vc.vc_rope(1, (ctypes.c_int32 * 4)(8), 0, 2, 1e4)])
def test_mrope_refuses_descriptions(desc):
    assert _rope(desc) == vc.VC_ERR_INVALID_ARG


def test_mrope_without_rows_does_nothing():
    assert _rope(rows=0, positions=None, q=None, k=None, qo=None, ko=None) == vc.VC_OK


def _cache(**kw):
    v = dict(K_codes=P, V_codes=P, K_scale=P, V_scale=P, n_pages=8, Hkv=2, page=16, d=64)
    v.update(kw)
    return vc.vc_kv8(*v.values())


def _step(**kw):
    v = dict(n_req=2, max_pages=4, block_table=P, seq_lens=P, row_start=P, n_rows=3)
    v.update(kw)
    return vc.vc_kv8_step(*v.values())


BAD_CACHE = [dict(K_codes=None), dict(V_codes=P + 4), dict(K_scale=None), dict(V_scale=P + 4), dict(n_pages=0),
             dict(Hkv=0), dict(Hkv=1025), dict(page=24), dict(page=256), dict(d=96), dict(n_pages=1 << 26)]
BAD_STEP = [dict(n_req=0), dict(n_req=1025), dict(max_pages=0), dict(max_pages=1 << 28), dict(block_table=None),
            dict(seq_lens=None), dict(row_start=None), dict(n_rows=-1), dict(n_rows=(1 << 24) + 1)]


@pytest.mark.parametrize("cache,step", [(_cache(**b), _step()) for b in BAD_CACHE] +
                         [(_cache(), _step(**b)) for b in BAD_STEP])
def test_kv8_entries_refuse_bad_caches_and_steps(cache, step):
    lib, big = vc.lib(), 1 << 40
    assert lib.viscache_kv8_append(cache, step, 0, P, 128, 64, P, 128, 64, P, big, None) == vc.VC_ERR_INVALID_ARG
    assert lib.viscache_kv8_read(cache, step, 0, P, P, P, big, None) == vc.VC_ERR_INVALID_ARG
    assert lib.viscache_kv8_attention(cache, step, 0, 4, P, 256, 0.0, 1, P, None, P, big,
                                      None) == vc.VC_ERR_INVALID_ARG


def test_kv8_entries_refuse_bad_rows_and_workspaces():
    lib, big, c, s = vc.lib(), 1 << 40, _cache(), _step()
    app = lambda K=P, kr=128, kh=64, V=P, vr=128, vh=64, ws=P, n=big, dt=0: lib.viscache_kv8_append(
        c, s, dt, K, kr, kh, V, vr, vh, ws, n, None)
    for bad in (dict(K=None), dict(V=None), dict(K=P + 8), dict(kr=63), dict(kr=130), dict(kh=60), dict(vr=32),
                dict(vh=68), dict(dt=2)):
        assert app(**bad) == vc.VC_ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(ws=P + 16), dict(n=255)):
        assert app(**bad) == vc.VC_ERR_WORKSPACE, bad
    assert lib.viscache_kv8_read(c, s, 0, None, P, P, big, None) == vc.VC_ERR_INVALID_ARG
    assert lib.viscache_kv8_read(c, s, 0, P, P, P, 16, None) == vc.VC_ERR_WORKSPACE
    assert lib.viscache_kv8_read(None, s, 0, P, P, P, big, None) == vc.VC_ERR_INVALID_ARG
    att = lambda Hq=4, q=P, qs=256, sc=0.0, out=P, lse=None, ws=P, n=big, dt=0: lib.viscache_kv8_attention(
        c, s, dt, Hq, q, qs, sc, 1, out, lse, ws, n, None)
    for bad in (dict(Hq=3), dict(Hq=0), dict(q=None), dict(q=P + 8), dict(qs=255), dict(qs=252), dict(out=None),
                dict(sc=-1.0), dict(sc=float("inf")), dict(sc=float("nan")), dict(lse=P + 2), dict(dt=7)):
        assert att(**bad) == vc.VC_ERR_INVALID_ARG, bad
    need = vc.viscache_kv8_workspace_size(3, 4, 2, 64)
    assert need > 0 and need % 256 == 0
    assert att(n=need - 1) == vc.VC_ERR_WORKSPACE and att(ws=P + 64) == vc.VC_ERR_WORKSPACE
    for bad in ((-1, 4, 2, 64), (3, 3, 2, 64), (3, 4, 2, 96), (3, 4, 0, 64), ((1 << 24) + 1, 4, 2, 64)):
        assert vc.viscache_kv8_workspace_size(*bad) == 0


def test_handles_check_their_tensors():
    z = lambda *shape, dt=torch.uint8: torch.zeros(shape, dtype=dt)
    ok = (z(2, 1, 16, 64), z(2, 1, 16, 64), z(2, 1, dt=torch.float32), z(2, 1, dt=torch.float32))
    vc.Kv8Cache(*ok)
    for i, bad in ((0, z(2, 1, 16, 64, dt=torch.int32)), (1, z(2, 1, 16, 128)), (2, z(2, 2, dt=torch.float32)),
                   (3, z(2, 1, dt=torch.float64)), (1, z(2, 1, 64, 16).transpose(2, 3))):
        with pytest.raises(vc.VisCacheError):
            vc.Kv8Cache(*ok[:i], bad, *ok[i + 1:])
    i32 = lambda *shape: z(*shape, dt=torch.int32)
    vc.Kv8Step(i32(3, 4), i32(3), i32(4), 5)
    for bad in ((i32(2, 4), i32(3), i32(4)), (i32(3, 4), i32(3), i32(3)), (i32(3, 8)[:, ::2], i32(3), i32(4)),
                (i32(3, 4), z(3, dt=torch.int64), i32(4))):
        with pytest.raises(vc.VisCacheError):
            vc.Kv8Step(*bad, 5)
