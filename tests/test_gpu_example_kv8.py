"""The serving example end to end: one more token of every request against float64 attention
over what the cache reads back, and a replayed graph against the same steps one by one."""
import pytest
import torch

from examples import serve_kv8
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu


def _server():
    torch.manual_seed(3)                        # (page order)
    m = serve_kv8.Model(L=4, hidden=256, Hq=8, Hkv=2, d=128)
    requests = []
    for (t, h, w), n in (((4, 6, 8), 21), ((3, 5, 7), 9)):
        requests.append((m.rand(t * h * w + n, m.hidden), serve_kv8.positions_of(t, h, w, n, m.device), t * h * w))
    return m, serve_kv8.Server(m, requests)


def test_replayed_steps_are_the_steps():
    _, a = _server()
    _, b = _server()
    x = a.decode(6)
    for _ in range(6):
        b.token()
    torch.cuda.synchronize()
    assert torch.equal(x, b.x) and torch.isfinite(x).all()
    assert vc.prunekv_get_status(a.ws) == vc.VC_OK
    for layer in range(4):
        for p, q in zip(a.rows(layer), b.rows(layer)):
            assert all(torch.equal(s, t) for s, t in zip(p, q))
            assert [len(t) for t in p] == [n + 6 for n in a.lens[layer]]


def test_a_step_attends_over_what_the_cache_holds():
    m, s = _server()
    s.decode(3)
    x, positions = s.x.clone(), s.positions.clone()
    for layer in range(m.L):
        q, k, v = m.qkv(layer, x, positions)
        vc.viscache_kv8_append(s.pools[layer], s.steps[layer], k, v, ws=s.ws)
        out = vc.viscache_kv8_attention(s.pools[layer], s.steps[layer], q, ws=s.ws)
        lens = s.steps[layer].tensors[1].tolist()
        K, V = vc.viscache_kv8_read(s.pools[layer], m.step(s.table, lens, lens), torch.float32,
                                    ws=m.workspace(sum(lens)))
        for r, (Kr, Vr) in enumerate(zip(K.split(lens), V.split(lens))):
            G = m.Hq // m.Hkv
            Kd, Vd = (t.double().repeat_interleave(G, 1) for t in (Kr, Vr))
            p = torch.softmax(torch.einsum("hd,thd->ht", q[r].double(), Kd) * m.d ** -0.5, 1)
            ref = torch.einsum("ht,thd->hd", p, Vd)
            # scores below 2^7 with fp32 sums of 128 products and 2^-24 of their absolute sum a
            # step; probabilities rounded to 2^-11; the output's rounding
            size = torch.einsum("hd,thd->ht", q[r].double().abs(), Kd.abs()).amax(1) * m.d ** -0.5
            rel = 2.0 ** -11 + 2 * size * 14 * 2.0 ** -23 + (lens[r] / 16 + 40) * 2.0 ** -23 + 2.0 ** -20
            absv = torch.einsum("ht,thd->hd", p, Vd.abs())
            tol = rel[:, None] * absv + 2.0 ** -8 * ref.abs() * (1 + rel[:, None]) + lens[r] * 2.0 ** -28 * Vd.abs().amax()
            assert ((out[r].double() - ref).abs() <= tol).all()
        x = x + out.view(x.shape[0], -1) @ m.w_o[layer]


def test_main_runs(capsys):
    serve_kv8.main()
    assert "layer 3" in capsys.readouterr().out
