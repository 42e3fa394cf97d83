"""The serving example held to a budget: the caches stop growing, and a replayed graph gives what the
steps give one by one."""
import pytest
import torch

from examples import serve_kv8
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu


def _server(budget):
    torch.manual_seed(3)                        # (page order)
    m = serve_kv8.Model(L=3, hidden=256, Hq=8, Hkv=2, d=128)
    requests = []
    for (t, h, w), n in (((4, 6, 8), 21), ((3, 5, 7), 9)):
        requests.append((m.rand(t * h * w + n, m.hidden), serve_kv8.positions_of(t, h, w, n, m.device), t * h * w))
    return serve_kv8.Server(m, requests, budget=budget)


def test_the_caches_stop_growing():
    a, b = _server(48), _server(48)
    x = a.decode(12)
    for _ in range(12):
        b.token()
    torch.cuda.synchronize()
    assert torch.equal(x, b.x) and torch.isfinite(x).all()
    assert vc.prunekv_get_status(a.ws) == vc.prunekv_get_status(a.evict_ws) == vc.VC_OK
    for layer in range(3):
        lens = [min(n + 12, 48) for n in a.lens[layer]]
        for p, q in zip(a.rows(layer), b.rows(layer)):
            assert [len(t) for t in p] == lens and all(torch.equal(s, t) for s, t in zip(p, q))


def test_a_budget_that_is_never_reached_changes_nothing():
    a, b = _server(0), _server(500)
    assert torch.equal(a.decode(5), b.decode(5))
