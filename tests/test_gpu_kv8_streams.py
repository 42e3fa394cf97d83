"""Calls on a side stream that make their own workspaces and outputs, while the current stream
allocates and fills memory before they have run."""
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_kv8 import BF, DEV, _filled, _rand

pytestmark = pytest.mark.gpu


def test_memory_of_a_call_in_flight_is_not_handed_out():
    lens, rows = [9000, 700], [1, 3]
    pool = _filled(lens, 2, 64, 128)
    step = pool.step(lens, rows)
    q, kv = _rand((4, 8, 128), 1, BF).to(DEV), _rand((4, 2, 128), 2, BF).to(DEV)
    vc.viscache_kv8_append(pool.cache, step, kv, kv)
    want = vc.viscache_kv8_attention(pool.cache, step, q)
    rope = vc.make_rope((16, 24, 24))
    pos = torch.arange(12, dtype=torch.int32, device=DEV).view(3, 4)
    turned, _ = vc.viscache_mrope(rope, pos, q)
    need = vc.viscache_kv8_workspace_size(4, 8, 2, 128)
    a = torch.randn(4096, 4096, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            for _ in range(4):
                b = a @ a                       # some milliseconds in front of the calls
        vc.viscache_kv8_append(pool.cache, step, kv, kv, stream=side)
        got = vc.viscache_kv8_attention(pool.cache, step, q, stream=side)
        spun, _ = vc.viscache_mrope(rope, pos, q, stream=side)
        held = [torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(6)]
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(spun, turned)
        assert all(bool((t == 0xFF).all()) for t in held)
        del b, got, spun, held


def test_a_stream_of_another_library():
    # an object with a handle alone, as other libraries' streams have
    import types
    lens, rows = [300], [2]
    pool = _filled(lens, 1, 64, 128)
    q = _rand((2, 4, 128), 1, BF).to(DEV)
    step = pool.step(lens, rows)
    want = vc.viscache_kv8_attention(pool.cache, step, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = vc.viscache_kv8_attention(pool.cache, step, q, stream=types.SimpleNamespace(cuda_stream=side.cuda_stream))
    side.synchronize()
    assert torch.equal(got, want)
