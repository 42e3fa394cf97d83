"""Guard regions, poisoned outputs and overlapping calls of the rotary positions and of the
8-bit paged cache: nothing outside an output, a pool or the workspace is written, every output
row is, and calls on two streams with a workspace each do not disturb one another."""
import numpy as np
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc
from tests.test_gpu_guards import Guarded
from tests.test_gpu_kv8 import BF, DEV, F32, _filled, _rand

pytestmark = pytest.mark.gpu


def _ws(rows, Hq, Hkv, d):
    return Guarded(vc.viscache_kv8_workspace_size(rows, Hq, Hkv, d), torch.uint8, 0x5A)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,Hq,Hkv,d,half", [(1, 3, 1, 64, 32), (7, 28, 4, 128, 64), (133, 5, 5, 128, 24)])
def test_rope_stays_in_its_rows(rows, Hq, Hkv, d, half, dtype):
    # outputs with room after each row: the gap keeps its poison
    x = _rand((rows, Hq + Hkv, d), rows, dtype).to(DEV)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)[None]
    gap = 2 * d
    out = [Guarded(rows * (h * d + gap), dtype) for h in (Hq, Hkv)]
    q, k = (o.view(rows, h * d + gap)[:, :h * d].unflatten(1, (h, d)) for o, h in zip(out, (Hq, Hkv)))
    vc.viscache_mrope(vc.make_rope((half,)), pos, x[:, :Hq], x[:, Hq:], q_out=q, k_out=k)
    for o, y, h in zip(out, (q, k), (Hq, Hkv)):
        o.check("rope")
        assert torch.isfinite(y).all()
        assert torch.isnan(o.view(rows, h * d + gap)[:, h * d:]).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page", [(7, 1, 128, 64), (4, 4, 64, 16), (6, 3, 128, 128)])
def test_cache_calls_stay_in_their_buffers(Hq, Hkv, d, page, dtype):
    lens, rows = [260, 3, 131, 0, 129], [40, 3, 65, 0, 1]
    total = sum(rows)
    pool = _filled(lens, Hkv, page, d)
    # the pool between guards, with the same contents
    parts = [Guarded(t.numel(), t.dtype, 0) for t in pool.cache.tensors]
    for g, t in zip(parts, pool.cache.tensors):
        g.body.copy_(t.flatten())
    pool.cache = vc.Kv8Cache(*(g.view(*t.shape) for g, t in zip(parts, pool.cache.tensors)))
    step = pool.step(lens, rows)
    K, V = (Guarded(total * Hkv * d, dtype) for _ in range(2))
    ws = _ws(total, Hkv, Hkv, d)
    shape = (total, Hkv, d)
    vc.viscache_kv8_read(pool.cache, step, out=(K.view(*shape), V.view(*shape)), ws=ws.body)
    for g in (K, V, ws):
        g.check("read")
    assert torch.isfinite(K.body).all() and torch.isfinite(V.body).all()
    # a row of code * scale is a code again (4 bits fit both types): it reads back as it was
    vc.viscache_kv8_append(pool.cache, step, K.view(*shape), V.view(*shape), ws=ws.body)
    for g in parts + [ws]:
        g.check("append")
    a, b = (torch.empty(shape, dtype=F32, device=DEV) for _ in range(2))
    vc.viscache_kv8_read(pool.cache, step, out=(a, b), ws=ws.body)
    assert torch.equal(a, K.view(*shape).float()) and torch.equal(b, V.view(*shape).float())
    q = _rand((total, Hq, d), 3, dtype).to(DEV)
    for m, want in ((rows, total), ([1, 1, 1, 0, 1], 4)):
        out, lse = Guarded(want * Hq * d, dtype), Guarded(want * Hq, F32)
        ws = _ws(want, Hq, Hkv, d)
        vc.viscache_kv8_attention(pool.cache, pool.step(lens, m), q[:want], out=out.view(want, Hq, d),
                                  lse=lse.view(want, Hq), ws=ws.body)
        for g in (out, lse, ws) + tuple(parts):
            g.check("attention")
        assert torch.isfinite(out.body).all() and torch.isfinite(lse.body).all()


def test_many_rows_call_stays_in_its_buffers():
    # enough units for the other kernel: 8 KV heads, 40 rows of 8 heads
    lens, rows, Hq, Hkv, d = [700, 90], [150, 61], 64, 8, 128
    total = sum(rows)
    pool = _filled(lens, Hkv, 32, d)
    q = _rand((total, Hq, d), 3, BF).to(DEV)
    out, lse, ws = Guarded(total * Hq * d, BF), Guarded(total * Hq, F32), _ws(total, Hq, Hkv, d)
    vc.viscache_profile_enable(True)
    try:
        vc.viscache_kv8_attention(pool.cache, pool.step(lens, rows), q, out=out.view(total, Hq, d),
                                  lse=lse.view(total, Hq), ws=ws.body)
        torch.cuda.synchronize()
        assert list(vc.viscache_profile_read()) == ["kv8_attn_tc1"]
    finally:
        vc.viscache_profile_enable(False)
    for g in (out, lse, ws):
        g.check("attention")
    assert torch.isfinite(out.body).all() and torch.isfinite(lse.body).all()


def test_two_streams_with_a_workspace_each():
    rng = np.random.default_rng(4)
    jobs = []
    for i, (Hq, Hkv, d) in enumerate(((8, 2, 128), (16, 8, 64))):
        lens = rng.integers(400, 5000, 6).tolist()
        rows = rng.integers(1, 40, 6).tolist() if i else [1] * 6
        pool = _filled(lens, Hkv, 64, d)
        q = _rand((sum(rows), Hq, d), 8 + i, BF).to(DEV)
        ws = torch.empty(vc.viscache_kv8_workspace_size(sum(rows), Hq, Hkv, d), dtype=torch.uint8, device=DEV)
        jobs.append((pool, pool.step(lens, rows), q, ws, torch.cuda.Stream()))
    alone = [vc.viscache_kv8_attention(p.cache, s, q, ws=ws) for p, s, q, ws, _ in jobs]
    torch.cuda.synchronize()
    together = [torch.empty((20,) + tuple(o.shape), dtype=BF, device=DEV) for o in alone]
    torch.cuda.synchronize()
    for k in range(20):
        for (p, s, q, ws, st), o in zip(jobs, together):
            with torch.cuda.stream(st):
                vc.viscache_kv8_attention(p.cache, s, q, out=o[k], ws=ws)
    torch.cuda.synchronize()
    for one, many in zip(alone, together):
        assert all(torch.equal(one, x) for x in many)


def test_a_workspace_serves_calls_of_other_shapes_between_replays():
    # split units' flags of one call never count for another, nor for a replay of the same graph
    pool_a, pool_b = _filled([6000], 1, 64, 128), _filled([900, 2500], 2, 16, 64)
    qa, qb = _rand((1, 4, 128), 1, BF).to(DEV), _rand((90, 4, 64), 2, F32).to(DEV)
    sa, sb = pool_a.step([6000], [1]), pool_b.step([900, 2500], [50, 40])
    n = max(vc.viscache_kv8_workspace_size(1, 4, 1, 128), vc.viscache_kv8_workspace_size(90, 4, 2, 64))
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    wa, wb = (vc.viscache_kv8_attention(p.cache, s, q) for p, s, q in ((pool_a, sa, qa), (pool_b, sb, qb)))
    out = torch.empty_like(wa)
    vc.viscache_kv8_attention(pool_a.cache, sa, qa, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vc.viscache_kv8_attention(pool_a.cache, sa, qa, out=out, ws=ws)
    for _ in range(10):
        out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out, wa)
        assert torch.equal(vc.viscache_kv8_attention(pool_b.cache, sb, qb, ws=ws), wb)
