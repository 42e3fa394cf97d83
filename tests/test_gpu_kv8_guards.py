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


def test_pool_past_four_gigabytes():
    # pages on both sides of byte 2^32 of the pools hold the same tokens: the same codes, rows and outputs
    Hkv, page, d, n_pages = 8, 128, 128, 33200          # 4.35 GB of codes each for K and V
    cache = vc.Kv8Cache.empty(n_pages, Hkv, page, d, DEV)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    n, m = 700, 40
    low, high = i32([[5, 1, 9, 0, 3, 7]]), i32([[33199, 32800, 32766, 32768, 33000, 32767]])
    K, V = (_rand((n, Hkv, d), k, F32, 3.0).to(DEV) for k in (1, 2))
    got = []
    for table in (low, high):
        step = lambda rows: vc.Kv8Step(table, i32([n]), i32([0, rows]), rows)
        vc.viscache_kv8_append(cache, step(n), K, V)
        out = list(vc.viscache_kv8_read(cache, step(n), F32))
        wide = torch.full((1, 3200), -7, dtype=torch.int32, device=DEV)
        wide[:, :6] = table
        for dtype in (BF, F32):
            out.append(vc.viscache_kv8_attention(cache, step(1), _rand((1, 16, d), 3, dtype).to(DEV)))
            q = _rand((m, 64, d), 4, dtype).to(DEV)
            for rows in (m, 4):                         # 512-row and 32-row units of a KV head and fewer
                out.append(vc.viscache_kv8_attention(cache, vc.Kv8Step(wide, i32([n]), i32([0, rows]), rows), q[:rows]))
            q = _rand((80, 64, d), 5, dtype).to(DEV)
            out.append(vc.viscache_kv8_attention(cache, vc.Kv8Step(wide, i32([n]), i32([0, 80]), 80), q))
        got.append(out)
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_rows_past_four_gigabytes():
    # rows 2.5 GB apart
    d, H, stride = 128, 3, (5 << 28)
    buf = torch.zeros(2 * stride + H * d, dtype=BF, device=DEV)
    x = _rand((3, H, d), 1, BF).to(DEV)
    far = buf.as_strided((3, H, d), (stride, d, 1))
    far.copy_(x)
    pos = torch.tensor([[5, 70, 900]] * 3, dtype=torch.int32, device=DEV)
    rope = vc.make_rope((16, 24, 24))
    near, _ = vc.viscache_mrope(rope, pos, x)
    out, _ = vc.viscache_mrope(rope, pos, far)
    assert torch.equal(out, near)
    vc.viscache_mrope(rope, pos, far, q_out=far)
    assert torch.equal(far, near)
    caches = [vc.Kv8Cache.empty(1, H, 16, d, DEV) for _ in range(2)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    step = vc.Kv8Step(i32([[0]]), i32([3]), i32([0, 3]), 3)
    rows, outs = [], []
    for cache, k in zip(caches, (near, far)):
        vc.viscache_kv8_append(cache, step, k, k)
        rows += vc.viscache_kv8_read(cache, step)
        outs.append(vc.viscache_kv8_attention(cache, step, k))
    assert torch.equal(rows[0], rows[2]) and torch.equal(rows[1], rows[3]) and torch.equal(*outs)
