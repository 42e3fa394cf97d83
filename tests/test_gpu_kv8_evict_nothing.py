"""A budget of no tokens (viscache_kv8_evict with keep 0): nothing is read of what shared memory held
before, nothing is written but the length."""
import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _fill_shared_memory():
    """Leaves most of each SM's shared memory full of ones: codes and weights of that kind go through
    the rings of the few-rows weighing kernel, four chunks of 32 tokens of each of 12 warps at least."""
    Hkv, page, d, length = 8, 128, 128, 65536
    n = length // page
    codes = torch.full((n, Hkv, page, d), 255, dtype=torch.uint8, device=DEV)
    cache = vc.Kv8Cache(codes, codes, *(torch.ones(n, Hkv, device=DEV) for _ in range(2)))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = vc.Kv8Step(torch.arange(n, dtype=torch.int32, device=DEV)[None], i32([length]), i32([0, 1]), 1)
    weights = torch.full((n, Hkv, page), -1, dtype=torch.int32, device=DEV).view(torch.float32)
    vc.viscache_kv8_weigh(cache, step, torch.zeros(1, 8, d, dtype=torch.bfloat16, device=DEV),
                          torch.zeros(1, 8, device=DEV), weights)


@pytest.mark.parametrize("lens,page", [([40], 16), ([700, 3, 513], 64), ([20000] * 30, 128), ([30000], 128)],
                         ids=["short", "a few", "held keys", "more than the held"])
def test_nothing_stays(lens, page):
    Hkv, d, max_keep = 4, 64, 64
    need = [-(-x // page) for x in lens]
    table = torch.zeros(len(lens), max(need), dtype=torch.int32)
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = torch.arange(at, at + k)
        at += k
    g = torch.Generator(device=DEV).manual_seed(1)
    codes = [torch.randint(0, 120, (at, Hkv, page, d), dtype=torch.uint8, device=DEV, generator=g) for _ in range(2)]
    scales = [torch.ones(at, Hkv, device=DEV) for _ in range(2)]
    weights = torch.rand(at, Hkv, page, device=DEV, generator=g)
    before = [t.clone() for t in (*codes, *scales, weights)]
    cache = vc.Kv8Cache(*codes, *scales)
    n = len(lens)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = vc.Kv8Step(table.to(DEV), i32(lens), i32(list(range(n + 1))), n)
    kept = torch.full((n, Hkv, max_keep), -7, dtype=torch.int32, device=DEV)
    ws = torch.empty(vc.viscache_kv8_evict_workspace_size(n, Hkv), dtype=torch.uint8, device=DEV)
    for _ in range(5):
        _fill_shared_memory()
        new_lens = torch.full((n,), -9, dtype=torch.int32, device=DEV)
        vc.viscache_kv8_evict(cache, step, weights, i32([0] * n), max_keep, 4, 16, kept=kept, new_lens=new_lens, ws=ws)
        assert vc.prunekv_get_status(ws) == vc.VC_OK
        assert new_lens.tolist() == [0] * n and (kept == -7).all()
        assert all(torch.equal(x, y) for x, y in zip(before, (*codes, *scales, weights)))


def test_binding_refuses_no_room_for_the_list():
    codes = torch.zeros(2, 1, 16, 64, dtype=torch.uint8, device=DEV)
    cache = vc.Kv8Cache(codes, codes.clone(), torch.ones(2, 1, device=DEV), torch.ones(2, 1, device=DEV))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    step = vc.Kv8Step(i32([[0, 1]]), i32([20]), i32([0, 1]), 1)
    for max_keep in (0, -1):
        with pytest.raises(vc.VisCacheError):
            vc.viscache_kv8_evict(cache, step, torch.zeros(2, 1, 16, device=DEV), i32([0]), max_keep)
