"""The norm's gradient stays within its workspace where nearly all of its blocks are one kind's."""
import numpy as np
import pytest
import torch

from oracle import step as ostep
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GUARD = 4096


def test_one_query_head_beside_thousands_of_key_heads():
    rows, Hkv, d, sec = 4900, 2600, 64, (12, 10, 10)
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(torch.bfloat16)
    q, yq, k, yk, w = rand(rows, 1, d), rand(rows, 1, d), rand(rows, Hkv, d), rand(rows, Hkv, d), rand(2, d)
    pos = torch.randint(0, 3000, (3, rows), dtype=torch.int32, device=DEV, generator=g)
    need = vc.viscache_norm_mrope_grad_workspace_size(rows, 1, Hkv, d)
    buf = torch.full((need + GUARD,), 0x5A, dtype=torch.uint8, device=DEV)
    want_k, want_wk = vc.viscache_norm_mrope_grad(vc.make_rope(list(sec), theta=1e6), pos, k, None, yk, None, w[1], None)[::2]
    dq, dk, dwq, dwk = vc.viscache_norm_mrope_grad(vc.make_rope(list(sec), theta=1e6), pos, q, k, yq, yk, w[0], w[1],
                                                   k_grad=yk, ws=buf[:need])
    assert (buf[need:] == 0x5A).all()
    X, Y, W = (t.double().cpu().numpy() for t in (q, yq, w[0]))
    dx, dw = ostep.norm_mrope_grad(X, Y, W, pos.cpu().numpy().astype(np.int64), sec, 1e6, 1e-6)
    n = np.abs(X / np.sqrt((X * X).mean(-1, keepdims=True) + 1e-6))
    # each term within 2^-20, added up in fp32 in pieces
    total = (np.abs(Y).max(-1, keepdims=True) * 1.5 * n).sum((0, 1))
    assert (np.abs(dwq.double().cpu().numpy() - dw) <= 2.0 ** -19 * (total + 1e-9)).all()
    # the key heads: the same rows by themselves, shared out over one block more
    assert torch.equal(dk, want_k)
    assert torch.allclose(dwk, want_wk, rtol=0, atol=2.0 ** -19 * rows * Hkv)     # (a mean term is 0.64)
