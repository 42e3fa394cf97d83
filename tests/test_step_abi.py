"""CPU checks of the entry points of include/viscache_step.h: declared, exported and bound under
the same names; refusals as codes, before any device work; what a call makes for itself belongs to
the stream it runs on."""
import contextlib
import ctypes
import inspect
import os
import re
import types

import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def z(*shape, dt=BF):
    return torch.zeros(shape, dtype=dt)


def test_library_exports_every_declared_symbol():
    src = open(os.path.join(ROOT, "include", "viscache_step.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(\w+)\s*\(", src, flags=re.M))
    assert names == set(vc.EXPORTED_STEP)
    for name in names:
        assert hasattr(vc.lib(), name) and callable(getattr(vc, name))


def _cache():
    return vc.Kv8Cache(z(4, 2, 16, 64, dt=U8), z(4, 2, 16, 64, dt=U8), z(4, 2, dt=F32), z(4, 2, dt=F32))


def _step():
    return vc.Kv8Step(z(1, 4, dt=I32), torch.full((1,), 3, dtype=I32), torch.tensor([0, 3], dtype=I32), 3)


# the arguments of a call that makes its own workspace and outputs
CALLS = {
    "viscache_norm_mrope": lambda: (vc.make_rope((16, 16)), z(2, 3, dt=I32), z(3, 4, 64), z(3, 2, 64), z(64), z(64)),
    "viscache_norm_mrope_grad": lambda: (vc.make_rope((16, 16)), z(2, 3, dt=I32), z(3, 4, 64), z(3, 2, 64), z(3, 4, 64),
                                         z(3, 2, 64), z(64), z(64)),
    "viscache_kv8_weigh": lambda: (_cache(), _step(), z(3, 4, 64), z(3, 4, dt=F32), z(4, 2, 16, dt=F32)),
    "viscache_kv8_evict": lambda: (_cache(), _step(), z(4, 2, 16, dt=F32), z(1, dt=I32), 2),
    "viscache_sample": lambda: (z(3, 40), z(3, dt=F32), z(3, dt=F32)),
}


class _Library:
    """The library with its host arithmetic; what would launch answers with success."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        return getattr(self.real, name) if name.endswith("_size") else lambda *a: vc.VC_OK


def test_every_entry_with_a_stream_is_listed():
    assert {n for n in vc.EXPORTED_STEP if "stream" in inspect.signature(getattr(vc, n)).parameters} == set(CALLS)


@pytest.mark.parametrize("name", CALLS)
def test_a_call_allocates_on_its_own_stream(name, monkeypatch):
    side, on, made = types.SimpleNamespace(cuda_stream=77, device="cuda"), [None], []
    args, fake = CALLS[name](), _Library(vc.lib())

    @contextlib.contextmanager
    def stream(s):
        on.append(s)
        yield
        on.pop()

    def noted(real):
        def make(*a, **kw):
            made.append(on[-1])
            return real(*a, **kw)
        return make

    monkeypatch.setattr(vc, "lib", lambda: fake)
    monkeypatch.setattr(vc, "_current_device", lambda: -1)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    for f in ("empty", "zeros", "empty_like"):
        monkeypatch.setattr(torch, f, noted(getattr(torch, f)))
    getattr(vc, name)(*args, stream=side)
    assert made and all(s is side for s in made), made


# ---- refusals: addresses that no call gets to use, every argument right but one

A = 1 << 20                             # an aligned address


def _refused(name, good, bad, code=vc.VC_ERR_INVALID_ARG):
    """`good`: arguments by name in order; each of `bad` replaces some of them."""
    for change in bad:
        assert set(change) <= set(good), change
        rc = getattr(vc.lib(), name)(*{**good, **change}.values())
        assert rc == code, (change, rc)


def _rope(**kw):
    return vc.vc_rope(**{**dict(n_axes=2, sections=(ctypes.c_int32 * 4)(16, 16), order=0, pairing=0, theta=1e4), **kw})


ROPES = [dict(rope=r) for r in (None, _rope(n_axes=0), _rope(n_axes=5), _rope(theta=0.5), _rope(theta=float("inf")),
                                _rope(order=2), _rope(pairing=-1), _rope(sections=(ctypes.c_int32 * 4)(16, 12)),
                                _rope(sections=(ctypes.c_int32 * 4)(64, 64)),
                                _rope(sections=(ctypes.c_int32 * 4)(-8, 16)))]
SIZES = [dict(dtype=2), dict(n_rows=-1), dict(n_rows=(1 << 24) + 1), dict(Hq=-1), dict(Hq=4097), dict(Hkv=4097),
         dict(d=96), dict(eps=0.0), dict(eps=2.0), dict(eps=float("nan")), dict(positions=None)]


def _norm_args():
    return dict(rope=_rope(), positions=A, dtype=0, n_rows=3, Hq=4, Hkv=2, d=64, q=A, q_stride=256, k=A, k_stride=128,
                q_weight=A, k_weight=A, eps=1e-6, q_out=A, q_out_stride=256, k_out=A, k_out_stride=128, stream=None)


def test_norm_mrope_refuses():
    rows = [{p: v} for p in ("q", "k", "q_weight", "k_weight", "q_out", "k_out") for v in (None, A + 8)]
    strides = [{p + "_stride": v} for p, n in (("q", 256), ("k", 128), ("q_out", 256), ("k_out", 128))
               for v in (n - 8, n + 4, -n)]
    _refused("viscache_norm_mrope", _norm_args(), ROPES + SIZES + rows + strides)
    assert vc.lib().viscache_norm_mrope(*{**_norm_args(), "n_rows": 0}.values()) == vc.VC_OK
    assert vc.lib().viscache_norm_mrope(*{**_norm_args(), "Hq": 0, "Hkv": 0, "q": None, "k": None}.values()) == vc.VC_OK


def test_norm_mrope_grad_refuses():
    size = vc.viscache_norm_mrope_grad_workspace_size
    good = dict(rope=_rope(), positions=A, dtype=0, n_rows=3, Hq=4, Hkv=2, d=64, q=A, q_stride=256, k=A, k_stride=128,
                q_out_grad=A, q_out_grad_stride=256, k_out_grad=A, k_out_grad_stride=128, q_weight=A, k_weight=A,
                eps=1e-6, q_grad=A, q_grad_stride=256, k_grad=A, k_grad_stride=128, q_weight_grad=A, k_weight_grad=A,
                ws=A, ws_bytes=size(3, 4, 2, 64), stream=None)
    rows = [{p: v} for p in ("q", "k", "q_weight", "k_weight", "q_out_grad", "k_out_grad", "q_grad", "k_grad",
                             "q_weight_grad", "k_weight_grad") for v in (None, A + 4)]
    strides = [{p + "_stride": v} for p, n in (("q", 256), ("k", 128), ("q_out_grad", 256), ("k_out_grad", 128),
                                               ("q_grad", 256), ("k_grad", 128)) for v in (n - 8, n + 4)]
    _refused("viscache_norm_mrope_grad", good, ROPES + SIZES + rows + strides)
    _refused("viscache_norm_mrope_grad", good, [dict(ws=None), dict(ws=A + 16), dict(ws_bytes=size(3, 4, 2, 64) - 1)],
             vc.VC_ERR_WORKSPACE)
    assert size(-1, 4, 2, 64) == 0 and size(3, 4, 2, 96) == 0 and size(3, 4097, 2, 64) == 0
    assert size(1 << 24, 64, 8, 128) == size(3, 64, 8, 128)


def _pool(**kw):
    return vc.vc_kv8(*{**dict(K_codes=A, V_codes=A, K_scale=A, V_scale=A, n_pages=4, Hkv=2, page=16, d=64), **kw}.values())


def _requests(**kw):
    return vc.vc_kv8_step(*{**dict(n_req=2, max_pages=3, block_table=A, seq_lens=A, row_start=A, n_rows=5), **kw}.values())


POOLS = [dict(cache=None)] + [dict(cache=_pool(**kw)) for kw in (
    dict(K_codes=None), dict(V_codes=A + 4), dict(K_scale=None), dict(V_scale=A + 8), dict(n_pages=0), dict(page=48),
    dict(d=32), dict(Hkv=0), dict(Hkv=1025), dict(n_pages=1 << 27))]
STEPS = [dict(step=None)] + [dict(step=_requests(**kw)) for kw in (
    dict(block_table=None), dict(seq_lens=None), dict(row_start=None), dict(n_req=0), dict(n_req=1025),
    dict(max_pages=0), dict(max_pages=1 << 28), dict(n_rows=-1), dict(n_rows=(1 << 24) + 1))]


def test_kv8_weigh_refuses():
    need = vc.viscache_kv8_workspace_size(5, 4, 2, 64)
    good = dict(cache=_pool(), step=_requests(), dtype=0, Hq=4, q=A, q_stride=256, lse=A, scale=0.0, causal=1,
                weights=A, ws=A, ws_bytes=need, stream=None)
    own = [dict(dtype=2), dict(Hq=3), dict(Hq=0), dict(Hq=8192), dict(q=None), dict(q=A + 8), dict(q_stride=248),
           dict(q_stride=260), dict(lse=None), dict(lse=A + 2), dict(scale=-1.0), dict(scale=float("inf")),
           dict(scale=float("nan")), dict(weights=None), dict(weights=A + 4)]
    _refused("viscache_kv8_weigh", good, POOLS + STEPS + own)
    _refused("viscache_kv8_weigh", good, [dict(ws=None), dict(ws=A + 16), dict(ws_bytes=1024)], vc.VC_ERR_WORKSPACE)
    long = dict(cache=_pool(Hkv=1024, n_pages=1 << 10), Hq=1024, step=_requests(n_rows=1 << 20, max_pages=1 << 26),
                q_stride=1 << 16)
    _refused("viscache_kv8_weigh", good, [long], vc.VC_ERR_UNSUPPORTED)


def test_kv8_evict_refuses():
    size = vc.viscache_kv8_evict_workspace_size
    good = dict(cache=_pool(), step=_requests(), weights=A, keep=A, max_keep=8, sink=0, recent=0, kept=A, new_lens=A,
                ws=A, ws_bytes=size(2, 2), stream=None)
    own = [{p: v} for p in ("weights", "keep", "kept", "new_lens") for v in (None, A + 2)] + [
        dict(weights=A + 4), dict(max_keep=0), dict(max_keep=(1 << 30) + 1), dict(sink=-1), dict(recent=-1)]
    _refused("viscache_kv8_evict", good, POOLS + STEPS + own)
    _refused("viscache_kv8_evict", good, [dict(ws=None), dict(ws=A + 16), dict(ws_bytes=size(2, 2) - 1)],
             vc.VC_ERR_WORKSPACE)
    assert size(0, 2) == 0 and size(1025, 2) == 0 and size(2, 0) == 0 and size(2, 1025) == 0


def test_sample_refuses():
    good = dict(dtype=0, n_rows=3, vocab=100, logits=A, stride=100, u=A, temperature=A, top_k=A, top_p=A, min_p=A,
                token=A, logprob=A, stream=None)
    _refused("viscache_sample", good, [
        dict(dtype=2), dict(n_rows=-1), dict(n_rows=65536), dict(vocab=0), dict(vocab=262145, stride=262145),
        dict(stride=99), dict(stride=1 << 40), dict(logits=None), dict(logits=A + 1), dict(dtype=1, logits=A + 2),
        dict(u=None), dict(temperature=None), dict(token=None)] +
        [{p: A + 2} for p in ("u", "temperature", "top_k", "top_p", "min_p", "token", "logprob")])
    assert vc.lib().viscache_sample(*{**good, "n_rows": 0, "logits": None}.values()) == vc.VC_OK
