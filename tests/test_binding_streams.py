"""Tensors that an entry point of the binding makes for itself (workspaces, outputs) belong to
the stream the call runs on: a workspace of another stream's pool, dropped when the call returns,
would be handed out again while the kernels that use it are still to run."""
import contextlib
import inspect
import types

import pytest
import torch

from paper_2608_24063_gb300 import viscache as vc

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
BATCH = vc.Batch([64], [8], [(1, 2)])
PARAMS = vc.make_params(2, 4, 2, 64, vc.VC_BF16)


def z(*shape, dt=BF):
    return torch.zeros(shape, dtype=dt)


def _cache():
    return vc.Kv8Cache(z(4, 2, 16, 64, dt=U8), z(4, 2, 16, 64, dt=U8), z(4, 2, dt=F32), z(4, 2, dt=F32))


def _step():
    return vc.Kv8Step(z(1, 4, dt=I32), torch.full((1,), 3, dtype=I32), torch.tensor([0, 3], dtype=I32), 3)


def _kv4():
    return z(8, 32, dt=U8), z(8, 32, dt=U8), z(2, 64, 2, dt=F32), z(8, 2, 2, dt=F32)


# the arguments of a call that makes its own workspace and outputs
CALLS = {
    "viscache_mrope": lambda: (vc.make_rope((16, 16)), z(2, 3, dt=I32), z(3, 4, 64), z(3, 2, 64)),
    "viscache_kv8_append": lambda: (_cache(), _step(), z(3, 2, 64), z(3, 2, 64)),
    "viscache_kv8_read": lambda: (_cache(), _step()),
    "viscache_kv8_attention": lambda: (_cache(), _step(), z(3, 4, 64)),
    "viscache_scout_mmr": lambda: (z(9, 16, dt=F32), z(1, 16, dt=F32), [9]),
    "prunekv_score": lambda: (z(2, 4, 8, 64), z(2, 2, 64, 64)),
    "prunekv_score_static": lambda: (z(2, 4, 8, 64), z(2, 2, 64, 64)),
    "prunekv_select": lambda: (z(2, 64, dt=F32), [8, 4], 12),
    "prunekv_fuse_compact": lambda: (z(2, 2, 64, 64), z(2, 2, 64, 64), [8, 4], 12, z(0, dt=I32), z(0, dt=I32)),
    "prunekv_compress": lambda: (BATCH, PARAMS, z(2, 4, 8, 64), z(2, 2, 64, 64), z(2, 2, 64, 64)),
    "viscache_decode_attention": lambda: (BATCH, PARAMS, 0, z(1, 4, 64), z(8, 64), z(8, 64)),
    "viscache_decode_attention_kv4": lambda: (BATCH, PARAMS, 0, z(1, 4, 64), _kv4()),
    "viscache_kv4_quantize": lambda: (BATCH, PARAMS, z(8, 64), z(8, 64)),
    "viscache_kv4_dequantize": lambda: (BATCH, PARAMS) + _kv4(),
}


class _Library:
    """The library with its host arithmetic; what would launch answers with success."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        if name.endswith(("_size", "_sizes")) or name.startswith("viscache_plan"):
            return getattr(self.real, name)

        def call(*a):
            if name == "viscache_scout_mmr":                # its answer on the host: keyframes a video
                self.real.viscache_scout_sizes(a[2], a[3], a[6], a[7], a[11])
            return vc.VC_OK
        return call


def test_every_entry_with_a_stream_is_listed():
    takes = {n for n in vc.EXPORTED if "stream" in inspect.signature(getattr(vc, n, len)).parameters}
    assert takes - {"prunekv_get_status", "prunekv_score_static_status"} == set(CALLS)


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


def test_a_handle_is_enough(monkeypatch):
    # a stream object that is not torch's: what it wraps
    entered = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: ("external", handle))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: entered.append(s) or contextlib.nullcontext())
    t = vc._workspace(300, "cpu", None, types.SimpleNamespace(cuda_stream=77))
    assert entered == [("external", 77)] and t.numel() == 300
