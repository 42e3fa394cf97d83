"""The operators of a decode step in the order a program runs them: heads normed and rotated, rows
appended, attended over, the attention weighed, the cache held to a budget, the next token drawn.
Each against its oracle on what the device held before it, then the whole step captured and
replayed against the same steps run eagerly."""
import numpy as np
import pytest
import torch

from oracle import kv8
from oracle import step as ostep
from paper_2608_24063_gb300 import viscache as vc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Server:
    """One layer, `n` requests a row each, held to `budget` tokens."""

    def __init__(self, lens, budget, Hq=8, Hkv=2, d=64, page=16, vocab=501, dtype=BF, seed=3):
        self.g = torch.Generator(DEV).manual_seed(seed)
        rand = lambda *s, dt=dtype: torch.randn(*s, generator=self.g, device=DEV, dtype=F32).to(dt)
        n = len(lens)
        self.n, self.Hq, self.Hkv, self.d, self.page, self.dtype = n, Hq, Hkv, d, page, dtype
        self.budget, self.rand = budget, rand
        cap = -(-(max(lens + [budget]) + 2) // page)
        order = torch.randperm(n * cap, generator=torch.Generator().manual_seed(seed)).to(I32)
        self.table = order.view(n, cap).contiguous().to(DEV)
        self.cache = vc.Kv8Cache.empty(n * cap, Hkv, page, d, DEV)
        self.lens = torch.tensor(lens, dtype=I32, device=DEV)
        start = np.concatenate([[0], np.cumsum(lens)]).tolist()
        first = vc.Kv8Step(self.table, self.lens, torch.tensor(start, dtype=I32, device=DEV), start[-1])
        vc.viscache_kv8_append(self.cache, first, rand(start[-1], Hkv, d), rand(start[-1], Hkv, d))
        self.weights = torch.rand(n * cap, Hkv, page, generator=self.g, device=DEV)
        self.rope = vc.make_rope([d // 8, 3 * d // 16, 3 * d // 16], 1e6, interleaved=True)
        self.pos = torch.tensor([lens] * 3, dtype=I32, device=DEV).contiguous()
        self.norms = (1.0 + 0.3 * rand(2, d, dt=F32)).to(dtype)
        self.w_qkv, self.w_out = rand(n, Hq * d, (Hq + 2 * Hkv) * d) * (Hq * d) ** -0.5, rand(Hq * d, vocab) * 0.3
        self.x = rand(n, 1, Hq * d)
        self.u, self.T = torch.rand(n, generator=self.g, device=DEV), torch.full((n,), 0.8, device=DEV)
        self.top_k = torch.full((n,), 40, dtype=I32, device=DEV)
        self.top_p = torch.full((n,), 0.9, device=DEV)
        self.keep = torch.full((n,), budget, dtype=I32, device=DEV)
        self.kept = torch.zeros(n, Hkv, budget, dtype=I32, device=DEV)
        self.lse = torch.zeros(n, Hq, device=DEV)
        self.token = torch.zeros(n, dtype=I32, device=DEV)
        self.logprob = torch.zeros(n, device=DEV)
        self.step = vc.Kv8Step(self.table, self.lens, torch.arange(n + 1, dtype=I32, device=DEV), n)
        u8 = lambda k: torch.empty(k, dtype=torch.uint8, device=DEV)
        self.ws = u8(vc.viscache_kv8_workspace_size(n, Hq, Hkv, d))
        self.ews = u8(vc.viscache_kv8_evict_workspace_size(n, Hkv))
        self.check = None                       # called between the operators

    def state(self):
        return [t for t in self.cache.tensors] + [self.weights, self.lens, self.pos, self.x, self.kept, self.token, self.logprob]

    def run(self):
        """One token of every request; nothing comes from the host."""
        see = self.check or (lambda *a: None)
        n, Hq, Hkv, d = self.n, self.Hq, self.Hkv, self.d
        y = torch.bmm(self.x, self.w_qkv).view(n, Hq + 2 * Hkv, d)
        q, k, v = y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:]
        see("before", y)
        vc.viscache_norm_mrope(self.rope, self.pos, q, k, self.norms[0], self.norms[1], q_out=q, k_out=k)
        see("normed", y)
        self.lens += 1
        vc.viscache_kv8_append(self.cache, self.step, k, v, ws=self.ws)
        out = vc.viscache_kv8_attention(self.cache, self.step, q, lse=self.lse, ws=self.ws)
        see("attended", q, out)
        vc.viscache_kv8_weigh(self.cache, self.step, q, self.lse, self.weights, ws=self.ws)
        see("weighed", q)
        vc.viscache_kv8_evict(self.cache, self.step, self.weights, self.keep, self.budget, sink=2, recent=8, kept=self.kept,
                              new_lens=self.lens, ws=self.ews)
        see("evicted")
        logits = out.view(n, Hq * d) @ self.w_out
        vc.viscache_sample(logits, self.u, self.T, self.top_k, self.top_p, token=self.token, logprob=self.logprob)
        see("sampled", logits)
        self.pos += 1
        self.u.mul_(0.7).add_(0.1)
        self.x.copy_(torch.tanh(out.view(n, 1, Hq * d) + 0.1 * self.token[:, None, None].to(self.dtype)))


class Oracle:
    def __init__(self, s):
        self.s, self.seen = s, []

    def host(self):
        s = self.s
        k, v, ks, vs = (t.cpu().numpy() for t in s.cache.tensors)
        return [k, v], [ks, vs], s.table.cpu().numpy(), s.lens.tolist(), s.weights.cpu().numpy()

    def __call__(self, what, *a):
        s = self.s
        self.seen.append(what)
        if what == "before":
            self.y = a[0].double().cpu().numpy()
        elif what == "normed":
            sec = (s.d // 8, 3 * s.d // 16, 3 * s.d // 16)
            got = a[0].double().cpu().numpy()
            for lo, hi, w in ((0, s.Hq, 0), (s.Hq, s.Hq + s.Hkv, 1)):
                want = ostep.norm_mrope(self.y[:, lo:hi], s.norms[w].double().cpu().numpy(),
                                        s.pos.cpu().numpy().astype(np.int64), sec, 1e6, 1e-6, "interleaved")
                size = np.abs(want).max(-1, keepdims=True)
                assert (np.abs(got[:, lo:hi] - want) <= 2.0 ** -19 * size + 2.0 ** -8 * np.abs(want)).all()
            assert np.array_equal(got[:, s.Hq + s.Hkv:], self.y[:, s.Hq + s.Hkv:])
        elif what == "attended":
            codes, scale, table, lens, self.before = self.host()
            q, out = a[0].double().cpu().numpy(), a[1].double().cpu().numpy()
            for r, length in enumerate(lens):
                t = np.arange(length)
                for g in range(s.Hkv):
                    K, V = (kv8.VALUE[c[table[r][t // s.page], g, t % s.page]] * x[table[r][t // s.page], g][:, None].astype(np.float64)
                            for c, x in zip(codes, scale))
                    for j in range(g * s.Hq // s.Hkv, (g + 1) * s.Hq // s.Hkv):
                        z = K @ q[r, j] / np.sqrt(s.d)
                        p = np.exp(z - z.max())
                        assert abs(s.lse[r, j].item() - np.log(p.sum()) - z.max()) <= 2.0 ** -17 * max(1.0, abs(z).max())
                        assert np.abs(out[r, j] - p @ V / p.sum()).max() <= 2.0 ** -7 * np.abs(V).max()
        elif what == "weighed":
            codes, scale, table, lens, got = self.host()
            want = ostep.weigh(codes[0], scale[0], table, lens, [1] * s.n, a[0].double().cpu().numpy(),
                               s.lse.double().cpu().numpy(), self.before)
            live = np.zeros(want.shape, bool)
            for r, length in enumerate(lens):
                t = np.arange(length)
                live[table[r][t // s.page], :, t % s.page] = True
            assert (np.abs(got - want)[live] <= 2.0 ** -15 * np.abs(want[live]) + 1e-30).all()
            assert np.array_equal(got[~live], self.before[~live])
            self.cache, self.kept = self.host(), s.kept.cpu().numpy().copy()
        elif what == "evicted":
            codes, scale, table, lens, weights = self.cache
            new = ostep.evict(codes, scale, table, lens, weights, [s.budget] * s.n, 2, 8, self.kept)
            c2, s2, _, l2, w2 = self.host()
            assert l2 == new and np.array_equal(w2, weights) and np.array_equal(s.kept.cpu().numpy(), self.kept)
            assert all(np.array_equal(x, y) for x, y in zip(c2 + s2, codes + scale))
        else:
            x = a[0].double().cpu().numpy()
            f = lambda t, r: float(np.float32(t[r].item()))
            for r in range(s.n):
                token, logprob = ostep.sample(x[r], f(s.u, r), f(s.T, r), 40, f(s.top_p, r))
                assert s.token[r].item() == token and abs(s.logprob[r].item() - logprob) <= 2.0 ** -20 * max(1.0, abs(logprob))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_each_operator_on_what_the_one_before_left(dtype):
    s = Server([70, 33, 1, 64], 48, dtype=dtype)
    s.check = Oracle(s)
    for _ in range(6):
        s.run()
    assert s.lens.tolist() == [48, 39, 7, 48] and len(s.check.seen) == 36


def test_replayed_steps_are_the_eager_ones():
    a, b = Server([70, 33, 5], 40), Server([70, 33, 5], 40)
    a.run(), b.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run()
    for _ in range(12):
        a.run()
        g.replay()
    torch.cuda.synchronize()
    assert a.lens.tolist() == [40, 40, 18]
    for x, y in zip(a.state(), b.state()):
        if x.dtype == torch.uint8 or x.is_floating_point() and x.dim() > 1:
            continue                            # (slots that hold no token differ: the pools begin uninitialised)
        assert torch.equal(x, y)
    assert torch.equal(a.x, b.x)


def test_two_servers_on_streams_of_their_own():
    # calls of two programs at once, each with its workspaces
    a, b = Server([70, 33, 5], 40), Server([70, 33, 5], 40)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    assert torch.equal(a.token, b.token) and torch.equal(a.lens, b.lens) and torch.equal(a.x, b.x)
