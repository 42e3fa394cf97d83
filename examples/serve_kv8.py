"""A video request served from the 8-bit paged cache, on a small model with random weights.

    python examples/serve_kv8.py

Prefill: every layer rotates the rows of the prompt (visual tokens with time, height and width,
then text) with viscache_mrope, writes them into a scratch cache with viscache_kv8_append and
attends over them as one chunk with viscache_kv8_attention.  prunekv_compress then keeps each
layer's share of the visual tokens; its output goes into the cache that serves the request as it
lies ([Hkv][B_l][d], read in place), the text rows behind it.  Decoding replays one captured
graph: rotate, append, attend in every layer, for all requests, with the lengths, the positions
and the tokens on the device.  viscache_kv8_read gives a layer's rows back in 16 bits.

With a budget the cache stops growing: each step's attention is added up with viscache_kv8_weigh
and viscache_kv8_evict keeps the tokens of each layer and KV head that received most of it.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_24063_gb300 import viscache as vc  # noqa: E402

BF = torch.bfloat16


class Model:
    """Attention layers alone: x + W_o attention(W_qkv norm(x))."""

    def __init__(self, L=4, hidden=512, Hq=8, Hkv=2, d=128, page=64, device="cuda", seed=1):
        g = torch.Generator(device).manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device=device, dtype=BF)
        self.L, self.hidden, self.Hq, self.Hkv, self.d, self.page = L, hidden, Hq, Hkv, d, page
        self.device, self.rand = device, rand
        self.w_qkv = [rand(hidden, (Hq + 2 * Hkv) * d) * hidden ** -0.5 for _ in range(L)]
        self.w_o = [rand(Hq * d, hidden) * (Hq * d) ** -0.5 for _ in range(L)]
        self.rope = vc.make_rope([d // 8, 3 * d // 16, 3 * d // 16])

    def qkv(self, layer, x, positions):
        """Rotated query and key rows (in place in the fused projection) and value rows."""
        x = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(BF)
        y = (x @ self.w_qkv[layer]).view(x.shape[0], self.Hq + 2 * self.Hkv, self.d)
        q, k, v = y[:, :self.Hq], y[:, self.Hq:self.Hq + self.Hkv], y[:, self.Hq + self.Hkv:]
        vc.viscache_mrope(self.rope, positions, q, k, q_out=q, k_out=k)
        return q, k, v

    def attend(self, layer, x, q, cache, step, ws, lse=None):
        out = vc.viscache_kv8_attention(cache, step, q, lse=lse, ws=ws)
        return x + out.view(x.shape[0], -1) @ self.w_o[layer]

    def pool(self, pages):
        return vc.Kv8Cache.empty(pages, self.Hkv, self.page, self.d, self.device)

    def step(self, table, lens, rows):
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=self.device)
        start = [sum(rows[:r]) for r in range(len(rows) + 1)]
        return vc.Kv8Step(table, i32(lens), i32(start), start[-1])

    def workspace(self, rows):
        n = vc.viscache_kv8_workspace_size(rows, self.Hq, self.Hkv, self.d)
        return torch.empty(n, dtype=torch.uint8, device=self.device)


def positions_of(frames, height, width, text, device):
    """int32 [3][rows]: (t, y, x) of each visual token, then text with one position on all axes."""
    vis = torch.cartesian_prod(*(torch.arange(n) for n in (frames, height, width))).t()
    first = max(frames, height, width)
    return torch.cat([vis, (first + torch.arange(text)).expand(3, -1)], 1).to(torch.int32).contiguous().to(device)


def prefill(m, x, positions):
    """All rows of a request through the model: hidden rows, and each layer's rotated q, k, v."""
    rows = x.shape[0]
    pages = -(-rows // m.page)
    cache, ws = m.pool(pages), m.workspace(rows)
    step = m.step(torch.arange(pages, dtype=torch.int32, device=m.device)[None], [rows], [rows])
    kept = []
    for layer in range(m.L):
        q, k, v = m.qkv(layer, x, positions)
        vc.viscache_kv8_append(cache, step, k, v, ws=ws)
        x = m.attend(layer, x, q, cache, step, ws)
        kept.append((q, k, v))
    return x, kept


class Server:
    """Requests in the 8-bit cache of every layer, decoded together."""

    def __init__(self, m, requests, retain=(1, 5), room=64, budget=0):
        """requests: (hidden rows, positions, visual tokens) of each; budget: the most tokens of a layer (0: all)."""
        self.m, self.n, self.budget = m, len(requests), budget
        plans = [vc.viscache_plan_budgets(m.L, n, *retain)[0] for _, _, n in requests]
        text = [x.shape[0] - n for x, _, n in requests]
        self.lens = [[b[layer] + t for b, t in zip(plans, text)] for layer in range(m.L)]
        need = [-(-(max(b) + t + room) // m.page) for b, t in zip(plans, text)]
        order = torch.randperm(sum(need)).to(torch.int32)
        self.table = torch.zeros(self.n, max(need), dtype=torch.int32)
        for r, k in enumerate(need):
            self.table[r, :k] = order[sum(need[:r]):sum(need[:r]) + k]
        self.table = self.table.to(m.device)
        self.pools = [m.pool(sum(need)) for _ in range(m.L)]
        last = []
        for r, (x, positions, n) in enumerate(requests):
            h, kept = prefill(m, x, positions)
            last.append(h[-1])
            self.admit(r, kept, n, text[r], retain)
        self.x = torch.stack(last)
        self.positions = torch.stack([p[:, -1] + 1 for _, p, _ in requests], 1).contiguous()
        # one row a request; the lengths count the row that a step appends
        self.steps = [m.step(self.table, [n + 1 for n in self.lens[layer]], [1] * self.n) for layer in range(m.L)]
        self.ws = m.workspace(self.n)
        self.graph = None
        if budget:
            # what every token of the prompt starts from: nothing yet
            self.weights = [torch.zeros(sum(need), m.Hkv, m.page, device=m.device) for _ in range(m.L)]
            self.lse = torch.empty(self.n, m.Hq, device=m.device)
            self.keep = torch.full((self.n,), budget, dtype=torch.int32, device=m.device)
            self.kept = torch.empty(self.n, m.Hkv, budget, dtype=torch.int32, device=m.device)
            self.evict_ws = torch.empty(vc.viscache_kv8_evict_workspace_size(self.n, m.Hkv), dtype=torch.uint8,
                                        device=m.device)

    def admit(self, r, kept, n, text, retain):
        """A prefilled request: its visual tokens compressed, then text, into the cache."""
        m = self.m
        Q, K, V = (torch.stack([rows[i].transpose(0, 1) for rows in kept]) for i in range(3))   # [L][H][rows][d]
        window = min(text, 16)
        batch = vc.Batch([n], [window], [retain])
        params = vc.make_params(m.L, m.Hq, m.Hkv, m.d, vc.VC_BF16)
        K_new, V_new, _ = vc.prunekv_compress(batch, params, Q[:, :, -window:].contiguous(),
                                              K[:, :, :n].contiguous(), V[:, :, :n].contiguous())
        ws, at = m.workspace(max(n, text)), 0
        for layer in range(m.L):
            B = self.lens[layer][r] - text
            if B > 0:
                block = [t[at:at + m.Hkv * B].view(m.Hkv, B, m.d).transpose(0, 1) for t in (K_new, V_new)]
                vc.viscache_kv8_append(self.pools[layer], m.step(self.table[r:r + 1], [B], [B]), *block, ws=ws)
                at += m.Hkv * B
            _, k, v = kept[layer]
            vc.viscache_kv8_append(self.pools[layer], m.step(self.table[r:r + 1], [B + text], [text]), k[n:], v[n:],
                                   ws=ws)

    def token(self):
        """One step of every request; everything that changes from step to step is on the device."""
        m, x = self.m, self.x
        for layer in range(m.L):
            q, k, v = m.qkv(layer, x, self.positions)
            vc.viscache_kv8_append(self.pools[layer], self.steps[layer], k, v, ws=self.ws)
            cache, step = self.pools[layer], self.steps[layer]
            x = m.attend(layer, x, q, cache, step, self.ws, self.lse if self.budget else None)
            if self.budget:
                vc.viscache_kv8_weigh(cache, step, q, self.lse, self.weights[layer], ws=self.ws)
                vc.viscache_kv8_evict(cache, step, self.weights[layer], self.keep, self.budget, sink=4, recent=16,
                                      kept=self.kept, new_lens=step.tensors[1], ws=self.evict_ws)
        self.x.copy_(x)                         # (a model would draw a token with viscache_sample and look its row up)
        self.positions += 1
        for step in self.steps:
            step.tensors[1].add_(1)

    def decode(self, count):
        if self.graph is None:
            self.token()                        # outside a graph first: the libraries' own set-up
            torch.cuda.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.token()
            count -= 1
        for _ in range(count):
            self.graph.replay()
        return self.x

    def rows(self, layer):
        """A layer's cached rows in 16 bits, request after request, and their counts."""
        m, lens = self.m, (self.steps[layer].tensors[1] - 1).tolist()
        step = m.step(self.table, lens, lens)
        K, V = vc.viscache_kv8_read(self.pools[layer], step, ws=m.workspace(max(step.n_rows, 1)))
        return K.split(lens), V.split(lens)


def main():
    m = Model()
    grids, text = [(8, 12, 16), (16, 10, 14)], [45, 30]
    requests = []
    for (t, h, w), n in zip(grids, text):
        requests.append((m.rand(t * h * w + n, m.hidden), positions_of(t, h, w, n, m.device), t * h * w))
    server = Server(m, requests)
    before = [list(n) for n in server.lens]
    x = server.decode(32)
    torch.cuda.synchronize()
    assert torch.isfinite(x).all()
    for layer in range(m.L):
        K, V = server.rows(layer)
        print("layer %d: visual tokens kept + text, after 32 steps: %s (of %s rows in the prompts)"
              % (layer, [k.shape[0] for k in K], [r[0].shape[0] for r in requests]))
        assert [k.shape[0] for k in K] == [n + 32 for n in before[layer]]
    tokens = sum(len(k) for layer in range(m.L) for k in server.rows(layer)[0])
    print("cache: %.1f KB in 8 bits, %.1f KB in 16" % (2 * tokens * m.Hkv * m.d / 1e3, 4 * tokens * m.Hkv * m.d / 1e3))


if __name__ == "__main__":
    main()
