"""Host models of the barrier protocols of the attention kernels over the 8-bit cache
(csrc/kv8_attn.cu, csrc/kv8_attn_tc2.cu, csrc/kv8_attn_tc1.cu).

Each role of a kernel (producer or loader, consumers, converters, MMA issuer, softmax of a
row tile) is a coroutine that makes the kernel's waits and arrivals in the kernel's order;
copies land in any order; the tensor pipe executes the issuer's batches in issue order, its
commits arriving on their barriers; a random scheduler interleaves everything.  A wait
tells phases apart by their parity alone, as an mbarrier does, and the model knows which
phase was meant: a wait that passes at any other phase, or that can never pass, is an error,
and so is a buffer read with another tile's contents or written while it is still needed.
Planted mistakes (a wait left out; a consumer that passes over the tiles it has no work in,
which a parity cannot tell from the ones before) must be caught.  The models have no
arithmetic.
"""
import random

import pytest


class ProtocolError(AssertionError):
    pass


def need(cond, what):
    if not cond:
        raise ProtocolError(what)


class Bar:
    def __init__(self, count=1):
        self.count, self.pending, self.done = count, 0, 0

    def arrive(self):
        self.pending += 1
        need(self.pending <= self.count, "more arrivals than a phase takes")
        if self.pending == self.count:
            self.pending, self.done = 0, self.done + 1


def schedule(rnd, roles, events):
    """Runs the coroutines to their ends; `events`: callables that perform one pending event
    (a copy that lands, the next batch of the pipe) or return False if there is none; they are
    told whether anything else can go on (a slow copy then mostly does not land yet)."""
    waiting = {}                       # role -> (barrier, phase) or None
    live = dict(enumerate(roles))
    for k, g in list(live.items()):
        waiting[k] = next(g, "end")
        if waiting[k] == "end":
            del live[k]
    while live:
        # a wait passes when the phase of its parity counts as completed: the current one has the other
        ready = [k for k in live if waiting[k] is None or waiting[k][0].done & 1 != waiting[k][1] & 1]
        acts = ready + ["event"] * (1 + len(ready) // 2)
        rnd.shuffle(acts)
        for k in acts:
            if k == "event":
                if any(e(bool(ready)) for e in rnd.sample(events, len(events))):
                    break
                continue
            if waiting[k] is not None:
                bar, phase = waiting[k]
                need(bar.done == phase + 1, "a wait passed at another phase than it meant")
            waiting[k] = next(live[k], "end")
            if waiting[k] == "end":
                del live[k]
            break
        else:
            raise ProtocolError("nothing can go on")


# ---------------------------------------------------------------------------------------
# the few-rows kernel: a ring of tiles, chunks dealt to the consumers in turn

def run_ring(tiles, warps, stages, seed, mistake=None):
    rnd = random.Random(seed)
    chunks = 8
    full = [Bar(3) for _ in range(stages)]              # expected bytes, scales, the copies
    empty = [Bar(chunks if mistake == "pass over" else warps) for _ in range(stages)]
    content, readers, flying, seen = [None] * stages, [0] * stages, [], []
    slow = {f for f in range(tiles) if rnd.random() < 0.15}

    def producer():
        for f in range(tiles):
            st = f % stages
            if mistake != "empty":
                yield empty[st], f // stages - 1
            full[st].arrive()
            flying.append(f)
            yield None
            full[st].arrive()

    def consumer(w):
        for f in range(tiles):
            st = f % stages
            mine = [c for c in range(chunks) if (chunks * f + c) % warps == w]
            if mistake == "pass over" and not mine:
                continue
            if mistake != "full":
                yield full[st], f // stages
            for c in mine:
                readers[st] += 1
                yield None
                need(content[st] == f, "a chunk of another tile was read")
                readers[st] -= 1
                seen.append((f, c))
                if mistake == "pass over":
                    empty[st].arrive()
            if mistake != "pass over":
                empty[st].arrive()

    def land(busy):
        quick = [f for f in flying if f not in slow or not busy or rnd.random() < 0.02]
        if not quick:
            return False
        f = rnd.choice(quick)
        flying.remove(f)
        st = f % stages
        need(readers[st] == 0, "a copy landed on a tile that is being read")
        content[st] = f
        full[st].arrive()
        return True

    schedule(rnd, [producer()] + [consumer(w) for w in range(warps)], [land])
    need(sorted(seen) == [(f, c) for f in range(tiles) for c in range(chunks)], "a chunk was missed or done twice")


@pytest.mark.parametrize("warps,stages", [(15, 5), (11, 5), (7, 5), (15, 10), (3, 2)])
def test_ring_holds(warps, stages):
    for seed in range(40):
        run_ring(random.Random(seed).randrange(0, 40), warps, stages, seed)


@pytest.mark.parametrize("mistake", ["pass over", "empty", "full"])
def test_ring_mistakes_are_caught(mistake):
    caught = 0
    for seed in range(200):
        try:
            run_ring(60, 15, 5, seed, mistake)
        except ProtocolError:
            caught += 1
    assert caught > 0


# ---------------------------------------------------------------------------------------
# the many-rows kernel

K_STAGES, V_STAGES, CODE_STAGES, REFS = 3, 2, 2, 8


def run_chunks(segments, seed, mistake=None):
    """segments: (tiles, both row tiles have rows) of each."""
    rnd = random.Random(seed)
    mk = lambda n: [Bar() for _ in range(n)]
    k_full, k_empty, v_full, v_empty = mk(K_STAGES), mk(K_STAGES), mk(V_STAGES), mk(V_STAGES)
    code_full, code_empty, ref_full = mk(CODE_STAGES), mk(CODE_STAGES), mk(REFS)
    s_full, p_half, p_full, o_full, (q_full, q_empty) = mk(2), mk(2), mk(2), mk(2), mk(2)
    K, V, code, ref, q = [None] * K_STAGES, [None] * V_STAGES, [None] * CODE_STAGES, [None] * REFS, [None]
    S, sums = [None, None], [[], []]                        # sums: tiles added to O of a row tile
    P = [[None, None], [None, None]]                        # P of a row tile, in halves
    flying, pipe, read_o = [], [], [0, 0]

    def w(name, bar, phase):
        return None if mistake == name else (bar, phase)

    def loader():
        t = 0
        for n, _ in segments:
            for _ in range(n):
                yield w("k_empty", k_empty[t % K_STAGES], t // K_STAGES - 1)
                ref[t % REFS] = t
                ref_full[t % REFS].arrive()
                flying.append(("K", t))
                yield w("code_empty", code_empty[t % CODE_STAGES], t // CODE_STAGES - 1)
                flying.append(("V", t))
                t += 1

    def converters():
        t = 0
        for seg, (n, _) in enumerate(segments):
            yield w("q_empty", q_empty, seg - 1)
            need(not any(b[0] == "S" for b in pipe), "query rows written under an S that reads them")
            q[0] = seg
            q_full.arrive()
            for _ in range(n):
                st, cst = t % V_STAGES, t % CODE_STAGES
                yield w("code_full", code_full[cst], t // CODE_STAGES)
                yield w("v_empty", v_empty[st], t // V_STAGES - 1)
                need(code[cst] == t, "codes of another tile expanded")
                need(not any(b[0] == "PV" and b[2] % V_STAGES == st for b in pipe), "V written under its product")
                V[st] = t
                yield None
                code_empty[cst].arrive()
                v_full[st].arrive()
                t += 1

    def issuer():
        t, np = 0, [0, 0]
        for seg, (n, two) in enumerate(segments):
            xs = [0, 1] if two else [0]
            yield w("q_full", q_full, seg)
            yield w("k_full", k_full[t % K_STAGES], t // K_STAGES)
            for x in xs:
                pipe.append(("S", x, t, seg))
                pipe.append(("commit", s_full[x]))
            pipe.append(("commit", k_empty[t % K_STAGES]))
            for j in range(n):
                st, more = t % V_STAGES, j + 1 < n
                yield w("v_full", v_full[st], t // V_STAGES)
                for x in xs:
                    yield w("p_half", p_half[x], np[x])
                    pipe.append(("PV", x, t, 0, j == 0))
                    yield w("p_full", p_full[x], np[x])
                    np[x] += 1
                    pipe.append(("PV", x, t, 1, j == 0))
                    if not more:
                        pipe.append(("commit", o_full[x]))
                    if x == xs[-1]:
                        pipe.append(("commit", v_empty[st]))
                    if more:
                        if x == 0:
                            yield w("k_full", k_full[(t + 1) % K_STAGES], (t + 1) // K_STAGES)
                        pipe.append(("S", x, t + 1, seg))
                        pipe.append(("commit", s_full[x]))
                if more:
                    pipe.append(("commit", k_empty[(t + 1) % K_STAGES]))
                t += 1
            pipe.append(("commit", q_empty))

    def softmax(x):
        t, ns, no = 0, 0, 0
        for seg, (n, two) in enumerate(segments):
            if x == 1 and not two:
                t += n
                continue
            for j in range(n):
                if mistake == "scales first":
                    yield ref_full[t % REFS], t // REFS
                yield w("s_full", s_full[x], ns)
                ns += 1
                if mistake != "scales first":
                    yield ref_full[t % REFS], t // REFS
                if j == 0:
                    yield q_full, seg
                need(S[x] == t, "scores of another tile")
                need(ref[t % REFS] == t, "scales of another tile")
                if j and rnd.random() < 0.3:        # O is rescaled
                    need(sums[x] == list(range(t - j, t)), "O rescaled under a product")
                    yield None
                    need(sums[x] == list(range(t - j, t)), "O rescaled under a product")
                S[x], P[x] = None, [t, None]
                yield None
                p_half[x].arrive()
                yield None
                P[x][1] = t
                yield None
                p_full[x].arrive()
                t += 1
            yield w("o_full", o_full[x], no)
            no += 1
            need(sums[x] == list(range(t - n, t)), "O read before its last product")
            yield None
            need(sums[x] == list(range(t - n, t)), "O overwritten while it is read")

    def land(_):
        if not flying:
            return False
        kind, t = flying.pop(rnd.randrange(len(flying)))
        if kind == "K":
            need(not any(b[0] == "S" and b[2] % K_STAGES == t % K_STAGES for b in pipe), "K written under its product")
            K[t % K_STAGES] = t
            k_full[t % K_STAGES].arrive()
        else:
            code[t % CODE_STAGES] = t
            code_full[t % CODE_STAGES].arrive()
        return True

    def batch(_):
        if not pipe:
            return False
        b = pipe[0]
        if b[0] == "commit":
            b[1].arrive()
        elif b[0] == "S":
            _, x, t, seg = b
            need(K[t % K_STAGES] == t and q[0] == seg, "S of other keys or rows")
            need(S[x] is None, "S written before it was read")
            S[x] = t
        else:
            _, x, t, h, first = b
            need(P[x][h] == t and V[t % V_STAGES] == t, "PV of another tile")
            P[x][h] = None
            if h:
                sums[x] = [t] if first else sums[x] + [t]
        pipe.pop(0)
        return True

    schedule(rnd, [loader(), converters(), issuer(), softmax(0), softmax(1)], [land, batch])


def _segments(seed):
    r = random.Random(1000 + seed)
    return [(r.choice([1, 1, 2, 3, 5, 12, 30]), r.random() < 0.6) for _ in range(r.randrange(1, 7))]


def test_chunk_protocol_holds():
    for seed in range(150):
        run_chunks(_segments(seed), seed)


@pytest.mark.parametrize("mistake", ["k_empty", "code_empty", "code_full", "v_empty", "q_empty", "q_full", "k_full",
                                     "v_full", "p_half", "p_full", "s_full", "o_full", "scales first"])
def test_chunk_protocol_mistakes_are_caught(mistake):
    caught = 0
    for seed in range(150):
        try:
            run_chunks(_segments(seed), seed, mistake)
        except ProtocolError:
            caught += 1
    assert caught > 0, mistake


# ---------------------------------------------------------------------------------------
# one row tile, two S buffers; fp32 rows: K expanded a tile ahead of V; 16-bit rows: K by TMA

def run_rows(segments, seed, f32, mistake=None):
    """segments: tiles of each."""
    rnd = random.Random(seed)
    mk = lambda n: [Bar() for _ in range(n)]
    ks, vs, ring = (2, 1, 4) if f32 else (3, 2, 3)
    fold = 4 if f32 else 1 << 30        # tiles whose products O takes before it goes into the sum
    k_full, k_empty, v_full, v_empty, pv_done = mk(ks), mk(ks), mk(vs), mk(vs), Bar()
    code_full, code_empty, ref_full = mk(ring), mk(ring), mk(REFS)
    s_full, p_half, p_full, q_full, q_empty = mk(2), mk(2), Bar(), Bar(), Bar()
    K, V, code, ref, q, qs = [None] * ks, [None] * vs, [None] * ring, [None] * REFS, [None], [None]
    S, P, added = [None, None], [[None, None], [None, None]], []
    flying, pipe, late = [], [], []     # late: commits whose batches are done; they arrive in any order

    def w(name, bar, phase):
        return None if mistake == name else (bar, phase)

    def items(n, t, ahead):
        # the order of a segment whose first tile is t: K, K, V, K, V, ... or K, V, K, V, ...
        for j in range(n + 1):
            if j < n:
                yield "K", t + j
            if ahead and j > 0:
                yield "V", t + j - 1
            elif not ahead and j < n:
                yield "V", t + j

    def k_free(x):
        need(not any(b[0] == "S" and b[1] % ks == x % ks for b in pipe), "K written under its product")

    def loader():
        t, item = 0, 0
        for n in segments:
            for kind, x in items(n, t, f32):
                if kind == "K" and not f32:
                    yield w("k_empty", k_empty[x % ks], x // ks - 1)
                else:
                    yield w("code_empty", code_empty[item % ring], item // ring - 1)
                if kind == "K":
                    ref[x % REFS] = x
                    ref_full[x % REFS].arrive()
                flying.append((kind, x, item))
                item += kind == "V" or f32
            t += n

    def converters():
        t, item = 0, 0
        for seg, n in enumerate(segments):
            yield w("q_empty", q_empty, seg - 1)
            need(not any(b[0] == "S" for b in pipe), "query rows written under an S that reads them")
            q[0], qs[0] = seg, seg
            yield None
            q_full.arrive()
            for kind, x in items(n, t, f32):
                if kind == "K" and not f32:
                    continue
                yield w("code_full", code_full[item % ring], item // ring)
                if kind == "K":
                    yield w("k_empty", k_empty[x % ks], x // ks - 1)
                    k_free(x)
                    K[x % ks] = x
                else:
                    yield w("v_empty", v_empty[x % vs], x // vs - 1)
                    need(not any(b[0] == "PV" and b[1] % vs == x % vs for b in pipe), "V written under its product")
                    need(ref[x % REFS] == x, "scales of another tile")
                    V[x % vs] = x
                need(code[item % ring] == (kind, x), "codes of another tile expanded")
                yield None
                code_empty[item % ring].arrive()
                (k_full[x % ks] if kind == "K" else v_full[x % vs]).arrive()
                item += 1
            t += n

    def issuer():
        t = 0
        for seg, n in enumerate(segments):
            yield w("q_full", q_full, seg)
            for kind, x in items(n, t, True):
                if kind == "K":
                    yield w("k_full", k_full[x % ks], x // ks)
                    pipe.append(("S", x, seg))
                    pipe.append(("commit", s_full[x & 1]))
                    pipe.append(("commit", k_empty[x % ks]))
                    if mistake == "rows early" and x == t + n - 1:
                        pipe.append(("commit", q_empty))
                else:
                    yield w("v_full", v_full[x % vs], x // vs)
                    yield w("p_half", p_half[x & 1], x >> 1)
                    pipe.append(("PV", x, 0, (x - t) % fold == 0))
                    yield w("p_full", p_full, x)
                    pipe.append(("PV", x, 1, (x - t) % fold == 0))
                    pipe.append(("commit", pv_done))
                    pipe.append(("commit", v_empty[x % vs]))
            if mistake != "rows early":
                pipe.append(("commit", q_empty))
            t += n

    def softmax():
        t = 0
        for seg, n in enumerate(segments):
            for j in range(n):
                yield w("s_full", s_full[t & 1], t >> 1)
                yield ref_full[t % REFS], t // REFS
                if j == 0:
                    yield q_full, seg
                    need(qs[0] == seg, "powers of two of other rows")
                need(S[t & 1] == t, "scores of another tile")
                need(ref[t % REFS] == t, "scales of another tile")
                if j == 0:
                    summed = []
                if j and (j % fold == 0 or rnd.random() < 0.3):     # O is rescaled, or added to the sum
                    yield w("rescale", pv_done, t - 1)
                    need(summed + added == list(range(t - j, t)), "O rescaled under a product")
                    yield None
                    need(summed + added == list(range(t - j, t)), "O rescaled under a product")
                    if j % fold == 0:
                        summed = summed + added
                S[t & 1], P[t & 1] = None, [t, None]
                yield None
                p_half[t & 1].arrive()
                yield None
                P[t & 1][1] = t
                if mistake != "in turn":
                    yield pv_done, t - 1
                p_full.arrive()
                t += 1
            yield w("last", pv_done, t - 1)
            need(summed + added == list(range(t - n, t)), "O read before its last product")
            yield None
            need(summed + added == list(range(t - n, t)), "O overwritten while it is read")

    def land(_):
        if not flying:
            return False
        kind, x, item = flying.pop(rnd.randrange(len(flying)))
        if kind == "K" and not f32:
            k_free(x)
            K[x % ks] = x
            k_full[x % ks].arrive()
        else:
            code[item % ring] = (kind, x)
            code_full[item % ring].arrive()
        return True

    def batch(_):
        if late and (not pipe or rnd.random() < 0.6):
            late.pop(rnd.randrange(len(late))).arrive()
            return True
        if not pipe:
            return False
        b = pipe.pop(0)
        if b[0] == "commit":
            late.append(b[1])
        elif b[0] == "S":
            _, x, seg = b
            need(K[x % ks] == x and q[0] == seg, "S of other keys or rows")
            need(S[x & 1] is None and P[x & 1] == [None, None], "S written before it was read, or over a P")
            S[x & 1] = x
        else:
            _, x, h, first = b
            need(P[x & 1][h] == x and V[x % vs] == x, "PV of another tile")
            P[x & 1][h] = None
            if h:
                added[:] = [x] if first else added + [x]
        return True

    schedule(rnd, [loader(), converters(), issuer(), softmax()], [land, batch])


def _tiles(seed):
    r = random.Random(2000 + seed)
    return [r.choice([1, 1, 1, 2, 2, 3, 5, 12, 30]) for _ in range(r.randrange(1, 8))]


@pytest.mark.parametrize("f32", [False, True])
def test_row_tile_protocol_holds(f32):
    for seed in range(250):
        run_rows(_tiles(seed), seed, f32)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("mistake", ["code_empty", "code_full", "k_empty", "k_full", "v_empty", "v_full", "q_empty",
                                     "s_full", "p_half", "p_full", "rescale", "in turn", "last", "rows early"])
def test_row_tile_protocol_mistakes_are_caught(mistake, f32):
    caught = 0
    for seed in range(300):
        try:
            run_rows(_tiles(seed), seed, f32, mistake)
        except ProtocolError:
            caught += 1
    assert caught > 0, mistake


def test_issuers_wait_for_query_rows():
    # needed where K comes by TMA; where K is expanded it is implied (a segment's rows come before its first K)
    for seed in range(200):
        run_rows(_tiles(seed), seed, True, "q_full")
    with pytest.raises(ProtocolError):
        for seed in range(200):
            run_rows(_tiles(seed), seed, False, "q_full")
