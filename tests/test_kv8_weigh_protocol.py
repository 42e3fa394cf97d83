"""Host model of the barrier protocol of the many-rows kernel of viscache_kv8_weigh
(csrc/kv8_weigh_tc.cu): loaders, MMA issuer and epilogue warps as coroutines that make the
kernel's waits and arrivals in its order, under the scheduler of the attention kernels' models."""
import random

import pytest

from tests.test_kv8_protocol import Bar, ProtocolError, need, schedule

LOADERS, EPILOGUE = 4, 16


def run(segments, seed, mistake=None):
    """segments: (steps, K tiles) of each unit's piece."""
    rnd = random.Random(seed)
    q_full, q_empty = [Bar(2) for _ in range(2)], [Bar() for _ in range(2)]
    l_full, l_empty = [Bar(LOADERS) for _ in range(2)], [Bar(EPILOGUE) for _ in range(2)]
    d_full, d_empty = [Bar() for _ in range(2)], [Bar(EPILOGUE) for _ in range(2)]
    k_full = Bar(EPILOGUE)
    K, Q, lse = [None] * EPILOGUE, [None, None], [[None] * LOADERS for _ in range(2)]
    D, pipe, sums, flying = [None, None], [], [], []
    start, meet = Bar(EPILOGUE), Bar(EPILOGUE)                        # the epilogue warps at a segment's end
    parts, wrote = {}, set()

    def w(name, bar, phase):
        return None if mistake == name else (bar, phase)

    def loader(me):
        step = 0
        for seg, (n, _) in enumerate(segments):
            for j in range(n):
                st = step & 1
                if me == 0 or mistake == "all wait":
                    yield w("q_empty", q_empty[st], (step >> 1) - 1)
                if me == 0:
                    need(all(b[0] != "P" or b[2] != st for b in pipe), "query rows written under a product")
                    flying.append(step)
                    q_full[st].arrive()
                yield w("l_empty", l_empty[st], (step >> 1) - 1)
                lse[st][me] = step
                l_full[st].arrive()
                step += 1

    def issuer():
        step = prod = 0
        for seg, (n, nt) in enumerate(segments):
            yield w("k_full", k_full, seg)
            for j in range(n):
                st = step & 1
                yield w("q_full", q_full[st], step >> 1)
                for kt in range(nt):
                    yield w("d_empty", d_empty[prod & 1], (prod >> 1) - 1)
                    pipe.append(("P", prod & 1, st, seg, step, kt))
                    prod += 1
                pipe.append(("Q", st))
                step += 1

    def epilogue(me):
        step = prod = 0
        for seg, (n, nt) in enumerate(segments):
            start.arrive()
            yield w("start", start, seg)
            need(not any(b[0] == "P" for b in pipe), "K written under a product")
            need(parts.get(seg - 1, 4) == 4, "K written while the quarters' sums lie there")
            K[me] = seg
            k_full.arrive()
            for j in range(n):
                st = step & 1
                yield w("l_full", l_full[st], step >> 1)
                for kt in range(nt):
                    b = prod & 1
                    yield w("d_full", d_full[b], prod >> 1)
                    need(D[b] == (seg, step, kt), "another product's columns were read")
                    d_empty[b].arrive()
                    prod += 1
                    yield None
                    need(lse[st] == [step] * LOADERS, "another step's lse was read")
                    sums.append((me, seg, step, kt))
                l_empty[st].arrive()
                step += 1
            parts[seg] = parts.get(seg, 0)
            need(not any(b[0] == "P" for b in pipe), "sums written over K under a product")
            wrote.add((seg, me))
            meet.arrive()
            yield w("meet", meet, seg)
            parts.setdefault(seg, 0)
            if me < 4:                          # the quarter that adds the others' sums
                need(all((seg, x) in wrote for x in range(4, EPILOGUE)), "sums read before they were written")
                yield None
                parts[seg] += 1

    def execute(busy):
        if not pipe:
            return False
        b = pipe.pop(0)
        if b[0] == "Q":
            q_empty[b[1]].arrive()
            return True
        _, d, st, seg, step, kt = b
        need(K == [seg] * EPILOGUE, "a product of another unit's K")
        need(Q[st] == step, "a product of another step's rows")
        D[d] = (seg, step, kt)
        d_full[d].arrive()
        return True

    def land(busy):
        if not flying:
            return False
        step = flying.pop(rnd.randrange(len(flying)))
        need(all(b[0] != "P" or b[2] != step & 1 for b in pipe), "rows landed under a product that reads others")
        Q[step & 1] = step
        q_full[step & 1].arrive()
        return True

    schedule(rnd, [loader(i) for i in range(LOADERS)] + [issuer()] + [epilogue(i) for i in range(EPILOGUE)],
             [execute, land])
    want = EPILOGUE * sum(n * nt for n, nt in segments)
    need(len(sums) == len(set(sums)) == want, "a product was missed or added twice")


def _segments(seed):
    rnd = random.Random(seed)
    return [(rnd.randrange(1, 7), rnd.randrange(1, 4)) for _ in range(rnd.randrange(1, 6))]


def test_protocol_holds():
    for seed in range(60):
        run(_segments(seed), seed)


@pytest.mark.parametrize("mistake", ["k_full", "start", "q_empty", "q_full", "d_empty", "d_full", "l_empty", "l_full", "meet", "all wait"])
def test_mistakes_are_caught(mistake):
    caught = 0
    for seed in range(60):
        try:
            run(_segments(seed), seed, mistake)
        except ProtocolError:
            caught += 1
    assert caught > 0
