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
    q_full, q_empty = [Bar(LOADERS + 1) for _ in range(2)], [Bar() for _ in range(2)]
    l_full, l_empty = [Bar(LOADERS) for _ in range(2)], [Bar(EPILOGUE) for _ in range(2)]
    d_full, d_empty = [Bar() for _ in range(2)], [Bar(EPILOGUE) for _ in range(2)]
    k_empty = Bar(EPILOGUE)
    K, Q, lse = [None] * LOADERS, [None, None], [[None] * LOADERS for _ in range(2)]
    D, pipe, sums, flying = [None, None], [], [], []
    meet = Bar(EPILOGUE)                        # the epilogue warps at a segment's end
    parts = {}

    def w(name, bar, phase):
        return None if mistake == name else (bar, phase)

    def loader(me):
        step = 0
        for seg, (n, _) in enumerate(segments):
            for j in range(n):
                st = step & 1
                yield w("q_empty", q_empty[st], (step >> 1) - 1)
                need(all(b[0] != "P" or b[2] != st for b in pipe), "query rows written under a product")
                if me == 0:
                    flying.append(step)
                if j == 0:
                    # the first rows are on their way before the unit's K is
                    yield w("k_empty", k_empty, seg - 1)
                    need(not any(b[0] == "P" and b[3] < seg for b in pipe), "K written under a product")
                    need(parts.get(seg - 1, EPILOGUE) == EPILOGUE, "K written while the quarters' sums lie there")
                    K[me] = seg                 # (reported with the first step's rows)
                q_full[st].arrive()
                yield w("l_empty", l_empty[st], (step >> 1) - 1)
                lse[st][me] = step
                l_full[st].arrive()
                step += 1

    def issuer():
        step = prod = 0
        for seg, (n, nt) in enumerate(segments):
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
            meet.arrive()
            yield meet, seg
            parts[seg] += 1
            k_empty.arrive()

    def execute(busy):
        if not pipe:
            return False
        b = pipe.pop(0)
        if b[0] == "Q":
            q_empty[b[1]].arrive()
            return True
        _, d, st, seg, step, kt = b
        need(K == [seg] * LOADERS, "a product of another unit's K")
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


@pytest.mark.parametrize("mistake", ["k_empty", "q_empty", "q_full", "d_empty", "d_full", "l_empty", "l_full"])
def test_mistakes_are_caught(mistake):
    caught = 0
    for seed in range(60):
        try:
            run(_segments(seed), seed, mistake)
        except ProtocolError:
            caught += 1
    assert caught > 0
