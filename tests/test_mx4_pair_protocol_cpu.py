"""The barriers of the mx4 product's CTA pairs, as a model on the CPU: two copying threads a CTA, the second CTA's announcement of
its stages to the first, the first's MMAs, both epilogues, in random order. No deadlock; a wait never looks at a phase that
another has passed; MMAs find the bytes of their own stage and block of the contraction in both CTAs, and an empty accumulator."""
import random

import pytest


class Barrier:
    """mbarrier: `need` arrivals (and announced bytes) complete a phase."""

    def __init__(self, need):
        self.need, self.left, self.bytes, self.phase, self.waiting = need, need, 0, 0, set()

    def arrive(self, expect=0):
        assert self.left > 0, "an arrival more than the phase takes"
        self.left -= 1
        self.bytes += expect
        self.turn()

    def land(self, n):
        self.bytes -= n
        self.turn()

    def turn(self):
        if self.left == 0 and self.bytes == 0:
            self.phase, self.left = self.phase + 1, self.need

    def passed(self, parity, seen):
        """A wait for the completion of phase `seen` by its parity; at most one phase may have completed since."""
        assert parity == seen & 1 and self.phase <= seen + 1, "the wait looks at a phase that has been passed"
        return self.phase > seen


def run(seed, stages, blocks, items):
    rng = random.Random(seed)
    full = [[Barrier(2 if r == 0 else 1) for _ in range(stages)] for r in (0, 1)]
    empty = [[Barrier(1) for _ in range(stages)] for _ in (0, 1)]
    tfull, tempty = [Barrier(1), Barrier(1)], Barrier(4)  # (two warps of each CTA's epilogue)
    ring = [[{} for _ in range(stages)] for _ in (0, 1)]
    flying, pending, acc, out = [], [], {"state": "empty"}, []

    def copier(r, kind):
        for n in range(items * blocks):
            s, turn = n % stages, n // stages
            while turn and not empty[r][s].passed((turn - 1) & 1, turn - 1):
                yield
            if kind == "B":
                full[r][s].arrive(expect=2)
                yield
            flying.append((r, s, kind, n))
            yield

    def announcer():
        for n in range(items * blocks):
            s, turn = n % stages, n // stages
            while not full[1][s].passed(turn & 1, turn):
                yield
            full[0][s].arrive()
            yield

    def mma():
        for i in range(items):
            while i and not tempty.passed((i - 1) & 1, i - 1):
                yield
            assert acc["state"] == "empty"
            acc.update(state="filling", item=i)
            for k in range(blocks):
                n = i * blocks + k
                s, turn = n % stages, n // stages
                while not full[0][s].passed(turn & 1, turn):
                    yield
                for r in (0, 1):
                    assert ring[r][s] == {"A": n, "B": n}, "a stage that is not complete"
                pending.append(("empty", s))
                yield
            pending.append(("tfull", i))
            yield

    def hardware():
        while True:
            if flying and rng.random() < 0.5:
                r, s, kind, n = flying.pop(rng.randrange(len(flying)))
                ring[r][s][kind] = n
                full[r][s].land(1)
            elif pending and rng.random() < 0.5:  # commits, in order
                what, v = pending.pop(0)
                if what == "tfull":
                    acc["state"] = "full"
                for r in (0, 1):
                    (empty[r][v] if what == "empty" else tfull[r]).arrive()
            yield

    def epilogue(r):
        for i in range(items):
            while not tfull[r].passed(i & 1, i):
                yield
            assert acc["state"] == "full" and acc["item"] == i
            out.append((r, i))
            yield
            if len([o for o in out if o[1] == i]) == 4:
                acc["state"] = "empty"
            tempty.arrive()
            yield

    agents = [copier(r, k) for r in (0, 1) for k in "AB"] + [announcer(), mma()] + [epilogue(r) for r in (0, 0, 1, 1)]
    engine, live = hardware(), list(agents)
    for _ in range(400 * items * blocks + 4000):
        if not live:
            break
        a = rng.choice(live + [engine])
        try:
            next(a)
        except StopIteration:
            live.remove(a)
    assert not live, "the pair has stopped"
    assert sorted(out) == sorted((r, i) for i in range(items) for r in (0, 0, 1, 1))


@pytest.mark.parametrize("stages,blocks,items", [(6, 8, 5), (6, 9, 7), (6, 1, 9), (2, 5, 4), (6, 16, 3)])
def test_pairs(stages, blocks, items):
    for seed in range(20):
        run(seed, stages, blocks, items)


def test_a_lost_announcement_is_seen():
    """The model's own check: without the peer's announcement the first CTA's barrier never turns."""
    b = Barrier(2)
    b.arrive(expect=1)
    b.land(1)
    assert not b.passed(0, 0)
