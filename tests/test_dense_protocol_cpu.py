"""The barrier protocol of the dense block's products (dense_gemm_kernel in csrc/dense_gemm.cu), modelled on the CPU.

Two producers (one a CTA of the pair) fill the stages of a ring; both CTAs' bytes are counted on the leader's full[s], whose one arrival is
the leader's own. The leader's MMA thread consumes the stages in order; its commits arrive on empty[s] and tfull[b] of both CTAs.
Every epilogue warp of both CTAs releases an accumulator by an arrival on the leader's tempty[b]. Three forms of an item:

* plain: one accumulator, two of them in turn over the items;
* runs: an item's contraction by several accumulators, the two in turn over items and runs (operands in parts: runs of all products);
* both: dh into one of two buffers, then g and u into the one accumulator there is. Only the latter waits for tempty; dh's buffer
  is free because the turn before last has been released by then.

Over random interleavings of all of it, with copies and commits that complete late (commits in the order of their issue, as the tensor pipe
completes), the model checks that nothing deadlocks, that each parity wait is within one phase of its barrier, that arrivals
and bytes go to the phase that they belong to, and that no MMA writes an accumulator that an epilogue warp has yet to read, and no copy a
stage that an MMA has yet to read."""
import random

import pytest


class ProtocolError(AssertionError):
    pass


def _turns(form, items, run):
    """The accumulators in the order of their use: (barrier, phases), a phase (buffer, steps)."""
    out = []
    for steps in items:
        if form == "both":
            out.append((0, [(f"dh{len(out) % 2}", steps), ("gu", steps)]))
        else:
            left = steps
            while left > 0:
                n = min(run, left) if form == "runs" else left
                b = len(out) % 2
                out.append((b, [(f"acc{b}", n)]))
                left -= n
    return out


class Model:
    def __init__(self, form, items, stages, seed, run=3, warps=4, one_dh=False, releases=None):
        self.rnd, self.stages, self.warps = random.Random(seed), stages, warps
        self.turns = _turns(form, items, run)
        if one_dh:
            self.turns = [(b, [("dh0" if buf.startswith("dh") else buf, n) for buf, n in ph]) for b, ph in self.turns]
        self.both = form == "both"
        self.releases = 2 * warps if releases is None else releases
        self.total = sum(n for _, ph in self.turns for _, n in ph)
        self.done, self.count, self.bytes = {}, {}, {}
        self.landing, self.commits = [], []  # copies in flight (any order), commits in flight (in order)
        self.made, self.used = [0, 0], 0  # steps that each producer has issued, the MMA thread has consumed
        self.read = [0] * len(self.turns)  # epilogue warps that have read a turn's buffers
        self.written = {}  # buffer -> the last turn that wrote it
        self.freed = 0  # stages whose MMAs have completed
        self.warp_turn = {(r, w): 0 for r in (0, 1) for w in range(warps)}
        self.turn = self.phase = self.step = 0
        self.began = False

    def passed(self, name, phase):
        """Whether a wait by the parity of `phase` passes."""
        d = self.done.get(name, 0)
        if not phase <= d <= phase + 1:
            raise ProtocolError(f"a wait for phase {phase} of {name}, which has completed {d}")
        return d == phase + 1

    def complete(self, name, phase):
        if self.done.get(name, 0) != phase:
            raise ProtocolError(f"an arrival for phase {phase} of {name} in phase {self.done.get(name, 0)}")
        self.done[name] = phase + 1

    def fill(self, step, what):
        s, phase = step % self.stages, step // self.stages
        if self.done.get(("full", s), 0) != phase:
            raise ProtocolError(f"{what} of step {step} in another phase of full[{s}]")
        got = self.bytes.setdefault(s, set())
        if what in got:
            raise ProtocolError(f"{what} twice in a phase of full[{s}]")
        got.add(what)
        if len(got) == 3:
            got.clear()
            self.complete(("full", s), phase)

    def turn_index(self, t):
        """(barrier, phase of its tfull and tempty) of a turn."""
        return (0, t) if self.both else (t % 2, t // 2)

    def may_begin(self):
        """The MMA thread's wait for the accumulator of this turn and phase."""
        b, phase = self.turn_index(self.turn)
        if self.both and self.phase == 0:
            return True
        return phase == 0 or self.passed(("tempty", b), phase - 1)

    def moves(self):
        out = []
        for r in (0, 1):
            step = self.made[r]
            if step < self.total and (step < self.stages or self.passed(("empty", r, step % self.stages), step // self.stages - 1)):
                out.append(("make", r))
        if self.turn < len(self.turns):
            if not self.began:
                if self.may_begin():
                    out.append(("begin",))
            elif self.passed(("full", self.used % self.stages), self.used // self.stages):
                out.append(("mma",))
        for (r, w), t in self.warp_turn.items():
            if t < len(self.turns):
                b, phase = self.turn_index(t)
                if self.passed(("tfull", r, b), phase):
                    out.append(("read", r, w))
        if self.landing:
            out.append(("land",))
        if self.commits:
            out.append(("commit",))
        return out

    def do(self, m):
        if m[0] == "make":
            r, step = m[1], self.made[m[1]]
            if step >= self.stages and self.freed <= step - self.stages:
                raise ProtocolError("a copy over a stage that an MMA has yet to read")
            if r == 0:
                self.fill(step, "arrival")
            self.landing.append((r, step))
            self.made[r] += 1
        elif m[0] == "land":
            r, step = self.landing.pop(self.rnd.randrange(len(self.landing)))
            self.fill(step, f"bytes of {r}")
        elif m[0] == "begin":
            buf = self.turns[self.turn][1][self.phase][0]
            last = self.written.get(buf)
            if last is not None and self.read[last] != 2 * self.warps:
                raise ProtocolError(f"{buf} is written in turn {self.turn} before turn {last} has been read")
            self.written[buf] = self.turn
            self.began = True
        elif m[0] == "mma":
            self.commits.append(("empty", self.used))
            self.used += 1
            self.step += 1
            if self.step == self.turns[self.turn][1][self.phase][1]:
                self.step, self.began = 0, False
                self.phase += 1
                if self.phase == len(self.turns[self.turn][1]):
                    self.commits.append(("tfull", self.turn))
                    self.phase = 0
                    self.turn += 1
        elif m[0] == "commit":
            what, n = self.commits.pop(0)
            for r in (0, 1):
                if what == "empty":
                    self.complete(("empty", r, n % self.stages), n // self.stages)
                else:
                    b, phase = self.turn_index(n)
                    self.complete(("tfull", r, b), phase)
            if what == "empty":
                self.freed = n + 1
        else:
            _, r, w = m
            t = self.warp_turn[(r, w)]
            self.read[t] += 1
            b, phase = self.turn_index(t)
            if self.done.get(("tempty", b), 0) != phase and self.releases == 2 * self.warps:
                raise ProtocolError(f"a release for phase {phase} of tempty[{b}] in another")
            self.count[b] = self.count.get(b, 0) + 1
            if self.count[b] % self.releases == 0:
                self.done[("tempty", b)] = self.done.get(("tempty", b), 0) + 1
            self.warp_turn[(r, w)] = t + 1

    def run(self):
        for _ in range(10 ** 6):
            finished = self.turn == len(self.turns) and not self.landing and not self.commits
            if finished and all(t == len(self.turns) for t in self.warp_turn.values()):
                return True
            moves = self.moves()
            if not moves:
                raise ProtocolError("deadlock")
            self.do(self.rnd.choice(moves))
        raise ProtocolError("no end")


@pytest.mark.parametrize("form", ["plain", "runs", "both"])
@pytest.mark.parametrize("items,stages", [([1], 6), ([2, 2, 2], 6), ([22] * 5, 6), ([3] * 7, 4), ([16, 1, 5, 4, 64], 7), ([1] * 9, 2), ([7, 8, 9], 16)])
def test_random_interleavings(form, items, stages):
    for seed in range(30):
        assert Model(form, items, stages, seed).run()


def _caught(**wrong):
    n = 0
    for seed in range(60):
        try:
            Model(seed=seed, **wrong).run()
        except ProtocolError:
            n += 1
    return n


def test_the_model_finds_a_single_dh_buffer():
    assert _caught(form="both", items=[4] * 6, stages=6, one_dh=True) > 0


def test_the_model_finds_a_release_by_half_of_the_warps():
    assert _caught(form="runs", items=[9, 9, 9], stages=6, releases=4) > 0
