"""The clusters of few-token scored routing, as a model on the CPU: eight CTAs that begin in any order and run at any pace, the order of their
barriers and remote stores read from the kernel's source. No store reaches a leader that has not begun, and the leader reads
the logits when all of them are there."""
import os
import random
import re

import pytest

from paper_2609_34077_gb300 import build

CTAS = 8


def steps():
    """The kernel's cluster operations in the order of the source."""
    with open(os.path.join(build.CSRC, "route_scored.cu")) as f:
        src = f.read()
    body = src[src.index("route_scored_few_kernel(const __grid_constant__ ScoredArgs a) {"):]
    body = body[:body.index("\n}\n")]
    found = re.findall(r"\b(cluster_arrive|cluster_wait|cluster_barrier|store_leader|rank_scored_warp)\b", body)
    out = []
    for s in found:
        out += ["cluster_arrive", "cluster_wait"] if s == "cluster_barrier" else [s]
    return out


def run(order, seed):
    rng = random.Random(seed)
    started, arrived, stored = set(), [0] * CTAS, set()

    def cta(r):
        started.add(r)
        yield
        for s in order:
            if s == "cluster_arrive":
                arrived[r] += 1
            elif s == "cluster_wait":
                while min(arrived) < arrived[r]:
                    yield
            elif s == "store_leader":
                assert 0 in started, "a store to a leader that has not begun"
                stored.add(r)
            elif r == 0:
                assert len(stored) == CTAS, "the leader ranks before all logits are there"
            else:
                return  # (only the leader ranks)
            yield

    live = [cta(r) for r in range(CTAS)]
    for _ in range(5000):
        if not live:
            return
        c = rng.choice(live)
        try:
            next(c)
        except StopIteration:
            live.remove(c)
    raise AssertionError("the cluster has stopped")


def test_every_order():
    order = steps()
    assert order.count("store_leader") == 1 and order[-1] == "rank_scored_warp"
    for seed in range(300):
        run(order, seed)


@pytest.mark.parametrize("order,why", [
    (["store_leader", "cluster_arrive", "cluster_wait", "rank_scored_warp"], "has not begun"),
    (["cluster_arrive", "cluster_wait", "store_leader", "rank_scored_warp"], "before all logits")])
def test_a_missing_barrier_is_seen(order, why):
    """The model's own check."""
    with pytest.raises(AssertionError, match=why):
        for seed in range(300):
            run(order, seed)
