"""What the first CTA of a pair may know when it issues MMAs on both CTAs' stages, as a model on the CPU: bytes that a copy has brought in are
known to whoever waits for the copy's barrier, and to others only by an arrival that releases them. Whether the
second CTA's announcement does is read from the kernel's source."""
import os
import random
import re

import pytest

from paper_2609_34077_gb300 import build


def announcement_releases():
    with open(os.path.join(build.CSRC, "mx4_gemm.cu")) as f:
        src = f.read()
    loop = src[src.index("the leader's MMAs read this CTA's stages too"):]
    name = re.search(r"(\w+)\(peer_addr\(&ctl->full\[s\], 0\)\)", loop[:loop.index("mbar_wait_drain_cl")]).group(1)
    body = src[src.index(f"void {name}(uint32_t cluster_addr)"):]
    body = body[:body.index("\n}\n")]
    before, arrive = body.split("mbarrier.arrive", 1)
    return arrive.startswith(".release.cluster") or re.search(r"fence\.(release\.sync_restrict::shared::cta|acq_rel)\.cluster", before) is not None


def run(releases, seed, stages=4, blocks=40):
    rng = random.Random(seed)
    landed = [[-1] * stages, [-1] * stages]           # the block in each CTA's stage
    known = [[set() for _ in range(blocks)] for _ in (0, 1)]  # of each use of a `full` barrier: what waiting for it tells
    count = [[0] * blocks, [0] * blocks]              # arrivals there
    freed = [0]                                       # blocks whose MMAs have completed

    def copies(r):
        for n in range(blocks):
            while n >= freed[0] + stages:
                yield
            landed[r][n % stages] = n
            known[r][n].add((r, n))  # (a copy's completion releases the bytes it wrote)
            count[r][n] += 1
            yield

    def announcer():
        view = set()
        for n in range(blocks):
            while not count[1][n]:
                yield
            view |= known[1][n]
            if releases:
                known[0][n] |= view
            count[0][n] += 1
            yield

    def mma():
        view = set()
        for n in range(blocks):
            while count[0][n] < 2:
                yield
            view |= known[0][n]
            for r in (0, 1):
                assert landed[r][n % stages] == n
                assert (r, n) in view, "bytes that the issuing thread does not know of"
            freed[0] = n + 1
            yield

    live = [copies(0), copies(1), announcer(), mma()]
    for _ in range(200 * blocks):
        if not live:
            return
        a = rng.choice(live)
        try:
            next(a)
        except StopIteration:
            live.remove(a)
    raise AssertionError("the pair has stopped")


def test_the_kernel():
    releases = announcement_releases()
    for seed in range(20):
        run(releases, seed)


def test_a_relaxed_announcement_is_seen():
    """The model's own check."""
    with pytest.raises(AssertionError, match="does not know"):
        run(False, 0)
