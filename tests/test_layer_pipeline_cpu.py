"""The barriers of the matrices' gradient by pairs of blocks (layer_product.cu), as a model that is run under the worst orders of
its roles: a wait that the others do not hold back would run out on the GPU only now and then, and leaves meaningless outputs.

Every role is a generator that yields the condition it waits for; a scheduler advances, among the roles that can go on, always the
first of a given order, so that the last of it is as late as the barriers let it be."""
import itertools
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_04480_b200", "csrc")
STAGES, STEP = 6, 64


class Barrier:
    """Arrivals of a phase, and phases complete.  A wait tells phases by their parity alone."""
    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def passed(self, parity):
        return self.done & 1 != parity


class Pair:
    """Two blocks and their ring.  `every`: the first block's cleaning warp looks at every step's copies, which nothing holds back
    for it, instead of waiting for those alone that it has something to do in."""
    def __init__(self, tiles, every):
        self.tiles, self.every = tiles, every                        # rows of the expert, tile by tile
        new = lambda n: [Barrier(n) for _ in range(STAGES)]
        self.full, self.clean = new(4), new(2)                       # of the first block: both blocks' announcements and copies
        self.edge, self.empty = [new(2), new(2)], [new(1), new(1)]
        self.held = [[None] * STAGES, [None] * STAGES]               # (step, what its rows past the end hold)
        self.flying = []                                             # copies under way
        self.products = 0

    def steps(self):
        at = 0
        for tile, rows in enumerate(self.tiles):
            for k in range((rows + STEP - 1) // STEP):
                yield at, rows - k * STEP < STEP
                at += 1

    def load(self, rank):
        for at, ragged in self.steps():
            slot = at % STAGES
            yield lambda: self.empty[rank][slot].passed((at // STAGES & 1) ^ 1)
            own = ragged and not self.every or (ragged and rank == 1)
            bar = self.edge[rank][slot] if own else self.full[slot]
            bar.arrive()
            if self.every and ragged and rank == 0:                  # the second block's copy is not counted there
                bar.arrive(), bar.arrive()
            self.flying.append((rank, at, bar))

    def copies(self):
        while True:
            yield lambda: self.flying
            rank, at, bar = self.flying.pop(0)
            self.held[rank][at % STAGES] = (at, "other rows")
            bar.arrive()

    def issue(self):
        fulls, ends = [0] * STAGES, [0] * STAGES
        for at, ragged in self.steps():
            slot = at % STAGES
            if not ragged or self.every:
                yield lambda: self.full[slot].passed(fulls[slot])
                fulls[slot] ^= 1
            if ragged:
                if not self.every:
                    yield lambda: self.edge[0][slot].passed(ends[slot])
                yield lambda: self.clean[slot].passed(ends[slot])
                ends[slot] ^= 1
            for rank in (0, 1):
                assert self.held[rank][slot] == (at, "zeros" if ragged else "other rows")
            self.products += 1
            for rank in (0, 1):
                self.empty[rank][slot].arrive()

    def cleaner(self, rank):
        ends = [0] * STAGES
        for at, ragged in self.steps():
            slot = at % STAGES
            if self.every and rank == 0:
                yield lambda: self.full[slot].passed(at // STAGES & 1)
            elif ragged:
                yield lambda: self.edge[rank][slot].passed(ends[slot])
                ends[slot] ^= 1
            if ragged:
                assert self.held[rank][slot] == (at, "other rows")
                self.held[rank][slot] = (at, "zeros")
                self.clean[slot].arrive()

    def run(self, order):
        """Whether every role but the copies comes to its end."""
        roles = {"load 0": self.load(0), "load 1": self.load(1), "copies": self.copies(), "issue": self.issue(),
                 "clean 0": self.cleaner(0), "clean 1": self.cleaner(1)}
        waits = {name: next(role, None) for name, role in roles.items()}
        while True:
            ready = next((n for n in order(sorted(waits)) if waits[n] is not None and waits[n]()), None)
            if ready is None:
                return all(w is None for n, w in waits.items() if n != "copies")
            waits[ready] = next(roles[ready], None)


TILES = [[64] * 40, [1000, 1000, 1000], [1, 64, 130, 640, 63, 1, 900, 64 * 13, 2], [64 * 12 + 5] * 4, [33] * 20, [64 * 30, 17], []]


@pytest.mark.parametrize("tiles", TILES, ids=str)
def test_a_pair_comes_to_its_end_however_late_a_role_is(tiles):
    names = ["load 0", "load 1", "copies", "issue", "clean 0", "clean 1"]
    for order in itertools.permutations(names):
        pair = Pair(tiles, every=False)
        assert pair.run(lambda _: order), order
        assert pair.products == sum((r + STEP - 1) // STEP for r in tiles)
    for seed in range(50):
        rng = random.Random(seed)
        assert Pair(tiles, every=False).run(lambda ns: rng.sample(ns, len(ns)))


def test_the_model_notices_a_wait_that_is_not_held_back():
    """With the first block's cleaning warp looking at every step it is left behind, and waits for a phase that never comes."""
    late = ("load 0", "load 1", "copies", "issue", "clean 1", "clean 0")
    assert Pair([1000] * 3, every=True).run(lambda _: late[::-1])
    assert not Pair([1000] * 3, every=True).run(lambda _: late)
    assert not Pair([64] * 40, every=True).run(lambda _: late)


def test_the_cleaning_warp_waits_only_where_the_products_wait_for_it():
    text = open(os.path.join(CSRC, "layer_product.cu")).read()
    body = text[text.index("product_pair_kernel("):text.index("several SMs to the contraction")]
    roles = re.split(r"\} else if \(warp ", body)
    issue, cleaner = (next(r for r in roles if r.startswith("== " + n)) for n in ("kIssueWarp", "kCleanWarp"))
    waits = re.findall(r"^( *)(.*)bar_wait\(smem_addr\(&S\.(\w+)\[slot\]\)", cleaner, re.M)
    assert [(w[1], w[2]) for w in waits] == [("", "edge")], "one wait, in a branch of its own"
    branch = cleaner[:cleaner.index("bar_wait(")].rstrip().splitlines()[-1].strip()
    assert branch == "if (left < kStep) {"
    ragged = issue[issue.index("if (left < kStep) {"):]
    ragged = ragged[:ragged.index("} else {")]
    assert "S.edge[slot]" in ragged and "S.clean[slot]" in ragged and "S.full[slot]" not in ragged


def test_no_kernel_takes_memory_for_constant_that_the_launch_before_may_write():
    """A load through the path for constants promises that nothing writes the place while the kernel lives; kernels here start under
    the launch before theirs."""
    for name in os.listdir(CSRC):
        if name.startswith("layer_") and name.endswith((".cu", ".cuh", ".h")):
            assert not re.search(r"__ldg\(|ld\.global(\.\w+)*\.nc|__restrict__", open(os.path.join(CSRC, name)).read()), name
