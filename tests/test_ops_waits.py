"""The order of the weight gradient's waits (csrc/lc_wgrad.cu), as a model on the CPU.

A barrier's wait knows the parity of a round only: it passes whenever the number of completed phases has the other
parity than the one waited for, also when that is an earlier round's.  The model has the kernel's roles (loader,
two groups of converters, the thread that issues the products), in both CTAs of a pair, and lets them run in random
order, with copies that land in any order and products that end in theirs.  A converter that takes a place of the
ring whose copy has not landed is what must not happen.
"""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0
        if self.left == 0:
            self.done, self.left = self.done + 1, self.count

    def passes(self, parity):
        return self.done % 2 != parity


def run(places, stages, seed, after_empty):
    """One run of `stages` stages.  Returns the stages that a converter group took too early, None if nothing moved
    any more before the end.  after_empty: a group waits for its place's last products before it waits for the copy."""
    rng = random.Random(seed)
    ctas = range(2)
    full = [[Barrier(1) for _ in range(places)] for _ in ctas]
    empty = [[Barrier(1) for _ in range(places)] for _ in ctas]
    converted = [Barrier(4) for _ in range(places)]       # a stage has one group of either CTA, of two warps here
    early = []
    flying, products = [], []                             # copies on their way; products issued, in order
    holds = [[None] * places for _ in ctas]               # the stage whose copy has landed in a place

    def loader(c):
        for it in range(stages):
            if it >= places:
                yield lambda it=it: empty[c][it % places].passes((it // places & 1) ^ 1)
            flying.append((c, it))
            yield lambda: True

    def converters(c, group, warp):
        for it in range(group, stages, 2):
            at, parity = it % places, it // places & 1
            if after_empty and it >= places:
                yield lambda at=at, parity=parity: empty[c][at].passes(parity ^ 1)
            yield lambda at=at, parity=parity: full[c][at].passes(parity)
            if holds[c][at] != it:
                early.append((c, it))
                return
            converted[at].arrive()
            yield lambda: True

    def issuer():
        for it in range(stages):
            yield lambda it=it: converted[it % places].passes(it // places & 1)
            products.append(it)
            yield lambda: True

    roles = [loader(c) for c in ctas] + [converters(c, g, w) for c in ctas for g in range(2) for w in range(2)] + [issuer()]
    waits = [(r, next(r)) for r in roles]
    while waits and not early:
        moves = [("role", i) for i, (_, ready) in enumerate(waits) if ready()]
        moves += [("land", i) for i in range(len(flying))]
        if products:
            moves.append(("product", 0))
        if not moves:
            return None
        kind, i = rng.choice(moves)
        if kind == "land":
            c, it = flying.pop(i)
            holds[c][it % places] = it
            full[c][it % places].arrive()
        elif kind == "product":
            it = products.pop(0)
            for c in ctas:
                empty[c][it % places].arrive()
        else:
            role, _ = waits[i]
            try:
                waits[i] = (role, next(role))
            except StopIteration:
                del waits[i]
    return early


@pytest.mark.parametrize("places", [3, 5])
def test_converters_wait_for_their_own_round(places):
    for seed in range(400):
        assert run(places, 40, seed, after_empty=True) == []


@pytest.mark.parametrize("places", [3, 5])
def test_the_parity_alone_lets_an_earlier_round_pass(places):
    """What the first wait is for: an odd ring gives a place to either group in turn."""
    assert any(run(places, 40, seed, after_empty=False) for seed in range(400))


def test_an_even_ring_would_not_need_it():
    for seed in range(400):
        assert run(4, 40, seed, after_empty=False) == []
