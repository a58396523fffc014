"""The prefix pass's ring of tiles, modelled on the CPU: two producers, two issuers that wait on fills by their parity, one
tile per item (each issuer takes every other step) or two (both take all). With any interleaving a consumer has to find the
fill that it waits for and no tile may be filled while it is read.

A parity wait cannot tell a fill from the one before the last. Where an issuer comes to stages that the other one emptied
since, it would read an old tile; hence a stage has the same issuer in all parts of one tile, and the issuers meet before
they go through the ring together. Without either the model fails, as the kernel did about once in a thousand calls."""
import random

import pytest


class Ring:
    def __init__(self, stages, parts, same_owner, meet):
        self.NS, self.parts, self.same_owner, self.meet = stages, parts, same_owner, meet
        self.full, self.empty, self.arrived = [0] * stages, [0] * stages, [0] * stages
        self.held, self.reading, self.met = [None] * stages, [0] * stages, [0, 0]
        self.copies, self.landed = [], 0

    @staticmethod
    def passed(phases, parity):
        """try_wait.parity: whether the phase of this parity is not the one under way."""
        return (phases & 1) != parity

    def producer(self, kv, r):
        for step in range(sum(n for n, _ in self.parts)):
            i = 2 * step + kv
            s = i % self.NS
            while not self.passed(self.empty[s], ((i // self.NS) & 1) ^ 1):
                yield
            assert not self.reading[s], "filled while it is read"
            self.held[s] = None
            self.copies.append((s, step, kv))
            yield

    def memory(self, r):
        """Copies land in any order."""
        while self.landed < 2 * sum(n for n, _ in self.parts):
            if self.copies:
                s, step, kv = self.copies.pop(r.randrange(len(self.copies)))
                self.held[s] = (step, kv)
                self.full[s] += 1
                self.landed += 1
            yield

    def read(self, s, step, kv, arrivals, r):
        assert self.held[s] == (step, kv), f"{self.held[s]} for {(step, kv)}"
        self.reading[s] += 1
        for _ in range(r.randint(1, 4)):
            yield
        self.reading[s] -= 1
        self.arrived[s] += arrivals
        if self.arrived[s] == 2:
            self.arrived[s] = 0
            self.empty[s] += 1

    def issuer(self, w, r):
        at, done, apart, meetings = 0, 0, False, 0  # the next tile, steps before the part
        for steps, one in self.parts:
            if one:
                apart = True
                for k in range(w ^ (done & 1) if self.same_owner else w, steps, 2):
                    for kv in (0, 1):
                        i = at + 2 * k + kv
                        while not self.passed(self.full[i % self.NS], (i // self.NS) & 1):
                            yield
                        yield from self.read(i % self.NS, done + k, kv, 2, r)
            else:
                if apart and self.meet:
                    self.met[w ^ 1] += 1
                    while not self.passed(self.met[w], meetings & 1):
                        yield
                    meetings += 1
                apart = False
                for i in range(at, at + 2 * steps):
                    while not self.passed(self.full[i % self.NS], (i // self.NS) & 1):
                        yield
                    yield from self.read(i % self.NS, done + (i - at) // 2, i & 1, 1, r)
            at += 2 * steps
            done += steps


def play(stages, seed, same_owner=True, meet=True):
    r = random.Random(seed)
    ring = Ring(stages, [(r.randint(1, 9), r.random() < 0.6) for _ in range(r.randint(1, 6))], same_owner, meet)
    roles = [ring.producer(0, r), ring.producer(1, r), ring.issuer(0, r), ring.issuer(1, r), ring.memory(r)]
    alive, pace, turns = [0, 1, 2, 3, 4], [1.0] * 5, 0
    while alive:
        if turns % 400 == 0:
            pace = [r.random() ** 3 + 0.01 for _ in roles]
        i = r.choices(alive, [pace[j] for j in alive])[0]
        try:
            next(roles[i])
        except StopIteration:
            alive.remove(i)
        turns += 1
        assert turns < 200000, "stuck"


@pytest.mark.parametrize("stages", [4, 8])
def test_every_tile_is_the_one_waited_for(stages):
    for seed in range(400):
        play(stages, seed)


@pytest.mark.parametrize("without", [dict(same_owner=False), dict(meet=False)], ids=str)
def test_the_model_finds_what_either_rule_prevents(without):
    failed = 0
    for seed in range(400):
        try:
            play(4, seed, **without)
        except AssertionError:
            failed += 1
    assert failed
