"""Rounds of posts between the blocks of a cluster whose waits may run out (peer_round.h, compiled for the
host), against a model of the blocks, their slots and barriers under random schedules.

The model.  A block's threads share the posts of a round, each to some of the blocks, into the receiver's
slot of that round; the slot's barrier completes a phase when its block's first thread has announced the
round's posts and as many have been counted.  A thread waits for that phase, or gives up, reads the slot and
meets the other threads of its block.  What a thread reads that has not given up has to be the posts of its
own round, of every block: anything else would end up in finite, wrong states."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2607_05272_gb300 import build as B

BLOCKS, THREADS, ROUNDS = 3, 2, 6


class PeerRound(ctypes.Structure):
    _fields_ = [("state", ctypes.c_uint32)]


@pytest.fixture(scope="module")
def rounds(tmp_path_factory):
    d = tmp_path_factory.mktemp("peer")
    src, out = d / "p.cpp", str(d / "p.so")
    src.write_text('#include "%s"\nusing simx::PeerRound;\nextern "C" {\n'
                   'unsigned slot(PeerRound* p) { return p->slot(); }\n'
                   'unsigned parity(PeerRound* p) { return p->parity(); }\n'
                   'bool lost(PeerRound* p) { return p->lost(); }\n'
                   'bool posts(PeerRound* p) { return p->posts(); }\n'
                   'void end(PeerRound* p, bool came) { p->end(came); }\n}\n' % os.path.join(B.CSRC, "peer_round.h"))
    subprocess.run(["g++", "-shared", "-fPIC", "-std=c++17", "-o", out, str(src)], check=True)
    lib = ctypes.CDLL(out)
    lib.posts.restype = lib.lost.restype = ctypes.c_bool
    lib.end.argtypes = [ctypes.c_void_p, ctypes.c_bool]
    return lib


class Barrier:
    def __init__(self):
        self.phases, self.arrived, self.count = 0, False, 0

    def add(self, n, arrive=False):
        self.count += n
        self.arrived |= arrive
        if self.arrived and self.count == 0:
            self.phases, self.arrived = self.phases + 1, False

    def completed(self, parity):
        return self.phases % 2 != parity


def _run(lib, rng, posts, give_up, late):
    """One schedule; the number of rounds that threads read whole, and of those with another round's posts."""
    slots = [[[None] * BLOCKS for _ in range(2)] for _ in range(BLOCKS)]
    bars = [[Barrier(), Barrier()] for _ in range(BLOCKS)]
    met = [0] * BLOCKS
    whole = wrong = 0

    def thread(b, q):
        nonlocal whole, wrong
        p = PeerRound(0)
        r = ctypes.byref(p)
        for turn in range(ROUNDS):
            slot, parity = lib.slot(r), lib.parity(r)
            bar = bars[b][slot]
            if posts(r):
                if q == 0:
                    bar.add(BLOCKS, arrive=True)
                yield
                for to in range(q, BLOCKS, THREADS):
                    slots[to][slot][b] = turn
                    bars[to][slot].add(-1)
                    yield
            came = False
            while not lib.lost(r) and not came:
                came = bar.completed(parity)
                if not came:
                    if rng.random() < give_up:
                        break
                    yield
            lib.end(r, came)
            yield
            if not lib.lost(r):
                whole += 1
                wrong += any(v != turn for v in slots[b][slot])
            met[b] += 1
            while met[b] < THREADS * (turn + 1):
                yield

    live = [(b, thread(b, q)) for b in range(BLOCKS) for q in range(THREADS)]
    while live:
        weights = [late if b == 0 else 1.0 for b, _ in live]  # block 0 is slow
        k = rng.choices(range(len(live)), weights)[0]
        try:
            next(live[k][1])
        except StopIteration:
            del live[k]
    return whole, wrong


def test_without_giving_up_every_round_is_whole(rounds):
    rng = random.Random(1)
    for _ in range(200):
        assert _run(rounds, rng, rounds.posts, 0.0, 0.1) == (BLOCKS * THREADS * ROUNDS, 0)


def test_no_thread_takes_another_rounds_posts(rounds):
    rng = random.Random(2)
    total = 0
    for _ in range(3000):
        whole, wrong = _run(rounds, rng, rounds.posts, rng.choice([0.02, 0.1, 0.5]), rng.choice([0.02, 0.1, 1.0]))
        assert wrong == 0
        total += whole
    assert 0 < total < 3000 * BLOCKS * THREADS * ROUNDS  # waits ran out, and not all of them


def test_the_model_sees_posts_after_giving_up(rounds):
    """The mistake planted in the model: threads that gave up go on posting."""
    rng = random.Random(3)
    assert sum(_run(rounds, rng, lambda r: True, 0.1, 0.05)[1] for _ in range(500)) > 0
