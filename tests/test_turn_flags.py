"""The flags that the waves of a latent attention raise and look at, on the CPU: the kernel's own header under a
model of its turns, waves running ahead of one another as far as the barriers let them."""
import ctypes
import random
import subprocess

import pytest

from paper_2605_24793_amd import _build

SOURCE = """
#include "turn_flags.h"
static cospec::TurnFlags flags;
extern "C" void start() { flags.lower_all(); }
extern "C" int raised(int turn) { return flags.raised(turn); }
extern "C" void raise_flag(int turn) { flags.raise(turn); }
extern "C" void lower(int turn) { flags.lower(turn); }
"""
WAVES = 8                                                   # the first four find scores, the others sum


@pytest.fixture(scope="module")
def flags(tmp_path_factory):
    folder = tmp_path_factory.mktemp("flags")
    source, lib = folder / "flags.cpp", folder / "flags.so"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", _build.CSRC, "-o", str(lib), str(source)],
                   check=True)
    return ctypes.CDLL(str(lib))


def _wave(w, flags, segments, raises, met):
    """One wave: yields at every barrier, and before every access to the flags."""
    for s, turns in enumerate(segments):
        yield "barrier"                                     # the segment's pages
        for i in range(turns + 1):
            yield "barrier"
            yield "step"
            if flags.raised(i - 1):
                met[w].append((s, i - 1))
                yield "barrier"
                if w == 0:
                    yield "step"
                    flags.lower(i - 1)
                yield "barrier"
            if w < 4 and i < turns and w in raises.get((s, i), ()):
                yield "step"
                flags.raise_flag(i)


def _run(flags, segments, raises, next_wave):
    """next_wave(those not at a barrier): which one goes on.  Returns the flags that each wave met."""
    flags.start()
    met = [[] for _ in range(WAVES)]
    waves = [_wave(w, flags, segments, raises, met) for w in range(WAVES)]
    at_barrier, ended = set(), set()
    while len(ended) < WAVES:
        free = [w for w in range(WAVES) if w not in at_barrier and w not in ended]
        if not free:
            # a wave at a barrier that another one never reaches would wait for ever
            assert not ended, "waves met different barriers"
            at_barrier.clear()
            continue
        w = next_wave(free)
        try:
            if next(waves[w]) == "barrier":
                at_barrier.add(w)
        except StopIteration:
            ended.add(w)
    return met


@pytest.mark.parametrize("order", ["first wave first", "last wave first", "scores ahead", "sums ahead", "random"])
def test_every_wave_meets_the_flags_that_were_raised(flags, order):
    rng = random.Random(order)
    for trial in range(60):
        segments = [rng.randint(1, 9) for _ in range(rng.randint(1, 3))]
        often = (0.1, 0.5, 1.0)[trial % 3]
        raises = {}
        for s, turns in enumerate(segments):
            for i in range(turns):
                if rng.random() < often:
                    raises[s, i] = {w for w in range(4) if rng.random() < 0.6} or {rng.randrange(4)}
        pick = {"first wave first": min, "last wave first": max,
                "scores ahead": lambda free: rng.choice([w for w in free if w < 4] or free),
                "sums ahead": lambda free: rng.choice([w for w in free if w >= 4] or free), "random": rng.choice}[order]
        for met in _run(flags, segments, raises, pick):
            assert met == sorted(raises), (segments, raises)
