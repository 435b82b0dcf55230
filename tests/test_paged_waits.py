"""What the paged prompt's bounded waits decide (csrc/glide_waits.h), tried on the host."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_24788_b200", "csrc")
SHIM = r"""
#include "glide_waits.h"
extern "C" int wait_while_moving(int (*landed)(), int (*gave_up)(), uint32_t (*moves)(), int limit) {
  return glide::wait_while_moving([&] { return landed() != 0; }, [&] { return gave_up() != 0; }, moves, limit);
}
extern "C" void wait_for_copies(int q0, int q1, int tiles, int tails, int untrimmed, int stages, void (*wait)(int, int, int)) {
  glide::AskedCopies asked;
  asked.q[0] = q0, asked.q[1] = q1, asked.tiles = tiles, asked.tails = tails, asked.untrimmed = untrimmed;
  glide::wait_for_copies(asked, stages, [&](int what, int which, uint32_t parity) { wait(what, which, int(parity)); });
}
"""


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    folder = tmp_path_factory.mktemp("waits")
    (folder / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(folder / "shim.cpp"), "-o", str(folder / "shim.so")], check=True)
    return ctypes.CDLL(str(folder / "shim.so"))


def waited(shim, lands_at, moves_until, gives_up_at=1 << 30, limit=16):
    """Tries until it came back, and with what; the work moves once per try until moves_until, the barrier lands at try lands_at."""
    tries = 0

    def landed():
        nonlocal tries
        tries += 1
        return tries >= lands_at

    num = ctypes.CFUNCTYPE(ctypes.c_int)
    got = shim.wait_while_moving(num(landed), num(lambda: tries >= gives_up_at), ctypes.CFUNCTYPE(ctypes.c_uint32)(lambda: min(tries, moves_until)), limit)
    return bool(got), tries


def test_a_wait_lasts_as_long_as_the_work_moves(shim):
    """Rows that are computed once more may take longer than any limit: a million slots by one warp took more than sixteen tries."""
    assert waited(shim, 1, 0) == (True, 1)
    assert waited(shim, 16, 0) == (True, 16)
    assert waited(shim, 500, 500) == (True, 500)
    assert waited(shim, 110, 100) == (True, 110)


def test_a_wait_for_work_that_stands_still_ends(shim):
    got, tries = waited(shim, 1 << 30, 0)
    assert not got and tries == 16
    got, tries = waited(shim, 1 << 30, 100)
    assert not got and 100 <= tries <= 117
    got, tries = waited(shim, 1 << 30, 1 << 30, gives_up_at=7)
    assert not got and tries <= 8


class Barrier:
    """Phases that have been begun and completed; a wait for a parity comes back at once unless the phase that is open has it."""

    def __init__(self):
        self.begun = self.completed = 0

    def wait(self, parity):
        if self.completed & 1 != parity:
            return
        assert self.begun > self.completed, "a wait for a phase that no copy ends: it runs to its limit"
        self.completed += 1


@pytest.mark.parametrize("stages", [5, 8])
def test_no_copy_outlives_a_loader_that_gives_up(shim, stages):
    """The loader stops anywhere, with any of the copies under way that can be: it waits for each of them, and for nothing else."""
    rng = random.Random(stages)
    for _ in range(3000):
        q, ring, tail = [Barrier(), Barrier()], [Barrier() for _ in range(stages)], Barrier()
        n = [rng.randrange(4), rng.randrange(4)]
        for x in range(2):
            q[x].begun, q[x].completed = n[x], max(0, n[x] - rng.randrange(2))
        tiles, tails, untrimmed = rng.randrange(4 * stages), 0, -1
        for t in range(tiles):
            last = t == tiles - 1
            landed = t < tiles - stages or rng.random() < 0.5   # (a buffer is filled again only when it has been read)
            if t % 2 and rng.random() < 0.3:                    # V that has to be trimmed: the loader waits for it before it goes on
                tails += 1
                tail.begun += 1
                if not last or rng.random() < 0.5:
                    tail.completed += 1
                    ring[t % stages].begun += 1
                    ring[t % stages].completed += 1
                else:
                    untrimmed = t
                    tail.completed += rng.randrange(2)
            else:
                ring[t % stages].begun += 1
                ring[t % stages].completed += landed
        wait = ctypes.CFUNCTYPE(None, ctypes.c_int, ctypes.c_int, ctypes.c_int)
        errors = []

        def one(what, which, parity):
            try:
                (q if what == 0 else ring if what == 1 else [tail])[which].wait(parity)
            except AssertionError as e:
                errors.append(e)

        shim.wait_for_copies(n[0], n[1], tiles, tails, untrimmed, stages, wait(one))
        assert not errors, errors
        assert all(b.begun == b.completed for b in q + ring + [tail]), "a copy under way that nobody has waited for"
