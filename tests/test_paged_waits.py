"""What the paged prompt's bounded waits decide (csrc/glide_waits.h), tried on the host."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_24788_b200", "csrc")
SHIM = r"""
#include "glide_waits.h"
extern "C" int wait_while_moving(int (*landed)(), int (*gave_up)(), uint32_t (*moves)(), int limit) {
  return glide::wait_while_moving([&] { return landed() != 0; }, [&] { return gave_up() != 0; }, moves, limit);
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
