"""The order in which results pass through a warp's buffers (no GPU needed): the kernel's own header, compiled for the host."""
import ctypes
import itertools
import os
import shutil
import subprocess

import pytest

from tests.test_kernel_sources import CSRC

SHIM = """
#include "result_slots.cuh"
static svl::ResultSlots s;
extern "C" {
void start() { s = svl::ResultSlots(); }
void enter_last(int residual) { s.enter_last(residual != 0); }
int slot() { return s.slot; }
int unread() { return s.unread(); }
void stored() { s.stored(); }
}
"""


@pytest.fixture(scope="module")
def slots(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    at = tmp_path_factory.mktemp("slots")
    (at / "shim.cpp").write_text(SHIM)
    out = str(at / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, str(at / "shim.cpp"), "-o", out],
                   check=True)
    return ctypes.CDLL(out)


# chunks of a warp in each of a CTA's tiles (none where its rows or columns do not exist)
TILES = [t for n in (1, 2, 3, 4) for t in itertools.product((0, 1, 2, 3, 4), repeat=n)]


def test_no_chunk_is_written_while_a_store_may_read_its_buffer(slots):
    for tiles in TILES:
        slots.start()
        stores = []  # buffers, in the order of the stores
        for i, chunks in enumerate(tiles):
            if i == len(tiles) - 1:
                slots.enter_last(0)
            for _ in range(chunks):
                unread = slots.unread()
                assert slots.slot() not in stores[max(0, len(stores) - unread):], (tiles, stores)
                assert slots.slot() == 0 or i == len(tiles) - 1, tiles  # the stages are still in use
                stores.append(slots.slot())
                slots.stored()


def test_the_second_buffer_is_used(slots):
    """Two chunks of the last tile lie in different buffers."""
    for residual in (0, 1):
        slots.start()
        slots.enter_last(residual)
        seen = []
        for _ in range(4):
            seen.append(slots.slot())
            slots.stored()
        assert seen == ([0, 1, 0, 1] if residual else [1, 0, 1, 0])


def test_a_residual_is_read_from_the_buffer_it_was_requested_for(slots):
    """Requests go to buffer 0 at the start, to buffer 1 when the last tile begins, and to a chunk's own buffer behind it."""
    for tiles in TILES:
        slots.start()
        left = sum(tiles)
        asked = []

        def request(b):
            nonlocal left
            if left > 0:
                left -= 1
                asked.append(b)
        request(0)
        for i, chunks in enumerate(tiles):
            if i == len(tiles) - 1:
                slots.enter_last(1)
                request(1)
            for _ in range(chunks):
                assert asked.pop(0) == slots.slot(), tiles
                request(slots.slot())
                slots.stored()
        assert not asked and not left
