"""Arrays of a page or beam call that overlap where one is written are refused before anything is enqueued (no GPU)."""
import ctypes

import pytest

from helpers import ensure_library

OK, INVALID, UNSUPPORTED, CUDA_ERR, TIMEOUT, DEVCHECK, WORKSPACE = range(7)
FAKE = 0x10000  # a non-NULL, 16-byte aligned "device pointer" that validation never touches
BIG = 1 << 30


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


# One page set: 100 counts, a table of 4 rows of 8, 4 lengths, each in a place of its own.
REF, TABLE, LENS = FAKE, FAKE + 0x10000, FAKE + 0x20000
REF_BYTES, TABLE_BYTES, LENS_BYTES = 400, 128, 16
ARRAYS = [(REF, REF_BYTES), (TABLE, TABLE_BYTES), (LENS, LENS_BYTES)]


def pages(lla, **kw):
    p = lla.lla_pages(REF, 100, TABLE, 8, LENS, 4)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def over(at, size, width, align=4):
    """The first and the last places where an array of `width` bytes overlaps [at, at + size)."""
    last = (at + size - 1) // align * align
    return sorted({-(-(at - width + 1) // align) * align, at, last})


def test_compact(lla):
    need = ctypes.c_size_t()
    assert lla.library().lla_pages_compact_workspace_size(100, ctypes.byref(need)) == OK
    remap, live, ws = FAKE + 0x40000, FAKE + 0x50000, FAKE + 0x60000

    def compact(remap=remap, live=live, ws=ws, ws_bytes=BIG):
        return lla.library().lla_pages_compact(ctypes.byref(pages(lla)), None, 0, remap, live, ws, ws_bytes, None)

    for at, size in ARRAYS:
        for bad in over(at, size, 400):
            assert compact(remap=bad) == INVALID, hex(bad)
        for bad in over(at, size, 4):
            assert compact(live=bad) == INVALID, hex(bad)
        for bad in over(at, size, need.value, 16):
            assert compact(ws=bad) == INVALID, hex(bad)
        for good in (at + size, at - 4):  # beside it: the next check is the workspace's size
            assert compact(live=good, ws_bytes=need.value - 1) == WORKSPACE
    for at, size in ((remap, 400), (live, 4)):
        for bad in over(at, size, need.value, 16):
            assert compact(ws=bad) == INVALID, hex(bad)
    for bad in over(remap, 400, 4):
        assert compact(live=bad) == INVALID
