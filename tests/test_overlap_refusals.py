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


def test_a_page_set_s_own_arrays(lla):
    so, seqs = lla.library(), FAKE + 0x40000
    free = lambda **kw: so.lla_pages_free(ctypes.byref(pages(lla, **kw)), seqs, 2, None)
    for bad in over(TABLE, TABLE_BYTES, REF_BYTES, 16):
        assert free(ref_count=bad) == INVALID, hex(bad)
    for at, size in ARRAYS[:2]:
        for bad in over(at, size, LENS_BYTES):
            assert free(context_lens=bad) == INVALID, hex(bad)


def test_free(lla):
    so = lla.library()
    for at, size in ARRAYS:
        for bad in over(at, size, 8):
            assert so.lla_pages_free(ctypes.byref(pages(lla)), bad, 2, None) == INVALID, hex(bad)


def test_fork(lla):
    so = lla.library()
    table, lens, parents = FAKE + 0x40000, FAKE + 0x50000, FAKE + 0x60000

    def fork(parents=parents, **kw):
        to = pages(lla, **{**dict(block_table=table, context_lens=lens), **kw})
        return so.lla_pages_fork(ctypes.byref(pages(lla)), ctypes.byref(to), parents, None)

    for at, size in ARRAYS:  # what `from` and the ledger have
        for bad in over(at, size, TABLE_BYTES):
            assert fork(block_table=bad) == INVALID, hex(bad)
        for bad in over(at, size, LENS_BYTES):
            assert fork(context_lens=bad) == INVALID, hex(bad)
    for at, size in ((REF, REF_BYTES), (table, TABLE_BYTES), (lens, LENS_BYTES)):  # what is written
        for bad in over(at, size, 16):
            assert fork(parents=bad) == INVALID, hex(bad)


def test_extend(lla):
    so, need = lla.library(), ctypes.c_size_t()
    assert so.lla_pages_extend_workspace_size(4, ctypes.byref(need)) == OK
    names = ["slots", "cu", "skip", "before", "free", "ws"]
    place = {n: FAKE + 0x40000 + i * 0x10000 for i, n in enumerate(names)}
    size = dict(slots=24 * 8, cu=5 * 4, skip=4, before=16, free=4, ws=need.value)
    align = dict(slots=8, cu=4, skip=1, before=4, free=4, ws=16)

    def extend(**kw):
        a = {**place, **kw}
        return so.lla_pages_extend(ctypes.byref(pages(lla)), None, 0, a["slots"], 24, a["cu"], a["skip"], a["before"], a["free"], a["ws"], need.value, None)

    for n in names:
        for at, bytes_ in ARRAYS + [(place[m], size[m]) for m in names if m != n and {n, m} != {"cu", "skip"}]:
            for bad in over(at, bytes_, size[n], align[n]):
                assert extend(**{n: bad}) == INVALID, (n, hex(bad))
    for at, bytes_ in ARRAYS[:1] + [(place["cu"], 4)]:  # no sequence: the slots are still written
        for bad in over(at, bytes_, size["slots"], 8):
            assert so.lla_pages_extend(ctypes.byref(pages(lla, S=0)), None, 0, bad, 24, place["cu"], None, None, None, None, 0, None) == INVALID


def test_select(lla):
    so, need = lla.library(), ctypes.c_size_t()
    B, W, V, K = 2, 4, 100, 8
    assert so.lla_beam_select_workspace_size(B, W, V, K, 0, ctypes.byref(need)) == OK
    ins = dict(s=4 * B * W, fin=B * W, n=4 * B * W)
    outs = dict(parents=4 * B * K, tokens=4 * B * K, scores=4 * B * K, ended=B * K, lens=4 * B * K, ws=need.value)
    size = {**ins, **outs}
    place = {n: FAKE + 0x40000 + i * 0x10000 for i, n in enumerate(size)}
    align = {n: 1 if n in ("fin", "ended") else 16 if n == "ws" else 4 for n in size}

    def select(ws_bytes=need.value, **kw):
        a = {**place, **kw}
        return so.lla_beam_select(B, W, V, K, FAKE, V, 0, a["s"], a["fin"], a["n"], -1, 0.0, a["parents"], a["tokens"], a["scores"], a["ended"], a["lens"],
                                  a["ws"], ws_bytes, None)

    for n in outs:
        for m in size:
            if m != n:
                for bad in over(place[m], size[m], size[n], align[n]):
                    assert select(**{n: bad}) == INVALID, (n, m, hex(bad))
    # beside each other is no overlap: the next check is the workspace's size
    beside = dict(parents=place["s"] + size["s"], tokens=place["s"] - size["tokens"], ended=place["fin"] + size["fin"], lens=place["n"] - size["lens"])
    assert select(ws_bytes=need.value - 1, **beside) == WORKSPACE
