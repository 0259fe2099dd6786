"""Arguments of lla_beam_search that are wrong for every step are refused before the first one: nothing grows, and the model is
not called (no GPU)."""
import ctypes
import math

import pytest

from helpers import ensure_library
from test_overlap_refusals import ARRAYS, BIG, FAKE, INVALID, LENS, LENS_BYTES, REF, TABLE, TABLE_BYTES, over

B, W, V, STEPS = 1, 4, 100, 3


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


@pytest.fixture(scope="module")
def need(lla):
    n = ctypes.c_size_t()
    assert lla.library().lla_beam_search_workspace_size(B, W, V, 0, ctypes.byref(n)) == 0
    return n.value


PLACE = {n: FAKE + 0x40000 + i * 0x10000 for i, n in enumerate(["tokens", "scores", "finished", "lengths", "parents", "ws", "table", "lens"])}


def search(lla, need, L=0, pools=None, eos=-1, alpha=0.0, steps=STEPS, **kw):
    a = {**PLACE, **kw}
    called = []
    cb = lla.STEP_FN(lambda *_: called.append(1) or 1)
    first, second = lla.lla_pages(REF, 100, TABLE, 8, LENS, 4), lla.lla_pages(REF, 100, a["table"], 8, a["lens"], 4)
    st = lla.library().lla_beam_search(ctypes.byref(first), ctypes.byref(second), pools, L, B, W, V, 0, steps, eos, alpha, a["tokens"], a["scores"],
                                       a["finished"], a["lengths"], a["parents"], cb, None, a["ws"], need, None)
    assert not called
    return st


@pytest.mark.parametrize("steps", [0, STEPS])
@pytest.mark.parametrize("bad", [dict(eos=-2), dict(eos=V), dict(alpha=math.nan), dict(alpha=17.0), dict(alpha=-16.5), dict(alpha=math.inf)])
def test_options(lla, need, bad, steps):
    assert search(lla, need, steps=steps, **bad) == INVALID


def test_pools(lla, need):
    bad = (lla.lla_pool * 1)(lla.lla_pool(FAKE, 0, 192, 320))
    assert search(lla, need, L=1, pools=bad) == INVALID
    assert search(lla, need, L=1) == INVALID
    assert search(lla, need, L=-1) == INVALID
    assert search(lla, need, L=129, pools=bad) == 2  # unsupported


def test_slabs_that_overlap(lla, need):
    slab = (STEPS + 1) * B * W
    size = dict(tokens=slab * 4, scores=slab * 4, finished=slab, lengths=slab * 4, parents=STEPS * B * W * 4, ws=need)
    sets = ARRAYS + [(PLACE["table"], TABLE_BYTES), (PLACE["lens"], LENS_BYTES)]
    for n in size:
        for at, bytes_ in sets + [(PLACE[m], size[m]) for m in size if m != n]:
            for bad in over(at, bytes_, size[n], 1 if n == "finished" else 16 if n == "ws" else 4):
                assert search(lla, need, **{n: bad}) == INVALID, (n, hex(bad))
