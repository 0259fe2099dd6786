"""Host-side checks of the page and beam calls (no GPU): bad arguments are refused before anything is enqueued, the sizes
and descriptions that need no device, and arguments that the native marshalling leaves to Python."""
import ctypes

import pytest
import torch

from helpers import ensure_library

OK, INVALID, UNSUPPORTED, CUDA_ERR, TIMEOUT, DEVCHECK, WORKSPACE = range(7)
FAKE = 0x10000  # a non-NULL, 16-byte aligned "device pointer" that validation never touches
BIG = 1 << 30


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


def pages(lla, at=FAKE, **kw):
    p = lla.lla_pages(FAKE, 100, at + 0x100000, 8, at + 0x200000, 4)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def pool(lla, **kw):
    p = lla.lla_pool(FAKE, 4, 192, 320)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_PAGES = [(dict(ref_count=None), INVALID), (dict(ref_count=FAKE + 4), INVALID), (dict(num_blocks=0), INVALID), (dict(block_table=None), INVALID),
             (dict(context_lens=None), INVALID), (dict(max_blocks_per_seq=0), INVALID), (dict(S=-1), INVALID), (dict(S=1025), INVALID),
             (dict(num_blocks=(1 << 24) + 1), UNSUPPORTED), (dict(max_blocks_per_seq=(1 << 24) + 1), UNSUPPORTED)]
BAD_POOLS = [dict(base=None), dict(base=FAKE + 8), dict(pages=0), dict(pages=4097), dict(k_row_bytes=0), dict(k_row_bytes=6), dict(k_row_bytes=8196),
             dict(v_row_bytes=-4), dict(v_row_bytes=2), dict(v_row_bytes=8196)]


def test_pools_of_the_caches(lla):
    so, out = lla.library(), lla.lla_pool()
    g = lla.Geometry(4, 16, 128, 96, 160).c()
    assert so.lla_cache_pool(ctypes.byref(g), FAKE, ctypes.byref(out)) == OK
    assert (out.base, out.pages, out.k_row_bytes, out.v_row_bytes) == (FAKE, 16, 192, 320)
    assert so.lla_cache_2d_pool(ctypes.byref(g), FAKE, ctypes.byref(out)) == OK
    assert (out.pages, out.k_row_bytes, out.v_row_bytes) == (1, 192, 320)
    wide = lla.Geometry(4, 16, 128, 1152, 1920).c()
    assert so.lla_cache_pool(ctypes.byref(wide), FAKE, ctypes.byref(out)) == INVALID
    assert so.lla_cache_2d_pool(ctypes.byref(wide), FAKE, ctypes.byref(out)) == OK
    assert so.lla_rope_pool(64, FAKE, ctypes.byref(out)) == OK
    assert (out.pages, out.k_row_bytes, out.v_row_bytes) == (1, 128, 0)
    assert so.lla_rope_pool(20, FAKE, ctypes.byref(out)) == INVALID
    for fn, first in ((so.lla_cache_pool, ctypes.byref(g)), (so.lla_cache_2d_pool, ctypes.byref(g)), (so.lla_rope_pool, 64)):
        assert fn(first, None, ctypes.byref(out)) == INVALID
        assert fn(first, FAKE + 8, ctypes.byref(out)) == INVALID
        assert fn(first, FAKE, None) == INVALID
    assert so.lla_cache_pool(None, FAKE, ctypes.byref(out)) == INVALID


def test_fork_checks(lla):
    def fork(a=None, b=None, parents=FAKE + 0x900000):
        a = a or pages(lla)
        b = b or pages(lla, FAKE + 0x400000)
        return lla.library().lla_pages_fork(ctypes.byref(a), ctypes.byref(b), parents, None)

    for bad, status in BAD_PAGES:
        assert fork(a=pages(lla, **bad)) == status, bad
        assert fork(b=pages(lla, FAKE + 0x400000, **bad)) == status, bad
    assert fork(parents=None) == INVALID
    other = FAKE + 0x400000
    assert fork(b=pages(lla, other, ref_count=FAKE + 16)) == INVALID        # another ledger
    assert fork(b=pages(lla, other, num_blocks=99)) == INVALID
    a = pages(lla)
    assert fork(b=pages(lla)) == INVALID                                    # onto itself
    assert fork(b=pages(lla, other, block_table=a.block_table + 4 * 8 * 4 - 4)) == INVALID  # the last entry
    assert fork(b=pages(lla, other, context_lens=a.context_lens - 12)) == INVALID
    assert fork(parents=other + 0x200000) == INVALID                        # the lengths it writes
    assert fork(parents=other + 0x100000 + 16) == INVALID                   # the table it writes
    assert lla.library().lla_pages_fork(None, ctypes.byref(a), FAKE, None) == INVALID
    none = dict(S=0, block_table=None, context_lens=None)
    assert fork(a=pages(lla, **none), b=pages(lla, other, **none), parents=None) == OK


def test_extend_checks(lla):
    so, n = lla.library(), ctypes.c_size_t()
    assert so.lla_pages_extend_workspace_size(1024, ctypes.byref(n)) == OK
    assert so.lla_pages_extend_workspace_size(1025, ctypes.byref(n)) == INVALID
    assert so.lla_pages_extend_workspace_size(-1, ctypes.byref(n)) == INVALID
    assert so.lla_pages_extend_workspace_size(4, None) == INVALID

    def extend(p=None, pools=None, L=1, slots=FAKE, N=4, cu=None, ws=FAKE, ws_bytes=BIG):
        p = p or pages(lla)
        arr = (lla.lla_pool * 1)(pools or pool(lla))
        return so.lla_pages_extend(ctypes.byref(p), arr if L else None, L, slots, N, cu, None, None, None, ws, ws_bytes, None)

    for bad, status in BAD_PAGES:
        assert extend(p=pages(lla, **bad)) == status, bad
    for bad in BAD_POOLS:
        assert extend(pools=pool(lla, **bad)) == INVALID, bad
    assert extend(L=-1) == INVALID
    assert extend(L=129) == UNSUPPORTED
    assert so.lla_pages_extend(ctypes.byref(pages(lla)), None, 1, FAKE, 4, None, None, None, None, FAKE, BIG, None) == INVALID
    assert extend(slots=None) == INVALID
    assert extend(N=-4) == INVALID
    assert extend(N=5) == INVALID                                           # no whole number of tokens a sequence
    assert extend(ws=None) == INVALID
    assert extend(ws=FAKE + 8) == INVALID
    assert extend(ws_bytes=n.value - 1) == WORKSPACE
    none = pages(lla, S=0, block_table=None, context_lens=None)
    assert extend(p=none, N=0, slots=None, ws=None) == OK
    assert extend(p=none, N=4) == INVALID


def test_free_and_compact_checks(lla):
    so, n = lla.library(), ctypes.c_size_t()

    def free(p=None, seqs=FAKE, k=2):
        return so.lla_pages_free(ctypes.byref(p or pages(lla)), seqs, k, None)

    for bad, status in BAD_PAGES:
        assert free(pages(lla, **bad)) == status, bad
    assert free(seqs=None) == INVALID
    assert free(k=-1) == INVALID
    assert free(k=1025) == INVALID
    assert free(seqs=None, k=0) == OK
    assert so.lla_pages_compact_workspace_size(100, ctypes.byref(n)) == OK
    need = n.value
    assert so.lla_pages_compact_workspace_size(0, ctypes.byref(n)) == INVALID
    assert so.lla_pages_compact_workspace_size((1 << 24) + 1, ctypes.byref(n)) == UNSUPPORTED
    assert so.lla_pages_compact_workspace_size(100, None) == INVALID

    def compact(p=None, pools=None, remap=FAKE + 0x800000, live=FAKE + 0x900000, ws=FAKE, ws_bytes=BIG):
        arr = (lla.lla_pool * 1)(pools or pool(lla))
        return so.lla_pages_compact(ctypes.byref(p or pages(lla)), arr, 1, remap, live, ws, ws_bytes, None)

    for bad, status in BAD_PAGES:
        assert compact(pages(lla, **bad)) == status, bad
    for bad in BAD_POOLS:
        assert compact(pools=pool(lla, **bad)) == INVALID, bad
    assert compact(remap=None) == INVALID
    assert compact(remap=FAKE + 4 * 99) == INVALID                          # the last count
    assert compact(remap=FAKE + 0x100000 - 4) == INVALID                    # a table
    assert compact(live=FAKE) == INVALID
    assert compact(live=FAKE + 0x800000 + 4) == INVALID
    assert compact(live=None) == INVALID
    assert compact(ws=None) == INVALID
    assert compact(ws=FAKE + 4) == INVALID
    assert compact(ws_bytes=need - 1) == WORKSPACE


def test_select_checks(lla):
    so, n = lla.library(), ctypes.c_size_t()
    size = lambda B=2, W=4, V=100, K=8, dt=0, out=ctypes.byref(n): so.lla_beam_select_workspace_size(B, W, V, K, dt, out)
    assert size() == OK and n.value > 0
    need = n.value
    for bad, status in ((dict(B=-1), INVALID), (dict(W=0), INVALID), (dict(V=0), INVALID), (dict(K=0), INVALID), (dict(dt=2), INVALID), (dict(out=None), INVALID),
                        (dict(W=33), UNSUPPORTED), (dict(K=33), UNSUPPORTED), (dict(V=(1 << 24) + 1), UNSUPPORTED), (dict(B=257), INVALID)):
        assert size(**bad) == status, bad

    at = lambda i: FAKE + i * 0x1000

    def select(B=2, W=4, V=100, K=8, z=FAKE, stride=100, dt=0, s=at(1), fin=at(2), n=at(3), eos=-1, alpha=0.0, parents=at(4), tokens=at(5),
               scores=at(6), ended=at(7), lens=at(8), ws=at(9), ws_bytes=BIG):
        return so.lla_beam_select(B, W, V, K, z, stride, dt, s, fin, n, eos, alpha, parents, tokens, scores, ended, lens, ws, ws_bytes, None)

    for bad, status in ((dict(B=-1), INVALID), (dict(W=0), INVALID), (dict(V=0), INVALID), (dict(K=0), INVALID), (dict(dt=2), INVALID), (dict(B=257), INVALID),
                        (dict(W=33), UNSUPPORTED), (dict(K=33), UNSUPPORTED), (dict(stride=99), INVALID), (dict(stride=1 << 41), INVALID),
                        (dict(z=None), INVALID), (dict(z=FAKE + 1), INVALID), (dict(z=FAKE + 2, dt=1), INVALID), (dict(s=None), INVALID),
                        (dict(eos=-2), INVALID), (dict(eos=100), INVALID), (dict(alpha=17.0), INVALID), (dict(alpha=float("nan")), INVALID),
                        (dict(n=None), INVALID), (dict(n=None, lens=None, alpha=1.0), INVALID), (dict(parents=None), INVALID), (dict(tokens=None), INVALID),
                        (dict(scores=None), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 8), INVALID), (dict(ws_bytes=need - 1), WORKSPACE),
                        (dict(scores=at(1)), INVALID), (dict(scores=at(1) - 60), INVALID), (dict(lens=at(3)), INVALID), (dict(ended=at(2) + 7), INVALID),
                        (dict(parents=at(3)), INVALID)):
        assert select(**bad) == status, bad
    assert select(B=0, z=None, s=None, parents=None, tokens=None, scores=None, ws=None) == OK


def test_search_checks(lla):
    so, n = lla.library(), ctypes.c_size_t()
    assert so.lla_beam_search_workspace_size(1, 4, 100, 0, ctypes.byref(n)) == OK
    need = n.value
    assert so.lla_beam_search_workspace_size(1, 33, 100, 0, ctypes.byref(n)) == UNSUPPORTED
    assert so.lla_beam_search_workspace_size(1, 4, 100, 0, None) == INVALID
    called = []
    cb = lla.STEP_FN(lambda *a: called.append(a) or 1)

    def search(a=None, b=None, B=1, W=4, V=100, dt=0, steps=3, step=cb, tokens=FAKE, scores=FAKE, finished=FAKE, lengths=FAKE, parents=FAKE, ws=FAKE,
               ws_bytes=BIG):
        return so.lla_beam_search(ctypes.byref(a or pages(lla)), ctypes.byref(b or pages(lla, FAKE + 0x400000)), None, 0, B, W, V, dt, steps, -1, 0.0,
                                  tokens, scores, finished, lengths, parents, step, None, ws, ws_bytes, None)

    for bad, status in ((dict(W=3), INVALID), (dict(W=33), UNSUPPORTED), (dict(a=pages(lla, S=5)), INVALID), (dict(b=pages(lla, S=3)), INVALID),
                        (dict(steps=-1), INVALID), (dict(V=0), INVALID), (dict(dt=3), INVALID), (dict(step=lla.STEP_FN(0)), INVALID), (dict(tokens=None), INVALID),
                        (dict(scores=None), INVALID), (dict(finished=None), INVALID), (dict(lengths=None), INVALID), (dict(parents=None), INVALID),
                        (dict(ws=None), INVALID), (dict(ws=FAKE + 4), INVALID), (dict(ws_bytes=need - 1), WORKSPACE),
                        (dict(a=pages(lla, ref_count=None)), INVALID), (dict(b=pages(lla)), INVALID)):
        assert search(**bad) == status, bad
    assert search(steps=0) == OK
    assert not called


@pytest.mark.parametrize("name", ["pages_fork", "pages_extend", "pages_free", "pages_compact", "beam_select"])
def test_unusual_arguments_are_left_to_python(lla, name):
    native = getattr(lla._native(), name)
    count = {"pages_fork": 4, "pages_extend": 9, "pages_free": 3, "pages_compact": 6, "beam_select": 13}[name]
    t = torch.zeros(2, 2, dtype=torch.int32)
    for x in (t, FAKE, "x", None, lla.Pages(t[0], t, t[0])):
        assert native(*[x] * count) is None
    with pytest.raises(TypeError):
        native(None)


def test_host_tensors_are_refused(lla):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    p = lla.Pages(i(10), i(4, 2), i(4))
    w = torch.zeros(1 << 16, dtype=torch.uint8)
    f = torch.zeros(1, 4)
    for call in (lambda: lla.lla_pages_fork(p, p, i(4)), lambda: lla.lla_pages_extend(p, lla.Pools(), torch.zeros(4, dtype=torch.int64), w),
                 lambda: lla.lla_pages_free(p, i(1)), lambda: lla.lla_pages_compact(p, lla.Pools(), i(10), i(1), w),
                 lambda: lla.lla_beam_select(torch.zeros(1, 4, 9), f, i(1, 4), i(1, 4), f, w), lambda: lla.Pools([lla.Pool(w, 1, 16, 16)])):
        with pytest.raises(ValueError, match="CUDA tensors"):
            call()
