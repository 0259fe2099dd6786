"""Host-side checks of the calls for shared prefixes, admission and rotary axes (no GPU): bad arguments are refused before
anything is enqueued."""
import ctypes

import pytest
import torch

from helpers import ensure_library

OK, INVALID, UNSUPPORTED, CUDA_ERR, TIMEOUT, DEVCHECK, WORKSPACE = range(7)
FAKE = 0x10000  # a non-NULL, 16-byte aligned "device pointer" that validation never touches
BIG = 1 << 40


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


def axes(lla, **kw):
    r = lla.lla_rope_axes(10000.0, lla.LLA_ROPE_HALF, (ctypes.c_int32 * 3)(16, 8, 8), lla.LLA_AXES_BLOCKS)
    for k, v in kw.items():
        setattr(r, k, (ctypes.c_int32 * 3)(*v) if k == "pairs" else v)
    return r


def prefix(lla, **kw):
    p = lla.lla_prefix(*(FAKE + 0x100000 * (i + 1) for i in range(5)))
    for k, v in kw.items():
        setattr(p, k, v)
    return p


BAD_AXES = [dict(base=1.0), dict(base=float("nan")), dict(base=1e300), dict(pairing=2), dict(pairing=-1), dict(order=2), dict(order=-1),
            dict(pairs=(16, 8, 9)), dict(pairs=(15, 8, 8)), dict(pairs=(33, -1, 0)), dict(pairs=(2**31 - 1, 2**31 - 1, 34))]


def test_rope_keys_axes_checks(lla):
    def store(d_rope=64, rope="", pool=FAKE, nb=4, k=FAKE, dt=0, pos=FAKE, slots=FAKE, N=3):
        rope = axes(lla) if rope == "" else rope
        return lla.library().lla_encode_rope_keys_axes(d_rope, None if rope is None else ctypes.byref(rope), pool, nb, k, dt, pos, slots, N, None)

    assert store(N=0) == OK
    assert store(N=0, k=None, pos=None, slots=None) == OK
    assert store(N=0, rope=axes(lla, pairs=(32, 0, 0))) == OK
    assert store(N=0, d_rope=16, rope=axes(lla, pairs=(0, 0, 8))) == OK
    for bad in BAD_AXES:
        assert store(N=0, rope=axes(lla, **bad)) == INVALID, bad
    for bad in (dict(rope=None), dict(d_rope=0), dict(d_rope=112), dict(d_rope=40), dict(pool=None), dict(pool=FAKE + 8), dict(nb=0),
                dict(k=None), dict(dt=2), dict(pos=None), dict(slots=None), dict(N=-1)):
        assert store(**bad) == INVALID, bad


def decode(lla, fn, rotary, has_plan, d=128, rk=96, rv=160, storage="bf16", d_rope=64, H=16, **kw):
    a = dict(B=0, max_ctx=512, loop=0, rope=axes(lla), pool=FAKE, w_up=FAKE, lens=FAKE, pos=FAKE, q=FAKE, qr=FAKE, ck=FAKE, cv=FAKE, ckr=FAKE,
             io=0, out=FAKE, ws=FAKE, ws_bytes=BIG, rope_pool=FAKE, plan=prefix(lla), num_blocks=100, max_blocks=8, table=FAKE)
    a.update(kw)
    ref = lambda x: None if x is None else ctypes.byref(x)
    g = lla.Geometry(4, H, d, rk, rv, storage).c()
    cd = lla.lla_codec(FAKE, FAKE, a["w_up"], FAKE, None, None)
    ch = lla.lla_cache(a["pool"], a["num_blocks"], a["table"], a["max_blocks"])
    args = [ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch)] + ([ref(a["plan"])] if has_plan else [])
    args += [a["rope_pool"], d_rope, ref(a["rope"]), a["pos"]] if rotary else []
    args += [a["lens"], a["B"], a["max_ctx"], a["loop"], a["q"]] + ([a["qr"]] if rotary else []) + [a["ck"], a["cv"]]
    args += ([a["ckr"]] if rotary else []) + [a["io"], a["out"], a["ws"], a["ws_bytes"], None]
    return getattr(lla.library(), fn)(*args)


@pytest.mark.parametrize("fn, rotary, has_plan", [("lla_decode_attn_prefix", False, True), ("lla_decode_attn_prefix_decoupled", True, True),
                                              ("lla_decode_attn_decoupled_axes", True, False)])
def test_decode_checks(lla, fn, rotary, has_plan):
    def call(**kw):
        return decode(lla, fn, rotary, has_plan, **kw)

    assert call() == OK
    assert call(lens=None, q=None, qr=None, out=None, ws=None, pos=None) == OK  # no batch
    assert call(ck=None, cv=None, ckr=None) == OK
    bad = [dict(w_up=None), dict(w_up=FAKE + 8), dict(pool=None), dict(pool=FAKE + 4), dict(table=None), dict(num_blocks=0), dict(max_blocks=0),
           dict(loop=4), dict(loop=-1), dict(B=-1), dict(B=1025), dict(max_ctx=-1), dict(max_ctx=513), dict(io=2), dict(ck=None), dict(cv=None),
           dict(B=1, lens=None), dict(B=1, q=None), dict(B=1, out=None), dict(B=1, ws=None), dict(d=12), dict(rk=3)]
    if rotary:
        bad += [dict(rope=None), dict(rope_pool=None), dict(rope_pool=FAKE + 8), dict(ckr=None), dict(B=1, qr=None), dict(d_rope=0), dict(d_rope=20)]
        bad += [dict(rope=axes(lla, **b)) for b in BAD_AXES]
    if has_plan:
        bad += [dict(plan=None), dict(plan=prefix(lla, num_groups=None)), dict(plan=prefix(lla, groups=None)), dict(plan=prefix(lla, groups=FAKE + 8)),
                dict(ws=FAKE + 8)]
        bad += [dict(B=1, plan=prefix(lla, **{n: None})) for n in ("members", "column", "own_page")]
    else:
        bad += [dict(B=1, pos=None)]
    for b in bad:
        assert call(**b) == INVALID, b
    unsupported = [dict(storage="fp32"), dict(d=64), dict(rk=192, rv=320), dict(rk=18, rv=30), dict(B=1024, max_ctx=2**31 - 1, max_blocks=2**25)]
    if rotary:
        unsupported += [dict(rk=128, rv=128), dict(d_rope=16, rope=axes(lla, pairs=(8, 0, 0)))]
    for b in unsupported:
        assert call(**b) == UNSUPPORTED, b


def test_prefix_workspace_checks(lla):
    so, n = lla.library(), ctypes.c_size_t()
    g = lambda **kw: ctypes.byref(lla.Geometry(**{**dict(T=4, H=16, d=128, r_k=96, r_v=160), **kw}).c())
    for B in (-1, 1025):
        assert so.lla_decode_prefix_workspace_size(g(), 0, B, ctypes.byref(n)) == INVALID
    assert so.lla_decode_prefix_workspace_size(g(), 0, 1, None) == INVALID
    assert so.lla_decode_prefix_workspace_size(None, 0, 1, ctypes.byref(n)) == INVALID
    for bad in (dict(r_k=192, r_v=320), dict(storage="fp32"), dict(d=64)):
        assert so.lla_decode_prefix_workspace_size(g(**bad), 0, 1, ctypes.byref(n)) == UNSUPPORTED
    assert so.lla_decode_prefix_workspace_size(g(r_k=128, r_v=128), 64, 1, ctypes.byref(n)) == UNSUPPORTED
    assert so.lla_decode_prefix_workspace_size(g(), 48, 1, ctypes.byref(n)) == UNSUPPORTED


def test_prefix_plan_checks(lla):
    B = 6
    place = dict(table=FAKE, lens=FAKE + 0x10000, num_groups=FAKE + 0x20000, groups=FAKE + 0x30000, members=FAKE + 0x40000, column=FAKE + 0x50000,
                 own_page=FAKE + 0x60000)
    size = dict(table=B * 8 * 4, lens=B * 4, num_groups=4, groups=9 * 16, members=3 * B * 4, column=3 * B * 4, own_page=B * 4)

    def plan(B=B, max_ctx=512, min_pages=1, num_blocks=100, max_blocks=8, cache=True, stop=False, **kw):
        a = {**place, **kw}
        ch = lla.lla_cache(None, num_blocks, a["table"], max_blocks)  # no pool is needed
        pl = lla.lla_prefix(*(a[n] for n in ("num_groups", "groups", "members", "column", "own_page")))
        return lla.library().lla_prefix_plan(ctypes.byref(ch) if cache else None, a["lens"], B, max_ctx, min_pages, ctypes.byref(pl), None)

    for bad in (dict(cache=False), dict(table=None), dict(lens=None), dict(B=-1), dict(B=1025), dict(max_ctx=-1), dict(max_ctx=513),
                dict(min_pages=0), dict(num_blocks=0), dict(max_blocks=0), dict(groups=FAKE + 0x30008)) + tuple({n: None} for n in list(place)[2:]):
        assert plan(**bad) == INVALID, bad
    assert plan(num_blocks=(1 << 24) + 1) == UNSUPPORTED
    assert plan(max_blocks=(1 << 24) + 1) == UNSUPPORTED
    for name in list(place)[2:]:  # what is written may overlap nothing
        step = 16 if name == "groups" else 4
        for other in place:
            if other != name:
                at = place[other]
                for bad in (at, at - (size[name] - 1) // step * step, at + (size[other] - 1) // step * step):
                    assert plan(**{name: bad}) == INVALID, (name, other)
    assert lla.library().lla_prefix_plan(None, None, 0, 0, 1, None, None) == INVALID


def test_admit_checks(lla):
    so, need = lla.library(), ctypes.c_size_t()
    assert so.lla_pages_admit_workspace_size(1024, ctypes.byref(need)) == OK
    for n in (-1, 1025):
        assert so.lla_pages_admit_workspace_size(n, ctypes.byref(need)) == INVALID
    assert so.lla_pages_admit_workspace_size(1, None) == INVALID
    n, N = 3, 50
    place = {k: FAKE + 0x10000 * i for i, k in enumerate(("ref", "table", "lens", "rows", "parents", "keep", "new", "slots", "cu", "admitted", "free", "ws"))}
    size = dict(ref=400, table=128, lens=16, rows=4 * n, parents=4 * n, keep=4 * n, new=4 * n, slots=8 * N, cu=4 * n + 4, admitted=n, free=4, ws=need.value)

    def admit(n=n, N=N, L=0, pools=None, ws_bytes=BIG, pages=None, **kw):
        a = {**place, **kw}
        p = lla.lla_pages(a["ref"], 100, a["table"], 8, a["lens"], 4)
        for k, v in (pages or {}).items():
            setattr(p, k, v)
        return so.lla_pages_admit(ctypes.byref(p), pools, L, a["rows"], a["parents"], a["keep"], a["new"], n, a["slots"], N, a["cu"], a["admitted"],
                                  a["free"], a["ws"], ws_bytes, None)

    assert admit(ws_bytes=need.value - 1) == WORKSPACE
    for bad in [dict(n=-1), dict(n=1025), dict(N=-1), dict(L=-1), dict(L=1), dict(ws=FAKE + 8), dict(ref=FAKE + 4), dict(pages=dict(S=1025)),
                dict(pages=dict(num_blocks=0)), dict(pages=dict(max_blocks_per_seq=0))] + [{k: None} for k in place if k != "free"]:
        assert admit(**bad) == INVALID, bad
    assert admit(L=129, pools=(lla.lla_pool * 129)()) == UNSUPPORTED
    assert admit(L=1, pools=(lla.lla_pool * 1)(lla.lla_pool(FAKE, 0, 16, 16))) == INVALID
    written = ("slots", "cu", "admitted", "free", "ws", "ref", "table", "lens")
    step = dict(slots=8, admitted=1, ws=16, ref=16)
    for name in written:
        for other in place:
            if other != name:
                for bad in (place[other], place[other] + (size[other] - 1) // step.get(name, 4) * step.get(name, 4)):
                    assert admit(**{name: bad}) == INVALID, (name, other)


def test_python_refuses_wrong_arrays(lla):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    w = torch.zeros(1 << 16, dtype=torch.uint8)
    p = lla.Pages(i(10), i(4, 2), i(4))
    g, cache, rope = lla.Geometry(4, 2, 128, 96, 160), lla.Cache(None, 10, i(4, 2), 2), lla.RopeAxes(1e4, 0, (16, 8, 8))
    plan = lla.Prefix.empty(4, "cpu")
    x = torch.zeros(4, 2, 128)
    codec = lla.Codec(x, x, x, x)
    for call in (lambda: lla.lla_pages_admit(p, lla.Pools(), i(2), i(2), i(2), i(2), torch.zeros(9, dtype=torch.int64), i(3), w[:2], w),
                 lambda: lla.lla_prefix_plan(cache, i(4), 128, plan),
                 lambda: lla.lla_encode_rope_keys_axes(64, rope, w, 1, torch.zeros(2, 64), i(3, 2), torch.zeros(2, dtype=torch.int64)),
                 lambda: lla.lla_decode_attn_prefix(g, codec, cache, plan, i(4), 128, 0, x, x, x, x, w),
                 lambda: lla.lla_decode_attn_prefix_decoupled(g, codec, cache, plan, w, 64, rope, None, i(4), 128, 0, x, x, x, x, x, x, w),
                 lambda: lla.lla_decode_attn_decoupled_axes(g, codec, cache, w, 64, rope, i(3, 4), i(4), 128, 0, x, x, x, x, x, x, w)):
        with pytest.raises(ValueError, match="CUDA tensors"):
            call()
    with pytest.raises(ValueError, match="pairs of 3 axes"):
        lla.RopeAxes(1e4, 0, (16, 16)).c()
    with pytest.raises(ValueError, match="k_rope"):
        lla.lla_encode_rope_keys_axes(64, rope, w, 1, torch.zeros(2, 32), i(3, 2), torch.zeros(2, dtype=torch.int64))


@pytest.mark.parametrize("name, count", [("encode_rope_keys_axes", 8), ("decode_attn_decoupled_axes", 18), ("prefix_plan", 6),
                                         ("decode_attn_prefix", 13), ("decode_attn_prefix_decoupled", 19), ("pages_admit", 12)])
def test_unusual_arguments_are_left_to_python(lla, name, count):
    native = getattr(lla._native(), name)
    t = torch.zeros(2, 2, dtype=torch.int32)
    for x in (t, FAKE, "x", None, lla.Pages(t[0], t, t[0]), lla.RopeAxes(1e4, 0, (1, 2)), lla.Prefix.empty(2, "cpu")):
        assert native(*[x] * count) is None
    with pytest.raises(TypeError):
        native(None)
