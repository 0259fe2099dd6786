"""lla_pages_admit against a plain model of the documented behaviour: after every call the ledger, every table entry, every
length, slot and byte of every pool are equal; and a run of requests through admission, plan, decode and growth."""
import random

import numpy as np
import pytest
import torch

from helpers import ensure_library
from test_pages_gpu import Both, dev, shapes, up

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, I64, U8 = torch.int32, torch.int64, torch.uint8


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    m.lla_clear_device_error()
    return m


@pytest.fixture(autouse=True)
def no_error_left(lla):
    yield
    word = lla.lla_get_device_error()
    lla.lla_clear_device_error()
    assert word == 0


def plain_admit(p, rows, parents, keep, new, N):
    """The call on a Plain: admitted, slots, cu_new, free blocks left.  (A request that is wrong is given as row None.)"""
    free = [b for b in range(p.nb) if not p.ref[b]]
    taken, tokens, ok, slots, cu = 0, 0, [], [], [0]
    full = False
    for r, q, k, n in zip(rows, parents, keep, new):
        need = up(n) - k // 64
        if r is not None:
            full = full or taken + need > len(free) or tokens + n - k > N
        if r is None or full:
            ok.append(0)
            cu.append(cu[-1])
            continue
        ok.append(1)
        mine = [int(b) for b in p.table[q, :k // 64]] if q >= 0 else []
        fresh = free[taken:taken + need]
        taken += need
        tokens += n - k
        for b in mine + fresh:
            p.ref[b] += 1
        if k % 64:
            p.copy_rows(int(p.table[q, k // 64]), fresh[0], k % 64)
        p.table[r, :up(n)] = mine + fresh
        p.lens[r] = n
        slots += [int(p.table[r, i // 64]) * 64 + i % 64 for i in range(k, n)]
        cu.append(cu[-1] + n - k)
    return ok, slots + [-1] * (N - len(slots)), cu, len(free) - taken


def admit(lla, x, i, rows, parents, keep, new, N, bad=(), free=True, **kw):
    n = len(rows)
    out = dict(slots=torch.full((N,), 12345, dtype=I64, device=DEV), cu=torch.full((n + 1,), 99, dtype=I32, device=DEV),
               admitted=torch.full((n,), 9, dtype=U8, device=DEV))
    left = torch.full((1,), 99, dtype=I32, device=DEV) if free else None
    ws = torch.full((lla.lla_pages_admit_workspace_size(n),), 0xA5, dtype=U8, device=DEV)
    lla.lla_pages_admit(x.sets[i], x.pools, dev(rows), dev(parents), dev(keep), dev(new), out["slots"], out["cu"], out["admitted"], ws,
                        free_blocks=left, **kw)
    ok, slots, cu, rest = plain_admit(x.plain[i], [None if j in bad else r for j, r in enumerate(rows)], parents, keep, new, N)
    assert out["admitted"].tolist() == ok
    assert out["cu"].tolist() == cu
    assert out["slots"].tolist() == slots
    assert left is None or left.item() == rest
    x.check(i)
    return ok


@pytest.mark.parametrize("name", ["heads", "granules of 4", "fp32", "2d", "with rotary planes", "none"])
def test_random_calls_in_a_row(lla, name):
    """Requests admitted, grown and ended as a scheduler does it, with room and without."""
    r = random.Random(len(name))
    S, nb, mb = 12, 67, 8
    x = Both(lla, shapes(lla, name), nb, mb, S)
    refused = 0
    for step in range(40):
        p = x.plain[0]
        empty = [s for s in range(S) if p.lens[s] == 0]
        live = [s for s in range(S) if p.lens[s]]
        if empty and r.random() < 0.6:
            n = r.randint(0, len(empty))
            rows, parents, keep, new = r.sample(empty, n), [], [], []
            for _ in range(n):
                q = r.choice(live) if live and r.random() < 0.7 else -1
                k = r.choice([0, p.lens[q], r.randint(0, p.lens[q]), p.lens[q] // 64 * 64]) if q >= 0 else 0
                parents.append(q)
                keep.append(k)
                new.append(min(mb * 64, k + r.choice([0, 1, 63, 64, 65, r.randint(0, 200)])))
            total = sum(a - k for a, k in zip(new, keep))
            ok = admit(lla, x, 0, rows, parents, keep, new, r.choice([total, total + 5, total // 2]), free=r.random() < 0.5)
            refused += ok.count(0)
        elif live and r.random() < 0.6:
            x.free(0, r.sample(live, r.randint(1, len(live))))
        elif live:
            x.extend(0, [int(s in live and p.lens[s] < mb * 64) for s in range(S)])
            lla.lla_clear_device_error()  # (no room is an error there)
    assert refused


@pytest.mark.parametrize("keep", [0, 1, 63, 64, 65, 127, 128, 130])
def test_every_way_to_keep(lla, keep):
    x = Both(lla, shapes(lla, "granules of 4"), 40, 6, 6)
    x.extend(0, [130, 0, 0, 0, 0, 0])
    news = [keep, keep + 1, 130 + keep, 384, keep]
    admit(lla, x, 0, [5, 1, 4, 2, 3], [0] * 5, [keep] * 5, news, sum(news) - 5 * keep)


def test_nothing_asked_for(lla):
    x = Both(lla, shapes(lla, "none"), 8, 2, 3)
    assert admit(lla, x, 0, [], [], [], [], 0) == []
    assert admit(lla, x, 0, [], [], [], [], 4) == []
    assert admit(lla, x, 0, [2], [-1], [0], [0], 0) == [1]


def test_the_first_without_room_ends_it(lla):
    x = Both(lla, shapes(lla, "heads"), 6, 6, 5)
    assert admit(lla, x, 0, [0, 1, 2, 3], [-1] * 4, [0] * 4, [128, 320, 64, 0], 1000) == [1, 0, 0, 0]     # 2 blocks, then 5 of 4
    assert admit(lla, x, 0, [1, 2, 3], [0, 0, 0], [128, 64, 0], [130, 90, 1], 28) == [1, 1, 0]            # the tokens run out
    assert admit(lla, x, 0, [3, 4], [0, 0], [128, 128], [128, 128], 0) == [1, 1]                          # nothing is needed


def test_wrong_requests_take_nothing(lla):
    seq, ctx = lla.LLA_DEVERR_SEQUENCE, lla.LLA_DEVERR_CONTEXT
    for wrong, bit in [((4, 0, 0, 9), seq), ((-1, 0, 0, 9), seq), ((2, 4, 0, 9), seq), ((2, -2, 0, 9), seq), ((1, 0, 0, 9), seq), ((0, 0, 0, 9), ctx),
                       ((2, 0, 101, 200), ctx), ((2, 0, -1, 9), ctx), ((2, 0, 50, 49), ctx), ((2, -1, 1, 9), ctx), ((2, 0, 0, 257), ctx),
                       ((2, 0, 0, -1), ctx), ((2, 0, 0, 2**31 - 1), ctx), ((2, 0, -2**31, 2**31 - 1), ctx), ((2, 3, 1, 9), ctx)]:
        x = Both(lla, shapes(lla, "fp32"), 30, 4, 4)
        x.extend(0, [100, 0, 0, 0])
        r, q, k, n = wrong
        admit(lla, x, 0, [1, r, 3], [0, q, 0], [70, k, 33], [90, n, 140], 300, bad=(1,))
        assert lla.lla_get_device_error() == bit, wrong
        lla.lla_clear_device_error()


def test_blocks_that_are_none(lla):
    for page, bit_only in ((1, True), (0, False)):
        x = Both(lla, [], 30, 4, 3)
        x.extend(0, [100, 0, 0])
        x.sets[0].block_table[0, page] = 30
        ws = torch.zeros(lla.lla_pages_admit_workspace_size(1), dtype=U8, device=DEV)
        cu, ok = torch.zeros(2, dtype=I32, device=DEV), torch.zeros(1, dtype=U8, device=DEV)
        lla.lla_pages_admit(x.sets[0], x.pools, dev([1]), dev([0]), dev([90]), dev([100]), torch.zeros(10, dtype=I64, device=DEV), cu, ok, ws)
        assert lla.lla_get_device_error() == lla.LLA_DEVERR_BLOCK_ID
        lla.lla_clear_device_error()
        assert ok.item() == (0 if bit_only else 1)


@pytest.mark.parametrize("nb", [4096, 100000])
def test_a_full_batch(lla, nb):
    """1024 sequences, long kept parts, both sizes of the planning cluster."""
    r = random.Random(nb)
    S, mb = 1024, 90
    x = Both(lla, [], nb, mb, S)
    lens = [r.randint(1, 5000) if s < 30 else 0 for s in range(S)]
    x.extend(0, lens)
    rows = list(range(30, S))
    r.shuffle(rows)
    parents = [r.randint(-1, 29) for _ in rows]
    keep = [r.randint(0, lens[q]) if q >= 0 else 0 for q in parents]
    new = [k + r.randint(0, 300) for k in keep]
    ok = admit(lla, x, 0, rows, parents, keep, new, sum(new) - sum(keep) + 3)
    assert (0 in ok) == (nb == 4096)


def test_captured_and_on_another_stream(lla):
    x = Both(lla, shapes(lla, "heads"), 50, 6, 6)
    x.extend(0, [200, 0, 0, 0, 0, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        admit(lla, x, 0, [1, 2], [0, 0], [70, 128], [100, 300], 202)
    torch.cuda.current_stream().wait_stream(side)
    x.free(0, [1, 2])
    args = [dev([1, 2]), dev([0, 0]), dev([70, 128]), dev([100, 300]), torch.zeros(202, dtype=I64, device=DEV), torch.zeros(3, dtype=I32, device=DEV),
            torch.zeros(2, dtype=U8, device=DEV), torch.zeros(lla.lla_pages_admit_workspace_size(2), dtype=U8, device=DEV)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lla.lla_pages_admit(x.sets[0], x.pools, *args)
    args[2].copy_(dev([1, 200]))
    g.replay()
    plain_admit(x.plain[0], [1, 2], [0, 0], [1, 200], [100, 300], 202)
    x.check(0)
    assert args[6].tolist() == [1, 1]


def test_requests_from_admission_to_decode(lla):
    """Samples of two resident prompts, as a serving step makes them: admission, the encodes of the new tokens, the plan, a
    decode, growth by a token and a decode with the same plan, in layers that share one table; all against 64 bits."""
    from test_prefix_decode_gpu import Batch

    H, rk, rv, dr, nb, mb, S = 2, 96, 160, 32, 64, 8, 12
    x = Batch(lla, [[0]] * S, [64] * S, H=H, d_rope=dr)
    g = torch.Generator().manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=g).to(DEV)
    x.nb, x.pool = nb, torch.zeros(nb, H, 64 * (rk + rv), dtype=torch.bfloat16, device=DEV)
    x.planes = torch.zeros(nb, 64 * dr, dtype=torch.bfloat16, device=DEV)
    pages = lla.Pages(torch.zeros(nb, dtype=I32, device=DEV), torch.full((S, mb), -1, dtype=I32, device=DEV), torch.zeros(S, dtype=I32, device=DEV))
    x.codec = lla.Codec(n(H, 512, rk).bfloat16() * 0.05, n(H, 512, rv).bfloat16() * 0.05, x.wk, x.wv)
    x.cache, x.lens_t, x.max_ctx = lla.Cache(x.pool, nb, pages.block_table, mb), pages.context_lens, mb * 64
    pools = lla.Pools([lla.lla_cache_pool(x.geom, x.pool), lla.lla_rope_pool(dr, x.planes)])
    ws = torch.zeros(lla.lla_pages_admit_workspace_size(S), dtype=U8, device=DEV)

    def step(rows, parents, keep, new, spare):
        tokens = sum(a - k for a, k in zip(new, keep))
        slots, cu, ok = torch.zeros(tokens + spare, dtype=I64, device=DEV), torch.zeros(len(rows) + 1, dtype=I32, device=DEV), torch.zeros(len(rows), dtype=U8, device=DEV)
        lla.lla_pages_admit(pages, pools, dev(rows), dev(parents), dev(keep), dev(new), slots, cu, ok, ws)
        encode(slots)
        return ok

    def encode(slots):
        N = slots.numel()
        lla.lla_encode(x.geom, x.codec, x.cache, n(4, N, H, 128), n(4, N, H, 128), slots)
        lla.lla_encode_rope_keys_axes(dr, x.rope, x.planes, nb, n(N, dr), torch.randint(0, 5000, (3, N), generator=g, dtype=I32).to(DEV), slots)

    assert step([3, 7], [-1, -1], [0, 0], [300, 190], 2).all()
    rows = [0, 1, 2, 4, 5, 6, 8, 9, 10, 11]
    assert step(rows, [3, 7, 3, 3, 7, 7, 3, 3, 7, 3], [300, 190, 299, 256, 128, 100, 64, 300, 190, 1], [310, 191, 299, 300, 200, 130, 64, 301, 200, 50], 1).all()
    x.lens = pages.context_lens.tolist()

    def check():
        x.table = pages.block_table.cpu()
        if hasattr(x, "_u8"):
            del x._u8
        for pass1 in (True, False):
            x.check(x.decode(pass1=pass1), pass1=pass1)

    x.replan()
    assert x.plan.num_groups.item() >= 3
    check()
    slots = torch.zeros(S, dtype=I64, device=DEV)
    lla.lla_pages_extend(pages, pools, slots, ws_extend := torch.zeros(lla.lla_pages_extend_workspace_size(S), dtype=U8, device=DEV))
    encode(slots)
    x.lens = [L + 1 for L in x.lens]
    assert pages.context_lens.tolist() == x.lens and ws_extend.numel()
    check()
    x.replan()
    check()
