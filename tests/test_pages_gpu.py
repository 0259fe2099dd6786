"""Sequences that share pages (lla_pages_fork, lla_pages_extend, lla_pages_free, lla_pages_compact) against a plain
model of the documented behaviour in Python integers: after every call the whole ledger, every table entry (those
that nobody holds, too), every length, slot and byte of every pool are equal."""
import numpy as np
import pytest
import torch

from helpers import ensure_library

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    m.lla_clear_device_error()
    return m


@pytest.fixture(autouse=True)
def no_error_left(lla):
    lla.lla_clear_device_error()
    yield
    assert lla.lla_get_device_error() == 0


def dev(v, t=I32):
    return torch.tensor(v, dtype=t, device=DEV)


def up(n):
    return -(-n // 64)


class Plain:
    """The documented behaviour, sequence by sequence."""

    def __init__(self, nb, mb, S, pools):
        self.nb, self.mb, self.S = nb, mb, S
        self.ref = [0] * nb
        self.table = np.full((S, mb), -7, np.int64)
        self.lens = [0] * S
        self.pools = pools  # [(array [nb][pages][bytes], k_row_bytes, v_row_bytes)]

    def held(self, s):
        return [int(b) for b in self.table[s, :up(self.lens[s])]]

    def fork(self, other, parents):
        """self's sequences from other's."""
        old = {s: other.held(s) for s in range(other.S)}
        for s, p in enumerate(parents):
            blocks = old[p] if p >= 0 else []
            self.table[s, :len(blocks)] = blocks
            self.lens[s] = other.lens[p] if p >= 0 else 0
            for b in blocks:
                self.ref[b] += 1
        for blocks in old.values():
            for b in blocks:
                self.ref[b] -= 1

    def extend(self, n, skip):
        n = [0 if skip[s] else n[s] for s in range(self.S)]
        before = list(self.lens)
        part = [s for s in range(self.S) if n[s] and self.lens[s] % 64]
        tails = {}
        for s in part:
            tails.setdefault(int(self.table[s, self.lens[s] // 64]), []).append(s)
        copies = {s for b, who in tails.items() if self.ref[b] > 1 for s in (who[1:] if len(who) == self.ref[b] else who)}
        need = sum(up(self.lens[s] + n[s]) - up(self.lens[s]) + (s in copies) for s in range(self.S))
        free = [b for b in range(self.nb) if not self.ref[b]]
        slots = [[] for _ in range(self.S)]
        if need > len(free):
            return before, None, len(free)
        taken = iter(free)
        for s in range(self.S):
            L = self.lens[s]
            if s in copies:
                old, new = int(self.table[s, L // 64]), next(taken)
                self.table[s, L // 64] = new
                self.ref[old] -= 1
                self.ref[new] = 1
                self.copy_rows(old, new, L % 64)
            for i in range(up(L), up(L + n[s])):
                b = next(taken)
                self.table[s, i] = b
                self.ref[b] = 1
            self.lens[s] = L + n[s]
            slots[s] = [int(self.table[s, p // 64]) * 64 + p % 64 for p in range(L, L + n[s])]
        return before, slots, len(free) - need

    def copy_rows(self, src, dst, rows):
        for a, k, v in self.pools:
            g = 16 if k % 16 == 0 else 4
            kp = a[:, :, :64 * k].reshape(self.nb, a.shape[1], k // g, 64, g)
            kp[dst, :, :, :rows] = kp[src, :, :, :rows]
            a[:, :, :64 * k] = kp.reshape(self.nb, a.shape[1], 64 * k)
            a[dst, :, 64 * k:64 * k + rows * v] = a[src, :, 64 * k:64 * k + rows * v]

    def free(self, seqs):
        for s in seqs:
            if s >= 0:
                for b in self.held(s):
                    self.ref[b] -= 1
                self.lens[s] = 0

    def compact(self):
        live = sum(r != 0 for r in self.ref)
        holes = [b for b in range(live) if not self.ref[b]]
        movers = [b for b in range(live, self.nb) if self.ref[b]]
        remap = [b if self.ref[b] else -1 for b in range(self.nb)]
        for src, dst in zip(movers, holes):
            remap[src] = dst
            self.ref[dst], self.ref[src] = self.ref[src], 0
            for a, _, _ in self.pools:
                a[dst] = a[src]
        for s in range(self.S):
            for i in range(up(self.lens[s])):
                self.table[s, i] = remap[self.table[s, i]]
        return remap, live


class Both:
    """The library's page sets (two, for forks) and the plain model's, with the same calls on both."""

    def __init__(self, lla, pools, nb, mb, S, S2=None, seed=0):
        self.lla, self.nb = lla, nb
        self.t_pools = []
        plain_pools = []
        g = torch.Generator().manual_seed(seed)
        for describe, geom, pages, k, v in pools:
            x = torch.randint(0, 256, (nb, pages, 64 * (k + v)), generator=g, dtype=torch.uint8)
            plain_pools.append((x.numpy().copy(), k, v))
            x = x.to(DEV)
            p = describe(geom, x)
            assert (p.pages, p.k_row_bytes, p.v_row_bytes) == (pages, k, v)
            self.t_pools.append(p)
        self.pools = lla.Pools(self.t_pools)
        ref = torch.zeros(nb, dtype=I32, device=DEV)
        self.ref = ref
        self.sets, self.plain = [], []
        for n in (S, S if S2 is None else S2):
            self.sets.append(lla.Pages(ref, torch.full((n, mb), -7, dtype=I32, device=DEV), torch.zeros(n, dtype=I32, device=DEV)))
            self.plain.append(Plain(nb, mb, n, plain_pools))
        self.plain[1].ref = self.plain[0].ref
        self.ws = torch.full((lla.lla_pages_extend_workspace_size(max(p.S for p in self.plain)),), 0xA5, dtype=torch.uint8, device=DEV)
        self.cws = torch.full((lla.lla_pages_compact_workspace_size(nb),), 0xA5, dtype=torch.uint8, device=DEV)

    def check(self, i):
        p, t = self.plain[i], self.sets[i]
        assert t.context_lens.tolist() == p.lens
        assert self.ref.tolist() == p.ref
        assert np.array_equal(t.block_table.cpu().numpy(), p.table)
        for x, (a, _, _) in zip(self.t_pools, p.pools):
            assert np.array_equal(x.base.cpu().numpy(), a)

    def fork(self, i, parents):
        self.lla.lla_pages_fork(self.sets[i], self.sets[1 - i], dev(parents))
        self.plain[1 - i].fork(self.plain[i], parents)
        self.plain[i].lens = [0] * self.plain[i].S  # nothing is held there any more
        self.sets[i].context_lens.zero_()
        self.check(1 - i)
        return 1 - i

    def extend(self, i, n, skip=None, packed=True, spare=0):
        S = self.plain[i].S
        skips = skip or [0] * S
        total = sum(n)
        slots = torch.full((total + spare,), 12345, dtype=torch.int64, device=DEV)
        before, free = torch.full((S,), 99, dtype=I32, device=DEV), torch.full((1,), 99, dtype=I32, device=DEV)
        cu = dev(np.cumsum([0] + list(n)).tolist()) if packed else None
        self.lla.lla_pages_extend(self.sets[i], self.pools, slots, self.ws, cu_new=cu,
                                  skip=None if skip is None else dev(skip, torch.uint8), lens_before=before, free_blocks=free)
        want_before, want, left = self.plain[i].extend(n, skips)
        flat = []
        for s in range(S):
            flat += want[s] if want is not None and not skips[s] else [-1] * n[s]
        assert slots.tolist() == flat + [-1] * spare
        assert before.tolist() == want_before and free.item() == left
        self.check(i)
        return want is not None

    def free(self, i, seqs):
        self.lla.lla_pages_free(self.sets[i], dev(seqs))
        self.plain[i].free(seqs)
        self.check(i)

    def compact(self, i):
        remap, live = torch.full((self.nb,), 99, dtype=I32, device=DEV), torch.full((1,), 99, dtype=I32, device=DEV)
        self.lla.lla_pages_compact(self.sets[i], self.pools, remap, live, self.cws)
        want, R = self.plain[i].compact()
        assert remap.tolist() == want and live.item() == R
        self.check(i)


def shapes(lla, name):
    """Pools as (describe, geometry, pages of a block, K row bytes, V row bytes)."""
    G = lla.Geometry
    heads = lambda H, rk, rv, st: (lla.lla_cache_pool, G(4, H, 128, rk, rv, st), H, rk * (2 if st == "bf16" else 4), rv * (2 if st == "bf16" else 4))
    return {"heads": [heads(2, 96, 160, "bf16")] * 2,
            "granules of 4": [heads(3, 18, 30, "bf16")] * 3,
            "fp32": [heads(1, 6, 10, "fp32"), heads(2, 8, 2, "fp32")],
            "2d": [(lla.lla_cache_2d_pool, G(4, 16, 128, 288, 480, "bf16"), 1, 576, 960)],
            "with rotary planes": [heads(2, 96, 160, "bf16"), (lla.lla_rope_pool, 64, 1, 128, 0), (lla.lla_rope_pool, 16, 1, 32, 0)],
            "none": []}[name]


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("name", ["heads", "granules of 4", "fp32", "2d", "with rotary planes", "none"])
def test_random_calls_in_a_row(lla, name, seed):
    """Forks, growths, ends and compactions in random order, as a scheduler makes them."""
    r = np.random.RandomState(seed)
    S, nb, mb = 9, 61, 7
    x = Both(lla, shapes(lla, name), nb, mb, S, seed=seed)
    i, refused = 0, 0
    for step in range(60):
        what = r.choice(["fork", "extend", "extend", "extend", "free", "compact"])
        room = [mb * 64 - L for L in x.plain[i].lens]
        if what == "fork":
            i = x.fork(i, [int(r.randint(-1, S)) for _ in range(S)])
        elif what == "extend":
            kind = r.randint(3)
            skip = [int(v) for v in r.randint(0, 3, S) == 0] if r.randint(2) else None
            if kind == 0:  # one token each, all beams
                skip = [int((skip or [0] * S)[s] or room[s] < 1) for s in range(S)]
                refused += not x.extend(i, [1] * S, skip, packed=bool(r.randint(2)))
            else:
                n = [int(min(room[s], r.choice([0, 1, 2, 63, 64, 65, r.randint(0, 200)]))) for s in range(S)]
                refused += not x.extend(i, n, skip, spare=int(r.randint(0, 3)))
            if lla.lla_get_device_error() == lla.LLA_DEVERR_PAGES and refused:
                lla.lla_clear_device_error()
        elif what == "free":
            x.free(i, [int(s) for s in r.permutation(S)[:r.randint(1, 4)]])
        else:
            x.compact(i)


@pytest.mark.parametrize("L", [0, 1, 63, 64, 65, 127, 128])
def test_beams_of_one_prompt_grow(lla, L):
    """A prompt forked into beams that all grow by a token: all but the lowest copy a page that is not full."""
    W = 5
    x = Both(lla, shapes(lla, "granules of 4"), 40, 4, W)
    x.extend(0, [L] + [0] * (W - 1))
    i = x.fork(0, [0] * W)
    held = x.sets[i].block_table[:, :up(L)].clone()
    x.extend(i, [1] * W, packed=False)
    if L % 64:
        assert torch.equal(x.sets[i].block_table[0, :up(L)], held[0])
        assert len(set(x.sets[i].block_table[:, L // 64].tolist())) == W
    # a beam that does not grow keeps the page, and every other copies it
    i = x.fork(i, [1] * W)
    x.extend(i, [0, 1, 1, 0, 1])
    x.compact(i)
    x.free(i, [3, 0, 3, -1, 3])
    x.extend(i, [7] * W, skip=[1, 0, 0, 0, 1])


def test_too_few_blocks_change_nothing(lla):
    x = Both(lla, shapes(lla, "heads"), 6, 8, 3)
    assert x.extend(0, [100, 65, 64])     # 5 of 6 blocks
    assert not x.extend(0, [64, 64, 64])  # 3 more
    assert lla.lla_get_device_error() == lla.LLA_DEVERR_PAGES
    lla.lla_clear_device_error()
    assert x.extend(0, [28, 60, 0])       # in the pages there are: none is needed
    assert x.extend(0, [0, 0, 1])
    assert not x.extend(0, [1, 0, 0])
    lla.lla_clear_device_error()
    x.free(0, [1])
    assert x.extend(0, [1, 0, 0])


def test_empty_batches_and_growths(lla):
    x = Both(lla, shapes(lla, "heads"), 10, 2, 4)
    x.extend(0, [0, 0, 0, 0])
    x.extend(0, [0, 0, 0, 0], spare=5)
    x.compact(0)
    x.free(0, [0, 1, 2, 3])
    i = x.fork(0, [-1, -1, 2, 0])
    x.extend(i, [1, 128, 0, 127])
    none = lla.Pages(x.ref, torch.zeros(0, 2, dtype=I32, device=DEV), torch.zeros(0, dtype=I32, device=DEV))
    slots, free = torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    lla.lla_pages_extend(none, x.pools, slots, x.ws, cu_new=dev([0]), free_blocks=free)
    assert slots.tolist() == [-1] * 3 and free.item() == 10 - 5
    lla.lla_pages_free(none, dev([]))
    x.check(i)
    # a fork into nothing frees everything
    lla.lla_pages_fork(x.sets[i], none, dev([]))
    assert x.ref.tolist() == [0] * 10


@pytest.mark.parametrize("S_to", [1, 3, 40])
def test_fork_to_another_number_of_sequences(lla, S_to):
    r = np.random.RandomState(S_to)
    x = Both(lla, [], 200, 5, 7, S_to)
    x.extend(0, [int(n) for n in r.randint(0, 320, 7)])
    x.fork(0, [int(p) for p in r.randint(-1, 7, S_to)])


def test_large_ledger_and_batch(lla):
    """Block ids behind the first part of a ledger that several CTAs share, 1024 sequences, rows longer than one CTA."""
    r = np.random.RandomState(3)
    S, nb, mb = 1024, 70001, 1500
    x = Both(lla, [], nb, mb, S)
    x.ref[:20000] = 1  # held by someone without a table here
    x.plain[0].ref[:20000] = [1] * 20000
    n = [int(v) for v in r.randint(0, 2500, S)]
    n[5] = 1500 * 64
    x.extend(0, n)
    i = x.fork(0, [int(p) for p in r.randint(-1, S, S)])
    x.free(i, [int(s) for s in r.permutation(S)[:500]])
    x.extend(i, [1] * S, skip=[int(L == mb * 64) for L in x.plain[i].lens], packed=False)
    x.compact(i)
    x.extend(i, [0 if L == mb * 64 else 1 for L in x.plain[i].lens])


def test_tables_and_lengths_in_slices(lla):
    """Arrays that start off a 16-byte boundary; rows of an odd length."""
    x = Both(lla, shapes(lla, "fp32"), 30, 3, 4)
    for i in range(2):
        big = torch.full((1 + 4 * 3,), -7, dtype=I32, device=DEV)
        x.sets[i].block_table = big[1:].view(4, 3)
        x.sets[i].context_lens = torch.zeros(7, dtype=I32, device=DEV)[3:]
    x.extend(0, [64, 3, 130, 0])
    i = x.fork(0, [2, 2, 1, 1])
    x.extend(i, [1] * 4, packed=False)
    x.compact(i)


def test_bad_device_data_is_flagged_and_left_alone(lla):
    def fresh():
        x = Both(lla, shapes(lla, "granules of 4"), 12, 3, 4)
        x.extend(0, [70, 10, 64, 0])
        return x

    def flagged(bit):
        assert lla.lla_get_device_error() == bit
        lla.lla_clear_device_error()

    # parents outside the batch count as -1
    x = fresh()
    lla.lla_pages_fork(x.sets[0], x.sets[1], dev([4, -2, 0, 1]))
    flagged(lla.LLA_DEVERR_SEQUENCE)
    x.plain[1].fork(x.plain[0], [-1, -1, 0, 1])
    x.check(1)
    # a parent that the new table has no room for
    x = fresh()
    small = lla.Pages(x.ref, torch.full((2, 1), -7, dtype=I32, device=DEV), torch.zeros(2, dtype=I32, device=DEV))
    lla.lla_pages_fork(x.sets[0], small, dev([0, 1]))
    flagged(lla.LLA_DEVERR_CONTEXT)
    assert small.context_lens.tolist() == [0, 10] and x.ref.sum().item() == 1
    # sequence numbers outside the batch
    x = fresh()
    lla.lla_pages_free(x.sets[0], dev([4, 1, 1000]))
    flagged(lla.LLA_DEVERR_SEQUENCE)
    x.plain[0].free([1])
    x.check(0)
    # growth past the table, a length that no table holds, prefix sums that fall: those sequences stay
    slots = torch.zeros(200, dtype=torch.int64, device=DEV)
    for cu, lens, stay in (([0, 123, 124, 124, 124], None, [0]), ([0, 1, 2, 2, 2], [-5, 10, 64, 0], [0]),
                           ([0, 1, 2, 2, 2], [1 << 30, 10, 64, 0], [0]), ([0, 3, 1, 2, 2], None, [1]),
                           ([-1, 1, 2, 2, 2], None, [0]), ([0, 1, 2, 2, 201], None, [3])):
        x = fresh()
        if lens:
            x.sets[0].context_lens.copy_(dev(lens))
        was, table = x.sets[0].context_lens.tolist(), x.sets[0].block_table.clone()
        lla.lla_pages_extend(x.sets[0], x.pools, slots, x.ws, cu_new=dev(cu))
        flagged(lla.LLA_DEVERR_CONTEXT)
        now = x.sets[0].context_lens.tolist()
        for s in range(4):
            assert now[s] == (was[s] if s in stay else was[s] + cu[s + 1] - cu[s]), (cu, lens, s)
        assert torch.equal(x.sets[0].block_table[stay], table[stay])
    # a last page that is no block
    for bad in (-1, 12, 1 << 30):
        x = fresh()
        x.sets[0].block_table[1, 0] = bad
        lla.lla_pages_extend(x.sets[0], x.pools, slots[:4], x.ws)
        flagged(lla.LLA_DEVERR_BLOCK_ID)
        assert x.sets[0].context_lens.tolist() == [71, 10, 65, 1] and slots[1].item() == -1
        # freeing and compacting leave it, too
        lla.lla_pages_free(x.sets[0], dev([1]))
        flagged(lla.LLA_DEVERR_BLOCK_ID)
    x = fresh()
    x.sets[0].block_table[1, 0] = 40
    x.sets[0].context_lens[3] = -1
    remap, live = torch.zeros(12, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    lla.lla_pages_compact(x.sets[0], x.pools, remap, live, x.cws)
    flagged(lla.LLA_DEVERR_BLOCK_ID | lla.LLA_DEVERR_CONTEXT)
    assert live.item() == 4 and x.sets[0].block_table[1, 0].item() == 40
    x = fresh()
    x.sets[0].block_table[0, 1] = 12
    lla.lla_pages_fork(x.sets[0], x.sets[1], dev([0, 0, 2, 3]))
    flagged(lla.LLA_DEVERR_BLOCK_ID)


def test_wrong_tensors_are_refused(lla):
    x = Both(lla, shapes(lla, "heads"), 10, 2, 4)
    p, slots = x.sets[0], torch.zeros(4, dtype=torch.int64, device=DEV)
    lla.lla_pages_extend(p, list(x.t_pools), slots, x.ws, skip=torch.ones(4, dtype=torch.bool, device=DEV))  # a list, a bool mask
    assert slots.tolist() == [-1] * 4
    with pytest.raises(ValueError, match="int64"):
        lla.lla_pages_extend(p, x.pools, slots.to(I32), x.ws)
    with pytest.raises(ValueError, match="shape"):
        lla.lla_pages_extend(p, x.pools, slots, x.ws, cu_new=dev([0, 1, 2]))
    with pytest.raises(ValueError, match="blocks"):
        lla.lla_pages_extend(lla.Pages(torch.zeros(12, dtype=I32, device=DEV), p.block_table, p.context_lens), x.pools, slots, x.ws)
    with pytest.raises(ValueError, match="CUDA"):
        lla.lla_pages_extend(p, x.pools, slots.cpu(), x.ws)
    with pytest.raises(lla.LLAError, match="LLA_ERR_INVALID_ARG"):
        lla.lla_pages_extend(p, x.pools, slots[:3].contiguous(), x.ws)  # 3 tokens for 4 sequences
    with pytest.raises(lla.LLAError, match="LLA_ERR_WORKSPACE"):
        lla.lla_pages_extend(p, x.pools, slots, x.ws[:64])
    with pytest.raises(lla.LLAError, match="LLA_ERR_INVALID_ARG"):
        lla.lla_pages_fork(p, p, dev([0, 1, 2, 3]))
    with pytest.raises(ValueError, match="shape"):
        lla.lla_pages_fork(p, x.sets[1], dev([0, 1, 2]))
    with pytest.raises(ValueError, match="int32"):
        lla.lla_pages_free(p, dev([0], torch.int64))
    with pytest.raises(ValueError, match="shape"):
        lla.lla_pages_compact(p, x.pools, dev([0] * 9), dev([0]), x.cws)
    x.check(0)


def test_both_marshallings(lla, monkeypatch):
    """The native marshalling and Python's give the same."""
    def calls():
        x = Both(lla, shapes(lla, "heads"), 40, 4, 5, seed=9)
        x.extend(0, [70, 10, 64, 0, 100], skip=[0, 0, 0, 0, 1])
        i = x.fork(0, [0, 0, 1, 2, 0])
        x.extend(i, [1] * 5, packed=False)
        x.free(i, [1, 4])
        x.compact(i)
        return x

    native = []
    real = lla._native()
    for name in ("pages_fork", "pages_extend", "pages_free", "pages_compact"):
        class Spy:
            def __getattr__(self, n):
                def call(*a):
                    st = getattr(real, n)(*a)
                    native.append((n, st))
                    return st
                return call
    monkeypatch.setattr(lla, "_native_module", Spy())
    calls()
    assert {n for n, st in native if st == 0} == {"pages_fork", "pages_extend", "pages_free", "pages_compact"}
    monkeypatch.setattr(lla, "_native_module", lla._Absent())
    calls()


@pytest.mark.parametrize("how", ["stream", "graph"])
def test_another_stream_and_a_captured_graph(lla, how):
    """Two page sets' calls captured together in one graph (their own workspaces), replayed from the same start; and the
    same on a stream that is not the current one."""
    xs = [Both(lla, shapes(lla, "heads"), 50, 4, 6, seed=s) for s in (1, 2)]
    state = []
    for x in xs:
        x.extend(0, [64, 65, 3, 128, 0, 7])
        x.fork(0, [0, 0, 1, 2, 2, 5])
        state.append([t.clone() for t in (x.ref, x.sets[1].block_table, x.sets[1].context_lens)])
    slots = [torch.zeros(6, dtype=torch.int64, device=DEV) for _ in xs]
    parents = dev([0, 1, 1, 1, 4, -1])

    def calls(stream):
        for x, s in zip(xs, slots):
            lla.lla_pages_extend(x.sets[1], x.pools, s, x.ws, stream=stream)
            lla.lla_pages_fork(x.sets[1], x.sets[0], parents, stream=stream)
            lla.lla_pages_compact(x.sets[0], x.pools, x.remap, x.live, x.cws, stream=stream)

    for x in xs:
        x.remap, x.live = torch.zeros(50, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    if how == "stream":
        calls(side)
        side.synchronize()
    else:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            calls(side)
        for _ in range(3):  # each time from the same start
            for x, st in zip(xs, state):
                for t, v in zip((x.ref, x.sets[1].block_table, x.sets[1].context_lens), st):
                    t.copy_(v)
                for p, (a, _, _) in zip(x.t_pools, x.plain[0].pools):
                    p.base.copy_(torch.from_numpy(a))
            g.replay()
            torch.cuda.synchronize()
    for x, s in zip(xs, slots):
        _, want, _ = x.plain[1].extend([1] * 6, [0] * 6)
        assert s.tolist() == [w[0] for w in want]
        x.plain[0].fork(x.plain[1], parents.tolist())
        remap, live = x.plain[0].compact()
        assert x.remap.tolist() == remap and x.live.item() == live
        x.check(0)


def test_blocks_behind_four_gigabytes(lla):
    """Byte offsets that pass 32 bits: a copied and a moved block behind the first 4 GB of a pool."""
    geom = lla.Geometry(4, 16, 128, 192, 320)  # 1 MB a block
    nb = 4300
    pool = torch.zeros(nb, lla.lla_cache_block_bytes(geom), dtype=torch.uint8, device=DEV)
    ref = torch.ones(nb, dtype=I32, device=DEV)
    ref[nb - 1], ref[nb - 2] = 2, 0
    pool[nb - 1] = torch.randint(0, 256, (pool.shape[1],), dtype=torch.uint8, device=DEV)
    table = dev([[nb - 1, -1], [nb - 1, -1]])
    lens = dev([63, 63])
    pages = lla.Pages(ref, table, lens)
    pools = lla.Pools([lla.lla_cache_pool(geom, pool)])
    ws = torch.empty(lla.lla_pages_extend_workspace_size(2), dtype=torch.uint8, device=DEV)
    slots = torch.zeros(2, dtype=torch.int64, device=DEV)
    lla.lla_pages_extend(pages, pools, slots, ws)
    assert slots.tolist() == [(nb - 1) * 64 + 63, (nb - 2) * 64 + 63]
    a, b = (pool[i].view(16, 64 * 512 * 2) for i in (nb - 1, nb - 2))
    k = 64 * 384
    assert torch.equal(a[:, :k].reshape(16, 24, 64, 16)[:, :, :63], b[:, :k].reshape(16, 24, 64, 16)[:, :, :63])
    assert torch.equal(a[:, k:k + 63 * 640], b[:, k:k + 63 * 640]) and not b[:, k + 63 * 640:].any()
    ref[0] = 0
    ref[nb // 2] = 0
    want = [pool[nb - 2].clone(), pool[nb - 1].clone()]
    remap, live = torch.zeros(nb, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    cws = torch.empty(lla.lla_pages_compact_workspace_size(nb), dtype=torch.uint8, device=DEV)
    lla.lla_pages_compact(pages, pools, remap, live, cws)
    assert live.item() == nb - 2 and table[:, 0].tolist() == [nb // 2, 0]
    assert torch.equal(pool[0], want[0]) and torch.equal(pool[nb // 2], want[1])
