"""The page calls at the ends of their ranges: slot mappings of 2^31 - 1 tokens, ledgers of up to 2^24 blocks."""
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


def test_the_longest_slot_mapping(lla):
    """A mapping of 2^31 - 1 slots (17 GB), padded behind 70 tokens: the index of the last step over it does not fit 32 bits."""
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    N, S, nb = 2 ** 31 - 1, 3, 8
    pages = lla.Pages(torch.zeros(nb, dtype=I32, device=DEV), torch.full((S, 4), -7, dtype=I32, device=DEV), torch.zeros(S, dtype=I32, device=DEV))
    room = 1 << 20  # words in front of the mapping and behind it
    flat = torch.full((N + 2 * room,), 12345, dtype=torch.int64, device=DEV)
    slots = flat[room:room + N]
    ws = torch.empty(lla.lla_pages_extend_workspace_size(S), dtype=torch.uint8, device=DEV)
    cu = torch.tensor([0, 3, 68, 70], dtype=I32, device=DEV)
    lla.lla_pages_extend(pages, lla.Pools(), slots, ws, cu_new=cu)
    want = list(range(3)) + list(range(64, 129)) + list(range(192, 194))
    assert slots[:70].tolist() == want
    assert [int(x) for x in torch.aminmax(slots[70:])] == [-1, -1]
    for guard in (flat[:room], flat[room + N:]):
        assert [int(x) for x in torch.aminmax(guard)] == [12345, 12345]
    assert pages.context_lens.tolist() == [3, 65, 2]
    assert lla.lla_get_device_error() == 0
    # the same number for each of one sequence: refused on the device (2^31 - 1 tokens do not fit its row), every slot -1
    one = lla.Pages(pages.ref_count, pages.block_table[:1], pages.context_lens[:1])
    lla.lla_pages_extend(one, lla.Pools(), slots, ws)
    assert [int(x) for x in torch.aminmax(slots)] == [-1, -1]
    assert one.context_lens.tolist() == [3]
    assert lla.lla_get_device_error() == lla.LLA_DEVERR_CONTEXT
    lla.lla_clear_device_error()


@pytest.mark.parametrize("length", [-1, 257, -2 ** 31, 2 ** 31 - 1])
def test_fork_reports_a_length_out_of_range_that_no_child_has(lla, length):
    """Its pages cannot be given back, so the call says so, as lla_pages_free does; the others' are."""
    i = lambda *v: torch.tensor(v, dtype=I32, device=DEV)
    ref = i(1, 2, 1, 1)
    a = lla.Pages(ref, torch.tensor([[0, 1, -7, -7], [1, 2, 3, -7]], dtype=I32, device=DEV), i(100, length))
    b = lla.Pages(ref, torch.full((3, 4), -7, dtype=I32, device=DEV), i(9, 9, 9))
    lla.lla_pages_fork(a, b, i(0, -1, 0))
    assert lla.lla_get_device_error() == lla.LLA_DEVERR_CONTEXT
    lla.lla_clear_device_error()
    assert b.context_lens.tolist() == [100, 0, 100] and b.block_table.tolist() == [[0, 1, -7, -7], [-7] * 4, [0, 1, -7, -7]]
    assert ref.tolist() == [2, 3, 1, 1]


class Ledger:
    """A ledger of nb blocks with random counts 0 to 3, kept by one long and many short sequences."""

    def __init__(self, lla, nb, S, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lla, self.nb, self.S = lla, nb, S
        live = torch.rand(nb, generator=g, device=DEV) < 0.6
        held = torch.nonzero(live).view(-1).to(I32)
        held = held[torch.randperm(len(held), generator=g, device=DEV)]
        # sequence 0 has half of the blocks in use; the others split the rest, and the last holds the first's first 1000 too
        half = len(held) // 2
        cuts = [0, half] + [half + (len(held) - half) * (i + 1) // (S - 2) for i in range(S - 2)]
        rows = [held[a:b] for a, b in zip(cuts, cuts[1:])] + [held[:1000]]
        self.mb = max(len(r) for r in rows) + 8
        table = torch.full((S, self.mb), -7, dtype=I32, device=DEV)
        lens = []
        for s, r in enumerate(rows):
            table[s, :len(r)] = r
            lens.append(len(r) * 64 - (17 * s % 64 if s not in (0, S - 1) else 0))
        self.pages = lla.Pages(torch.zeros(nb, dtype=I32, device=DEV), table, torch.tensor(lens, dtype=I32, device=DEV))
        self.pages.ref_count.copy_(self.counts(self.pages))

    def counts(self, pages):
        n = (pages.context_lens.long() + 63) // 64
        at = torch.arange(self.mb, device=DEV)[None, :] < n[:, None]
        return torch.bincount(pages.block_table[at].long(), minlength=self.nb).to(I32)


@pytest.mark.parametrize("nb", [8192, 8193, 1 << 20, (1 << 24) - 5, 1 << 24])
def test_ledgers_of_every_size(lla, nb):
    """Growth, fork, freeing and compaction over ledgers of up to 2^24 blocks, against torch's own counting and ranking."""
    S = 9
    x = Ledger(lla, nb, S, nb)
    p = x.pages
    pool = torch.arange(nb, dtype=I32, device=DEV).view(nb, 1).repeat(1, 64)  # a plane of 4-byte rows: block b is full of b
    pools = lla.Pools([lla.Pool(pool, 1, 4, 0)])
    # growth: a token each, one sequence 130, one nothing
    n = [1, 130, 0] + [1] * (S - 3)
    before, ref, table = p.context_lens.clone(), p.ref_count.clone(), p.block_table.clone()
    cu = torch.tensor([0] + n, dtype=I32, device=DEV).cumsum(0).to(I32)
    slots = torch.zeros(sum(n), dtype=torch.int64, device=DEV)
    free = torch.zeros(1, dtype=I32, device=DEV)
    ws = torch.full((lla.lla_pages_extend_workspace_size(S),), 0xA5, dtype=torch.uint8, device=DEV)
    lla.lla_pages_extend(p, pools, slots, ws, cu_new=cu, free_blocks=free)
    lens = before.tolist()
    new = [-(-(a + b) // 64) - -(-a // 64) for a, b in zip(lens, n)]
    ranks = torch.nonzero(ref == 0).view(-1)
    assert free.item() == len(ranks) - sum(new)
    got = [int(p.block_table[s, -(-lens[s] // 64) + i]) for s in range(S) for i in range(new[s])]
    assert got == ranks[:sum(new)].tolist()
    assert p.context_lens.tolist() == [a + b for a, b in zip(lens, n)]
    want = [int(p.block_table[s, q // 64]) * 64 + q % 64 for s in range(S) for q in range(lens[s], lens[s] + n[s])]
    assert slots.tolist() == want
    for s in range(S):
        had = -(-lens[s] // 64)
        assert torch.equal(p.block_table[s, :had], table[s, :had])
    assert torch.equal(p.ref_count, x.counts(p))
    # fork: the long sequence twice, one dropped, one empty
    parents = [0, 0, -1] + list(range(3, S))
    to = lla.Pages(p.ref_count, torch.full((S, x.mb), -9, dtype=I32, device=DEV), torch.full((S,), 5, dtype=I32, device=DEV))
    lla.lla_pages_fork(p, to, torch.tensor(parents, dtype=I32, device=DEV))
    assert to.context_lens.tolist() == [p.context_lens[q].item() if q >= 0 else 0 for q in parents]
    for s, q in enumerate(parents):
        had = -(-to.context_lens[s].item() // 64)
        assert torch.equal(to.block_table[s, :had], p.block_table[q, :had]) and (to.block_table[s, had:] == -9).all()
    assert torch.equal(p.ref_count, x.counts(to))
    # freeing one of the long one's two holders, and a short one
    lla.lla_pages_free(to, torch.tensor([1, 4, -1, 4], dtype=I32, device=DEV))
    assert torch.equal(p.ref_count, x.counts(to))
    # compaction
    ref, table = to.ref_count.clone(), to.block_table.clone()
    remap, live = torch.full((nb,), 99, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    cws = torch.full((lla.lla_pages_compact_workspace_size(nb),), 0xA5, dtype=torch.uint8, device=DEV)
    lla.lla_pages_compact(to, pools, remap, live, cws)
    R = int((ref != 0).sum())
    ids = torch.arange(nb, device=DEV, dtype=I32)
    want = torch.where(ref != 0, ids, -1)
    holes, movers = torch.nonzero(ref[:R] == 0).view(-1), torch.nonzero(ref[R:] != 0).view(-1) + R
    want[movers] = holes.to(I32)
    assert live.item() == R and torch.equal(remap, want)
    assert (to.ref_count[:R] != 0).all() and (to.ref_count[R:] == 0).all() and torch.equal(to.ref_count, x.counts(to))
    for s in range(S):
        had = -(-to.context_lens[s].item() // 64)
        assert torch.equal(to.block_table[s, :had], want[table[s, :had].long()]) and torch.equal(to.block_table[s, had:], table[s, had:])
    assert torch.equal(pool[holes], movers.to(I32).view(-1, 1).expand(-1, 64))
    untouched = torch.ones(nb, dtype=torch.bool, device=DEV)
    untouched[holes] = False
    assert torch.equal(pool[untouched], ids[untouched].view(-1, 1).expand(-1, 64))
    assert lla.lla_get_device_error() == 0
