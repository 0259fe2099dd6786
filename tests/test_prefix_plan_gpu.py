"""lla_prefix_plan against the documented partition, set by set in Python."""
import random

import pytest
import torch

from helpers import ensure_library

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32 = torch.int32
BLOCK, LEVELS, MEMBERS = 64, 3, 64


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


def dev(v, t=I32):
    return torch.tensor(v, dtype=t, device=DEV)


def plain(rows, lens, min_pages=1):
    """(groups, members, column, own_page) of the sequences with table rows `rows` (lists) and lengths `lens`."""
    B = len(lens)
    full = [n // BLOCK for n in lens]
    groups, members, column, own = [], [], [[-1] * B for _ in range(LEVELS)], [0] * B
    sets = [(0, list(range(B)))]
    for level in range(LEVELS):
        found = []
        for page, who in sets:
            by = {}
            for s in who:
                if full[s] > page:
                    by.setdefault(rows[s][page], []).append(s)
            for mine in by.values():
                if len(mine) < 2:
                    continue
                end = page + 1
                while all(full[s] > end for s in mine) and len({rows[s][end] for s in mine}) == 1:
                    end += 1
                if end - page >= min_pages:
                    found.append((page, end, mine))
        found.sort(key=lambda x: x[2][0])
        for page, end, mine in found:
            parts = -(-len(mine) // MEMBERS)
            for i in range(parts):
                part = mine[i * len(mine) // parts:(i + 1) * len(mine) // parts]
                for r, s in enumerate(part):
                    column[level][s] = len(groups) * MEMBERS + r
                groups.append((page, end, len(members), len(part)))
                members += part
            for s in mine:
                own[s] = end
        sets = [(end, mine) for _, end, mine in found]
    return groups, members, column, own


def check(lla, rows, lens, min_pages=1, nb=1 << 20, mb=None, spare=0, **kw):
    B = len(lens)
    mb = mb or max([1] + [len(r) for r in rows]) + spare
    table = torch.full((B, mb), -1, dtype=I32)
    for s, r in enumerate(rows):
        table[s, :len(r)] = torch.tensor(r, dtype=I32)
    plan = lla.Prefix.empty(B)
    for t in (plan.num_groups, plan.groups, plan.members, plan.column, plan.own_page):
        t.fill_(77)
    lla.lla_prefix_plan(lla.Cache(None, nb, table.to(DEV), mb), dev(lens), mb * BLOCK, plan, min_pages=min_pages, **kw)
    groups, members, column, own = plain(rows, lens, min_pages)
    assert plan.num_groups.item() == len(groups)
    rest = plan.groups.shape[0] - len(groups)
    assert plan.groups.tolist() == [list(g) for g in groups] + [[0] * 4] * rest
    assert plan.members.tolist() == members + [-1] * (LEVELS * B - len(members))
    assert plan.column.tolist() == column
    assert plan.own_page.tolist() == own
    return groups


def tree(r, B, pages, fan):
    """Rows that share ever less: a batch forked again and again, in a random order."""
    nxt = [0]

    def grow(row, n):
        row = row + list(range(nxt[0], nxt[0] + n))
        nxt[0] += n
        return row

    rows = [grow([], r.randint(0, pages))]
    while len(rows) < B:
        i = r.randrange(len(rows))
        base = rows[i]
        rows[i] = grow(base, r.randint(0, pages))
        rows += [grow(base, r.randint(0, pages)) for _ in range(r.randint(1, fan))]
    rows = rows[:B]
    r.shuffle(rows)
    return rows, [max(0, len(x) * BLOCK - (r.randint(0, 63) if r.random() < 0.7 else 0)) for x in rows]


@pytest.mark.parametrize("B, pages, fan", [(2, 3, 1), (5, 4, 2), (33, 9, 40), (64, 40, 8), (65, 3, 70), (129, 300, 130), (700, 20, 9), (1024, 12, 300)])
@pytest.mark.parametrize("min_pages", [1, 3])
def test_forked_batches(lla, B, pages, fan, min_pages):
    for seed in range(3):
        rows, lens = tree(random.Random(seed * 1000 + B), B, pages, fan)
        check(lla, rows, lens, min_pages, spare=seed)


def test_any_table(lla):
    """Tables that no fork makes: the same block at different pages, twice in a row, rows that meet again."""
    for seed in range(20):
        r = random.Random(seed)
        B = r.randint(1, 40)
        rows = [[r.randint(0, 2) for _ in range(r.randint(0, 7))] for _ in range(B)]
        check(lla, rows, [max(0, len(x) * BLOCK - r.choice([0, 0, 1, 63])) for x in rows], nb=3, spare=r.randint(0, 2))


@pytest.mark.parametrize("B", [1, 64, 65, 128, 129, 1000, 1024])
def test_one_prompt_for_all(lla, B):
    groups = check(lla, [list(range(70)) + [100 + s] for s in range(B)], [70 * BLOCK + 1] * B)
    assert len(groups) == (0 if B == 1 else -(-B // MEMBERS))


def test_long_rows_differ_at_every_distance(lla):
    """The first difference lies before, in and behind each step of the comparison."""
    n = 600
    for at in (1, 31, 32, 33, 255, 256, 257, 288, 511, 513, 599):
        check(lla, [list(range(n)), list(range(at)) + list(range(1000, 1000 + n - at))], [n * BLOCK] * 2)


def test_short_and_empty_sequences(lla):
    check(lla, [[5], [5], [5, 6], []], [64, 63, 65, 0])          # 63 tokens have no full page
    check(lla, [[], [], []], [0, 0, 0])
    check(lla, [[5, 6, 7], [5, 6, 8], [5, 9]], [192, 191, 66])


def test_no_batch(lla):
    plan = lla.Prefix.empty(0)
    plan.num_groups.fill_(9)
    lla.lla_prefix_plan(lla.Cache(None, 4, torch.zeros(1, 1, dtype=I32, device=DEV), 1), torch.zeros(0, dtype=I32, device=DEV), 64, plan)
    assert plan.num_groups.item() == 0


def test_bad_lengths_and_blocks_are_flagged(lla):
    def word(rows, lens, mb, nb=100, max_ctx=None):
        plan = lla.Prefix.empty(len(lens))
        lla.lla_prefix_plan(lla.Cache(None, nb, dev(rows), mb), dev(lens), max_ctx or mb * BLOCK, plan)
        w = lla.lla_get_device_error()
        lla.lla_clear_device_error()
        return w, plan

    rows = [[1, 2], [1, 2], [1, 2]]
    w, plan = word(rows, [128, 129, 128], 2)
    assert w == lla.LLA_DEVERR_CONTEXT and plan.own_page.tolist() == [2, 0, 2] and plan.members.tolist()[:3] == [0, 2, -1]
    w, plan = word(rows, [128, -1, 128], 2)
    assert w == lla.LLA_DEVERR_CONTEXT and plan.column.tolist()[0] == [0, -1, 1]
    w, plan = word(rows, [128, 100, 100], 2, max_ctx=100)
    assert w == lla.LLA_DEVERR_CONTEXT and plan.own_page.tolist() == [0, 1, 1]
    for bad in (-1, 100, 2**31 - 1):
        w, plan = word([[bad, 2], [bad, 2], [1, 2]], [128] * 3, 2)
        assert w == lla.LLA_DEVERR_BLOCK_ID and plan.num_groups.item() == 0 and plan.own_page.tolist() == [0] * 3


def test_captured_and_on_another_stream(lla):
    rows, lens = tree(random.Random(5), 40, 6, 5)
    mb = max(len(r) for r in rows)
    table = torch.full((40, mb), -1, dtype=I32)
    for s, r in enumerate(rows):
        table[s, :len(r)] = torch.tensor(r, dtype=I32)
    cache, lens_t, plan = lla.Cache(None, 1 << 20, table.to(DEV), mb), dev(lens), lla.Prefix.empty(40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lla.lla_prefix_plan(cache, lens_t, mb * BLOCK, plan, stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lla.lla_prefix_plan(cache, lens_t, mb * BLOCK, plan)
    other = [max(0, n - 70) for n in lens]
    lens_t.copy_(dev(other))
    g.replay()
    groups, members, column, own = plain(rows, other)
    assert plan.num_groups.item() == len(groups) and plan.column.tolist() == column and plan.own_page.tolist() == own
