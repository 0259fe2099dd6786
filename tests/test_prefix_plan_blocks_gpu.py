"""lla_prefix_plan where tables hold entries that are no blocks: pages are shared up to such an entry, wherever it lies, and it is
flagged where it is the next page of a group."""
import pytest
import torch

from helpers import ensure_library
from test_prefix_plan_gpu import BLOCK, dev, plain

pytestmark = pytest.mark.gpu

NB = 1 << 16


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    m.lla_clear_device_error()
    return m


def run(lla, rows, lens, min_pages=1):
    """The plan, what it has to be (pages end before the first entry that is no block) and the error word."""
    plan = lla.Prefix.empty(len(lens))
    lla.lla_prefix_plan(lla.Cache(None, NB, dev(rows), len(rows[0])), dev(lens), len(rows[0]) * BLOCK, plan, min_pages=min_pages)
    word = lla.lla_get_device_error()
    lla.lla_clear_device_error()
    cut = [min([n] + [p * BLOCK for p in range(n // BLOCK) if not 0 <= r[p] < NB]) for r, n in zip(rows, lens)]
    return plan, plain(rows, cut, min_pages), word


def check(plan, want):
    groups, members, column, own = want
    assert plan.num_groups.item() == len(groups)
    assert plan.groups.tolist()[:len(groups)] == [list(g) for g in groups]
    assert plan.members.tolist()[:len(members)] == members
    assert plan.column.tolist() == column
    assert plan.own_page.tolist() == own


@pytest.mark.parametrize("bad", [-1, NB, 2**31 - 1, -2**31])
@pytest.mark.parametrize("B", [2, 65])
@pytest.mark.parametrize("at", [1, 2, 31, 32, 33, 255, 257, 511, 513])
def test_in_the_middle_of_shared_pages(lla, bad, B, at):
    n = 600
    row = list(range(n))
    row[at] = bad
    plan, want, word = run(lla, [row] * B, [n * BLOCK] * B)
    check(plan, want)
    assert plan.own_page.tolist() == [at] * B and word == lla.LLA_DEVERR_BLOCK_ID


def test_on_the_last_level_and_with_least_pages(lla):
    # page 0 of all, pages 1 and 2 of halves, page 3 of pairs, then an entry that is no block
    rows = [[1, 10 + s // 4, 20 + s // 4, 30 + s // 2, -1, 50 + s // 2] for s in range(8)]
    plan, want, word = run(lla, rows, [6 * BLOCK] * 8)
    check(plan, want)
    assert plan.own_page.tolist() == [4] * 8 and word == lla.LLA_DEVERR_BLOCK_ID
    plan, want, word = run(lla, [[1, 2, NB, 4]] * 3, [4 * BLOCK] * 3, min_pages=3)
    check(plan, want)
    assert plan.num_groups.item() == 0 and word == 0  # no group ends there: the decode flags it


def test_what_nobody_shares_is_left_to_the_decode(lla):
    """Entries that differ, behind a length, or in a page that is not full."""
    rows = [[1, 2, -1, 9], [1, 2, 3, 9], [1, 2, 5, NB]]
    plan, want, word = run(lla, rows, [2 * BLOCK, 4 * BLOCK, 2 * BLOCK + 63])
    check(plan, want)
    assert plan.own_page.tolist() == [2] * 3 and word == 0
