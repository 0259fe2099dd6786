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
