"""lla_decode_attn_prefix for up to five sequences, whose path depends on their number and on the longest context that the call
allows: the same results on both sides of every border."""
import pytest
import torch

from helpers import ensure_library
from test_prefix_decode_gpu import BLOCK, DEV, Batch, shared

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


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


def allow(x, tokens):
    """A block table that is wide enough for contexts of `tokens`, and the call's longest context."""
    wide = torch.full((x.B, -(-tokens // BLOCK)), -1, dtype=torch.int32)
    wide[:, :x.table.shape[1]] = x.table
    x.cache = x.lla.Cache(x.pool, x.nb, wide.to(DEV), wide.shape[1])
    x.max_ctx = tokens
    x.replan()


@pytest.mark.parametrize("B", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("rk, rv, d_rope, io", [(96, 160, 0, F32), (96, 160, 0, BF16), (128, 128, 0, F32), (72, 120, 0, F32), (96, 160, 64, F32)])
def test_short_sequences_in_wide_tables(lla, B, rk, rv, d_rope, io):
    x = Batch(lla, *shared(1, B, 6, 100, system=1, branch=2, seed=B), H=5, rk=rk, rv=rv, d_rope=d_rope, io=io, mu=True, garbage=True)
    for tokens in (8192, 16384, 16385, 1 << 20):
        allow(x, tokens)
        for pass1 in (True, False):
            x.check(x.decode(pass1=pass1), pass1=pass1, pairs=[(b, h) for b in range(B) for h in (0, 4)])


@pytest.mark.parametrize("B", [3, 4])
@pytest.mark.parametrize("pages", [255, 256, 257, 700])
def test_long_sequences(lla, B, pages):
    x = Batch(lla, *shared(1, B, pages - 2, 128, branch=1, seed=B), H=2)
    x.check(x.decode(), pairs=[(b, h) for b in range(B) for h in range(2)])
