"""lla_decode_attn_prefix where the trunk kernel runs, which takes batches of more than four sequences: every class of group sizes
(up to 16, 32 and 64 queries), one unit over all CTAs, and trunk kernels on several streams."""
import pytest
import torch

from helpers import ensure_library
from test_prefix_decode_gpu import Batch, shared

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


@pytest.mark.parametrize("W", [5, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("d_rope", [0, 32, 96])
def test_maxima_that_grow_late(lla, W, d_rope):
    """Scores that rise along the pages, so that what has been summed is scaled again and again.  (Content scores up to 32 times as
    large as those of the tolerance 2e-4: ten times it at least.)"""
    x = Batch(lla, *shared(1, W, 12, 90, seed=W), H=2, sigma=0.5, seed=W, d_rope=d_rope)
    for i, b in enumerate(x.table[0][:12].tolist()):
        x.pool[b] *= 2.0 ** (i / 2 - 1)
    x.check(x.decode(), tol=2e-3)


@pytest.mark.parametrize("W", [5, 20, 64])
@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("pages", [151, 900])
def test_one_unit_over_all_ctas(lla, W, io, pages):
    """One head: a page or a few of one unit in each CTA, in a run of its own."""
    x = Batch(lla, *shared(1, W, pages, 64, seed=W), H=1, io=io)
    x.check(x.decode(), pairs=[(b, 0) for b in range(0, W, 7)])


def test_three_streams_at_once(lla):
    """Calls on three streams, each with its own workspace and a trunk kernel, in any overlap of their kernels."""
    xs = [Batch(lla, *shared(4, 12, 30, 2000, seed=1), H=8), Batch(lla, *shared(1, 6, 40, 900, seed=2), H=8, d_rope=64),
          Batch(lla, *shared(2, 40, 25, 64, seed=3), H=8, io=BF16)]
    want = [x.decode() for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                outs.append(x.decode())
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, want[i % len(xs)])
