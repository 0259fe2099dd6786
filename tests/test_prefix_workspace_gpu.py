"""The workspace of lla_decode_attn_prefix: as large as what its kernels write, and no larger than the path of the batch needs."""
import pytest
import torch

from helpers import ensure_library
from test_prefix_decode_gpu import Batch, shared

pytestmark = pytest.mark.gpu

DEV = "cuda"
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


@pytest.mark.parametrize("rk, rv, d_rope", [(96, 160, 0), (128, 128, 0), (72, 120, 0), (96, 160, 96)])
def test_sizes(lla, rk, rv, d_rope):
    """Records of r_v + 4 floats: one per sequence, head and node of it, and one more for each query of a share that starts inside a
    unit (up to three shares a warp, nine warps an SM; up to 64 queries an SM beside them where there is a trunk), and q~ in ten bytes a
    value.  Up to four sequences have no trunk."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    geom = lla.Geometry(4, 16, 128, rk, rv)
    for B in (0, 1, 2, 4, 5, 64, 128, 1024):
        records = 4 * 16 * B + 3 * 9 * sms * (max(B, 1) if B <= 4 else 2) + (3 * 16 * B + min(B, 64) * sms if B > 4 else 0)
        most = records * (rv + 4) * 4 + 16 * B * ((rk + 15) // 16 * 16 + d_rope) * 10 + (1 << 17)
        assert lla.lla_decode_prefix_workspace_size(geom, B, d_rope) <= most, B


@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("B", [1, 2, 3, 4, 5, 9, 64, 130])
def test_nothing_is_written_behind_it(lla, B, io):
    """Few and many pages a warp, groups of all sizes: bytes behind the workspace stay, and so do the results."""
    for prompt, own, H in ((1, 64, 16), (40, 900, 16), (900, 3000, 1)):
        x = Batch(lla, *shared(1, B, prompt, own, seed=B), H=H, io=io)
        n = x.ws.numel()
        room = torch.full((n + (1 << 20),), 0x5A, dtype=torch.uint8, device=DEV)
        want = x.decode()
        x.ws = room[:n]
        assert torch.equal(x.decode(), want)
        assert (room[n:] == 0x5A).all()
        x.check(want, pairs=[(b, 0) for b in range(0, B, 17)])
