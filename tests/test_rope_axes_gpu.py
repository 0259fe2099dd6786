"""lla_encode_rope_keys_axes and lla_decode_attn_decoupled_axes: rotary positions with several axes, against rotations in 64
bits and against the calls with one axis."""
import numpy as np
import pytest
import torch

from helpers import ensure_library, f64
from test_prefix_decode_gpu import Batch, shared

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
BLOCK = 64


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


def axis_of(pairs, order):
    hp = sum(pairs)
    if order == 0:
        return [a for a in range(3) for _ in range(pairs[a])]
    return [j % 3 if j // 3 < pairs[j % 3] else 0 for j in range(hp)]


def turn(x, pos, pairs, order, pairing, base=10000.0):
    """x [N][d] turned at pos [3][N], in 64 bits."""
    hp = x.shape[1] // 2
    z = x[:, 0::2] + 1j * x[:, 1::2] if pairing else x[:, :hp] + 1j * x[:, hp:]
    theta = base ** (-np.arange(hp) / hp)
    z = z * np.exp(1j * pos[axis_of(pairs, order)].T * theta)
    return np.stack([z.real, z.imag], -1).reshape(x.shape) if pairing else np.concatenate([z.real, z.imag], 1)


def stored(planes, nb, d):
    return planes.view(nb, d // 8, BLOCK, 8).permute(0, 2, 1, 3).reshape(nb * BLOCK, d)


# Off by half a step of bf16 (2^-8 of the value) where fp32 turns it exactly; angles are held to 2^-33 turns, 1 - cos and sin to
# 2^-23, and the two products of a pair of size r round to 2^-24 r each: 4e-7 r in all, below which a tie may fall either way.
def assert_turned(got, want, x, pairing):
    hp = x.shape[1] // 2
    r = np.hypot(x[:, 0::2], x[:, 1::2]).repeat(2, 1) if pairing else np.tile(np.hypot(x[:, :hp], x[:, hp:]), 2)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-6 * r).all()


@pytest.mark.parametrize("d, pairs", [(16, (4, 2, 2)), (32, (0, 8, 8)), (48, (24, 0, 0)), (64, (8, 12, 12)), (80, (1, 0, 39)), (96, (16, 16, 16))])
@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_keys(lla, d, pairs, order, pairing, dtype):
    g = torch.Generator().manual_seed(d + order)
    for N in (1, 7, 64, 333):
        nb = N // BLOCK + 3
        k = torch.randn(N, d, generator=g).to(dtype).to(DEV)
        pos = torch.randint(0, 1 << 20, (3, N), generator=g, dtype=I32)
        pos[:, 0] = torch.tensor([0, 2**31 - 1, 5])
        slots = torch.randperm(nb * BLOCK, generator=g)[:N].clone()
        slots[torch.rand(N, generator=g) < 0.1] = -1
        planes = torch.randn(nb, BLOCK * d, generator=g).to(BF16).to(DEV)
        before = f64(stored(planes, nb, d)).copy()
        lla.lla_encode_rope_keys_axes(d, lla.RopeAxes(10000.0, pairing, pairs, order), planes, nb, k, pos.to(DEV), slots.to(DEV))
        after, keep = f64(stored(planes, nb, d)), (slots >= 0).numpy()
        want = turn(f64(k), pos.numpy().astype(np.float64), pairs, order, pairing)
        at = slots.numpy()[keep]
        assert_turned(after[at], want[keep], f64(k)[keep], pairing)
        rest = np.setdiff1d(np.arange(nb * BLOCK), at)
        assert np.array_equal(after[rest], before[rest])  # nothing else is written


@pytest.mark.parametrize("pairing", [0, 1])
def test_one_position_on_all_axes_is_the_call_with_one_axis(lla, pairing):
    N, d, nb = 500, 64, 9
    g = torch.Generator().manual_seed(1)
    k, slots = torch.randn(N, d, generator=g).to(DEV), torch.randperm(nb * BLOCK, generator=g)[:N].to(DEV)
    pos = torch.randint(0, 100000, (N,), generator=g, dtype=I32).to(DEV)
    a, b = torch.zeros(nb, BLOCK * d, dtype=BF16, device=DEV), torch.zeros(nb, BLOCK * d, dtype=BF16, device=DEV)
    lla.lla_encode_rope_keys(d, 10000.0, pairing, a, nb, k, pos, slots)
    lla.lla_encode_rope_keys_axes(d, lla.RopeAxes(10000.0, pairing, (8, 12, 12), 1), b, nb, k, pos.expand(3, N).contiguous(), slots)
    assert torch.equal(a, b)


def test_bad_positions_and_slots_are_flagged(lla):
    rope, d = lla.RopeAxes(10000.0, 0, (4, 2, 2)), 16
    for axis in range(3):
        planes = torch.zeros(2, BLOCK * d, dtype=BF16, device=DEV)
        pos = torch.ones(3, 3, dtype=I32)
        pos[axis, 1] = -1
        lla.lla_encode_rope_keys_axes(d, rope, planes, 2, torch.ones(3, d, device=DEV), pos.to(DEV), torch.tensor([0, 1, 2], device=DEV))
        assert lla.lla_get_device_error() == lla.LLA_DEVERR_CONTEXT
        lla.lla_clear_device_error()
        rows = stored(planes, 2, d).float().abs().sum(1)
        assert rows[0] > 0 and rows[1] == 0 and rows[2] > 0  # the whole token is skipped
    lla.lla_encode_rope_keys_axes(d, rope, planes, 2, torch.ones(3, d, device=DEV), pos.abs().to(DEV), torch.tensor([-1, 128, 2**40], device=DEV))
    assert lla.lla_get_device_error() == lla.LLA_DEVERR_SLOT
    lla.lla_clear_device_error()


def axes_decode(lla, x, pass1, loop=1, ws=None, **kw):
    out = torch.empty(x.B, x.H, 128, dtype=x.io, device=DEV)
    ws = torch.zeros(lla.lla_decode_decoupled_workspace_size(x.geom, x.dr, x.B), dtype=torch.uint8, device=DEV) if ws is None else ws
    lla.lla_decode_attn_decoupled_axes(x.geom, x.codec, x.cache, x.planes, x.dr, x.rope, x.pos, x.lens_t, x.max_ctx, loop, x.q, x.qr,
                                       *((x.ck, x.cv, x.ckr) if pass1 else (None, None, None)), out, ws, **kw)
    return out


@pytest.mark.parametrize("d_rope", [32, 64, 96])
@pytest.mark.parametrize("io, pass1", [(F32, True), (F32, False), (BF16, True), (BF16, False)])
def test_decode(lla, d_rope, io, pass1):
    rows, lens = shared(5, 2, 6, 200, seed=d_rope)
    x = Batch(lla, rows, [max(1, n) for n in lens], d_rope=d_rope, io=io, mu=True, garbage=True, H=4)
    x.check(axes_decode(lla, x, pass1), pass1=pass1)


def test_decode_at_the_index_is_the_call_without_axes(lla):
    x = Batch(lla, *shared(3, 2, 9, 100), d_rope=64, H=16)
    x.pos = x.lens_t.expand(3, x.B).contiguous()
    out, want = axes_decode(lla, x, True), torch.empty(x.B, x.H, 128, device=DEV)
    ws = torch.zeros(lla.lla_decode_decoupled_workspace_size(x.geom, 64, x.B), dtype=torch.uint8, device=DEV)
    lla.lla_decode_attn_decoupled(x.geom, x.codec, x.cache, x.planes, 64, 10000.0, 0, x.lens_t, x.max_ctx, 1, x.q, x.qr, x.ck, x.cv, x.ckr, want, ws)
    assert torch.equal(out, want)


def test_a_negative_position_is_flagged(lla):
    x = Batch(lla, *shared(1, 4, 2, 100), d_rope=32, H=2)
    x.pos[2, 1] = -1
    out = axes_decode(lla, x, True)
    assert lla.lla_get_device_error() == lla.LLA_DEVERR_CONTEXT
    lla.lla_clear_device_error()
    x.pos[2, 1] = 0
    assert torch.equal(out, axes_decode(lla, x, True))


def test_captured(lla):
    x = Batch(lla, *shared(2, 3, 4, 100), d_rope=64, H=4)
    want = axes_decode(lla, x, True)
    ws = torch.zeros(lla.lla_decode_decoupled_workspace_size(x.geom, 64, x.B), dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = axes_decode(lla, x, True, ws=ws)
    for _ in range(3):
        g.replay()
    assert torch.equal(out, want)
