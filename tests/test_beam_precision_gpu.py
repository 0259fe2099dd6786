"""How far lla_beam_select's scores are from their definition in 64 bits, at the bound that its formula gives.

A term 2^(z K - c), K = log2 e in fp32, c a whole number, takes one rounding of its exponent, of at most 2^-24 of |z - b| in
log S, b = c / K; K is off by less than 2^-26 of itself, which counts with |z - b| too; ex2.approx is off by 2^-22 of its result.  b is
the largest logit that the thread or its CTA had seen when it was set, to within 0.35 (c is whole), and a thread sets it anew
where a logit is 5 above that: so -0.35 - (largest - z) <= z - b <= 5.35.  A tile's terms are summed as a tree of five levels at
most, 2^-24 each, or logit by logit with ten roundings where some are not finite; what comes behind carries its errors along; the
logarithm is off by 4e-9.  Moving a sum to another b is exact,
or beyond +-65536, where terms are 2^((z - b) K) with a logit b (and are summed one by one), costs 2^-22 for another ex2, 2^-23 for its
factor, and 2^-24 of the distance moved, which is at most 2 d in all: the thread's own move, to its CTA's b, to the row's.  Weights are those of the softmax.

Scores are given so that results are near zero, where an fp32 output has no rounding of its own to speak of."""
import math

import numpy as np
import pytest
import torch

from helpers import ensure_library, f64

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
TREE, ONE_BY_ONE = 5 * 2.0 ** -24, 10 * 2.0 ** -24
EX2 = 2.0 ** -22


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    m.lla_clear_device_error()
    return m


def log_sum(x, tree=TREE, moves=0):
    """log sum exp of finite logits in 64 bits, and how far the kernel's may be off."""
    top = x.max()
    p = np.exp(x - top)
    S = math.fsum(p)
    d = float((p / S * np.maximum(5.0, top - x)).sum()) + 0.35
    return top + math.log(S), (1 + 1.5 * moves) * EX2 + tree + (1.25 + (2 if moves else 0)) * 2.0 ** -24 * d + 4e-9


def best_score(lla, z, score):
    """The score of each beam's best continuation (a sequence of one beam each)."""
    B, W, V = z.shape
    assert W == 1
    parents, tokens, out = torch.zeros(B, 1, dtype=I32, device=DEV), torch.zeros(B, 1, dtype=I32, device=DEV), torch.zeros(B, 1, device=DEV)
    ws = torch.empty(lla.lla_beam_select_workspace_size(B, 1, V, 1, z.dtype), dtype=torch.uint8, device=DEV)
    lla.lla_beam_select(z, score.view(B, 1), parents, tokens, out, ws)
    assert (parents.view(-1) == torch.arange(B, device=DEV)).all()
    return f64(out)[:, 0], tokens.view(-1).tolist()


def check(lla, z, *how):
    """Every row of z [B][1][V], with the beam's score set to what brings the result near zero."""
    x = f64(z)[:, 0]
    fin = [r[np.isfinite(r)] for r in x]
    want = [log_sum(r, *how) for r in fin]
    lift = np.array([np.float32(L - r.max()) for (L, _), r in zip(want, fin)], dtype=np.float32)
    got, _ = best_score(lla, z, torch.from_numpy(lift).to(DEV))
    for b, ((L, bound), r) in enumerate(zip(want, fin)):
        exact = float(lift[b]) + (r.max() - L)
        assert abs(got[b] - exact) <= bound + abs(exact) * 2.0 ** -24, (b, got[b], exact, bound)


def noise(seed, B, V, dtype, scale):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(B, 1, V, generator=g, device=DEV) * scale).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,V", [(3, 70000), (3, 1 << 20), (640, 20000)])  # many shares a row, one CTA a row
@pytest.mark.parametrize("scale", [0.5, 2.5, 8.0])
def test_noise(lla, dtype, B, V, scale):
    z = noise(V + B, B, V, dtype, scale)
    check(lla, z) if B <= 40 else check_some(lla, z)


def check_some(lla, z, *how):
    """All rows at once (so that a CTA has a whole one), 40 of them compared."""
    x = f64(z[::16])[:, 0]
    want = [log_sum(r[np.isfinite(r)], *how) for r in x]
    tops = [r[np.isfinite(r)].max() for r in x]
    lift = torch.zeros(len(z), device=DEV)
    lift[::16] = torch.tensor([L - t for (L, _), t in zip(want, tops)], dtype=torch.float64).float().to(DEV)
    got, _ = best_score(lla, z, lift)
    lift = f64(lift)
    for i, ((L, bound), top) in enumerate(zip(want, tops)):
        exact = lift[16 * i] + (top - L)
        assert abs(got[16 * i] - exact) <= bound + abs(exact) * 2.0 ** -24, (i, got[16 * i], exact, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shares", ["one", "many"])
def test_one_logit_far_above_the_first_tile(lla, dtype, shares):
    """A dominating logit 1 to 64 above everything that came before it, at the end of the row."""
    rise = torch.linspace(1, 64, 640 if shares == "one" else 12, device=DEV)
    z = noise(7, len(rise), 50000 if shares == "one" else 70000, dtype, 0.1)
    z[:, 0, -5] = rise.to(dtype)
    z[:, 0, -6] = (rise / 2).to(dtype)
    check_some(lla, z) if shares == "one" else check(lla, z)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rising_rows(lla, dtype):
    """Rows that rise by 5 to 80 from end to end: the base moves many times."""
    V = 200000
    z = noise(9, 640, V, dtype, 0.3)
    z += (torch.linspace(0, 1, V, device=DEV) * torch.linspace(5, 80, 640, device=DEV)[:, None, None]).to(dtype)
    check_some(lla, z)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_that_are_not_finite_in_every_tile(lla, dtype):
    """NaN and infinities lead past the usual sums, logit by logit: no less exact."""
    z = noise(11, 640, 60000, dtype, 1.0)
    ramp = torch.arange(60000, device=DEV)
    z[:, :, ramp % 13 == 4] = math.nan
    z[::2, :, ramp % 29 == 5] = math.inf
    z[:, :, ramp % 31 == 6] = -math.inf
    check_some(lla, z, ONE_BY_ONE)


@pytest.mark.parametrize("value", [1.4140625, -7.6875, 0.8203125])
def test_long_rows_of_equal_logits(lla, value):
    """Rows of 2^22 equal logits, one CTA each (512 tiles): a tile's tree is exact then, so log S is off by the exponent's
    and ex2's rounding alone, unless sums lose theirs from tile to tile."""
    rows, V = 608, 1 << 22
    if torch.cuda.mem_get_info()[0] < 20e9:
        pytest.skip("needs 20 GB")
    z = torch.full((rows, 1, V), value, dtype=BF16, device=DEV)
    lift = torch.full((rows,), math.log(V), device=DEV)
    got, _ = best_score(lla, z, lift)
    exact = float(f64(lift)[0]) - math.log(V)
    bound = EX2 + 1.25 * 2.0 ** -24 * 0.35 + 4e-9
    assert np.abs(got - exact).max() <= bound + abs(exact) * 2.0 ** -24, (got[0], exact, bound)


@pytest.mark.parametrize("shares", ["one", "many"])
@pytest.mark.parametrize("at", [65536.0, -65536.0])
def test_logits_on_both_sides_of_the_wide_base(lla, at, shares):
    """fp32 logits around +-65536, where terms change their form: tiles of a row, and threads of a tile, on either side."""
    B, V = (640, 40000) if shares == "one" else (12, 90000)
    g = torch.Generator(device=DEV).manual_seed(13)
    step = 2.0 ** -7
    z = at + torch.round(torch.randn(B, 1, V, generator=g, device=DEV) * 0.7 / step) * step
    # rows by kind: as they are; the first half 3 below; the second half 3 below; one logit far over; one side only
    z[1::5, :, :V // 2] -= 3
    z[2::5, :, V // 2:] -= 3
    z[3::5, :, V - 7] = at + 9
    z[4::5] = torch.where(z[4::5] > at, at - (z[4::5] - at), z[4::5])
    if shares == "one":
        check_some(lla, z, ONE_BY_ONE, 3)
    else:
        check(lla, z, ONE_BY_ONE, 3)


def test_a_beam_s_score_whatever_the_batch(lla):
    """The same row alone (cut into shares) and among many (not cut): equal within twice the bound."""
    V = 100000
    z = noise(17, 700, V, BF16, 2.5)
    _, bound = log_sum(f64(z[:1])[0, 0])
    lift = torch.zeros(700, device=DEV)
    L, _ = log_sum(f64(z[:1])[0, 0])
    lift[0] = L - float(z[0, 0].max())
    many, _ = best_score(lla, z, lift)
    alone, _ = best_score(lla, z[:1].contiguous(), lift[:1].contiguous())
    assert abs(many[0] - alone[0]) <= 2 * bound + 2.0 ** -24 * 1e-6
