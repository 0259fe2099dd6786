"""lla_decode_attn_prefix over long shared parts: the error of a sum does not grow with the pages that it goes over.

The rows repeat eight blocks of unit keys and positive values, so that attention over millions of tokens is attention over 512, in
64 bits, and every sum of the values grows to one side.  Tolerances, relative to a row's norm:
  p       scores between -1 and 0 in powers of two: 5.4e-7 for a weight against another (two roundings of q~, two additions in S,
          one difference, ex2), in numerator and denominator: 1.1e-6
  O       the tensor core cuts off what an addition leaves behind the last bits of a sum, all to one side.  Of the 24 bits of the sum
          that is half a step on average for each of 4 additions a page: over 24 pages of a sum that grows evenly
          2/3 x 96 x 2^-25 x 1.1 = 2.0e-6, and 2.4e-6 with six deviations
  joins   the runs of a CTA (88 here, at most) are added in fp32, rounded to nearest, with a product each; six deviations of as many
          steps, 0.29 sqrt(2 x 88 / 3) 2^-23 each, are 1.6e-6, in numerator and denominator
in all 6.7e-6 for fp32 outputs (found: 2.9e-6 of a row, 4.2e-6 of an output).  bf16 outputs go through runs of 128 pages: 1.1e-5 in O
from the sums' bits and, since the 64 products of a query and a page are themselves cut a few bits behind the sum's last one (three:
2/3 x 128 x 64 x 2^-28 x 1.1), 2.2e-5 from theirs; with 4.3e-6 from above 3.8e-5 (found with fp32 outputs and runs of 128: 3.6e-5).
Where a run has all of a CTA's pages (2100) the sums of 64 queries are off by more than 1.8e-4, with eight runs by more than 2.2e-5.
"""
import math

import pytest
import torch

from helpers import ensure_library, f64
from test_prefix_decode_gpu import BLOCK, D, Batch, dev

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


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


def long_batch(lla, W, pages, H, io):
    """W sequences that share `pages` pages, eight blocks again and again; and the outputs in 64 bits."""
    assert pages % 8 == 0
    x = Batch(lla, [list(range(8)) * (pages // 8)] * W, [pages * BLOCK] * W, H=H, io=io, seed=W)
    ids = x.table[0, :8].long().to(DEV)
    g = torch.Generator().manual_seed(W)
    values = (0.5 + torch.rand(8, H, BLOCK, 160, generator=g)).to(BF16)
    eye = torch.eye(BLOCK, 96, dtype=BF16).view(BLOCK, 12, 8).transpose(0, 1).reshape(-1)
    x.pool[ids, :, :BLOCK * 96] = eye.to(DEV)
    x.pool[ids, :, BLOCK * 96:] = values.view(8, H, -1).to(DEV)
    x.wk.copy_(torch.eye(D, 96, dtype=BF16, device=DEV).expand_as(x.wk))
    x.wv.copy_(torch.eye(D, 160, dtype=BF16, device=DEV).expand_as(x.wv))
    x.q.copy_(-torch.rand(W, H, D, generator=g) * (math.sqrt(D) * math.log(2.0)))
    p = torch.exp(x.q[:, :, :BLOCK].cpu().double() / math.sqrt(D))
    want = torch.einsum("bht,hte->bhe", p / p.sum(-1, keepdim=True), values.double().mean(0))
    return x, want[..., :D]


@pytest.mark.parametrize("W", [9, 20, 64])
def test_fp32_sums_over_millions_of_tokens(lla, W):
    x, want = long_batch(lla, W, 40000, 8, F32)
    off = torch.from_numpy(f64(x.decode(pass1=False))) - want
    assert (off.norm(dim=2) <= 6.7e-6 * want.norm(dim=2)).all()


@pytest.mark.parametrize("W", [9, 64])
def test_bf16_sums_over_millions_of_tokens(lla, W):
    """Every output is the bf16 number of a sum within 4.2e-5 of the exact one: 3.8e-5, and 2^-18 for p in two parts.  (Rounding keeps
    the order.  The mean error says less: the outputs of many sequences lie between the same few bf16 numbers.)"""
    x, want = long_batch(lla, W, 40000, 8, BF16)
    out = torch.from_numpy(f64(x.decode(pass1=False)))
    low, high = ((want * (1 + e)).to(BF16).double() for e in (-4.2e-5, 4.2e-5))
    assert (low <= out).all() and (out <= high).all()


@pytest.mark.parametrize("io, W, pages", [(F32, 9, 2000), (F32, 20, 2001), (F32, 64, 1999), (BF16, 40, 6001)])
def test_maxima_that_rise_from_run_to_run(lla, io, W, pages):
    """Scores that grow along the pages, so that a record is scaled again with every run: several runs of each unit in a CTA.
    (Scores up to 3.2 times those of the tolerance 2e-4.)"""
    x = Batch(lla, [list(range(pages))] * W, [pages * BLOCK] * W, H=8, io=io, seed=W, sigma=0.5)
    x.pool[x.table[0, :pages].long().to(DEV)] *= torch.linspace(0.2, 3.2, pages, device=DEV).to(BF16).view(-1, 1, 1)
    out = x.decode()
    x.check(out, pairs=[(0, 0), (W // 2, 3), (W - 1, 7)], tol=6.4e-4)
    for _ in range(3):
        assert torch.equal(x.decode(), out)


@pytest.mark.parametrize("W, pages, mean", [(64, 256, 0.0), (64, 4096, 0.0), (12, 4096, 0.0), (64, 4096, 1.0)])
def test_fp32_errors_are_those_of_an_fp32_evaluation(lla, W, pages, mean):
    """Random latents, and ones with a mean, whose sums grow to one side: the error against 64 bits, in the norm over all outputs, is that
    of the same products, exponentials and sums by torch in fp32, times 1.2 for the order of its sums, or less.  (Found: 0.45, 1.38, 0.48
    and 1.64e-6, where the fp32 evaluation has 2.3, 9.4, 0.68 and 7.3e-6.)"""
    x = Batch(lla, [list(range(pages))] * W, [pages * BLOCK] * W, H=2, seed=W + pages)
    if mean:
        x.pool += mean
    out = x.decode(pass1=False).double()
    page = x.pool[x.table[0, :pages].long().to(DEV)]
    for t in (torch.float64, F32):
        ck = page[..., :BLOCK * 96].view(pages, 2, 12, BLOCK, 8).permute(1, 0, 3, 2, 4).reshape(2, -1, 96).to(t)
        cv = page[..., BLOCK * 96:].view(pages, 2, BLOCK, 160).permute(1, 0, 2, 3).reshape(2, -1, 160).to(t)
        qt = torch.einsum("bhd,hdr->hbr", x.q.to(t), x.wk[:, 1].to(t))
        s = qt @ ck.transpose(1, 2) / math.sqrt(D)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.einsum("hbr,hdr->bhd", (p / p.sum(-1, keepdim=True)) @ cv, x.wv[:, 1].to(t)).double()
        if t == F32:
            err = (o - want).norm()
        else:
            want = o
        del ck, cv, s, p
    assert (out - want).norm() <= 1.2 * err
