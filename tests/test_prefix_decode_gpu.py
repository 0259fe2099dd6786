"""lla_decode_attn_prefix and lla_decode_attn_prefix_decoupled against attention over every sequence's own table row in
64 bits (keys and values rebuilt for every token), and against the same pages read without a plan.

Tolerance, per (sequence, head) row, relative to the row's norm, from the fp32 arithmetic at these inputs (latents, queries
N(0, 1); weights N(0, 1/r)): a q~ of 128 products in sums of 24 steps is off by 24 2^-24 sum |q w| ~ 24 2^-24 8 = 1.1e-5; a score
of r_k + d_rope products by scale (r_k 0.8 1.1e-5 + 24 2^-23 sum |q~ c|) ~ 0.09 (8e-4 + 2.4e-4) < 1e-4; weights e^s are off by as
much relative, in numerator and denominator: 2e-4.  Two bf16 parts of p add 2^-18.  bf16 outputs add half a step, 2^-8.
"""
import math
import random

import numpy as np
import pytest
import torch

from helpers import ensure_library, f64, unpack_head

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16
BLOCK, D, T = 64, 128, 4


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


class Batch:
    """Sequences with table rows `rows` (numbers of pages) and lengths `lens` over a pool of random latents."""

    def __init__(self, lla, rows, lens, H=3, rk=96, rv=160, io=F32, mu=False, d_rope=0, seed=0, garbage=False, sigma=1.0):
        self.lla, self.rows, self.lens, self.H, self.rk, self.rv, self.io, self.dr = lla, rows, lens, H, rk, rv, io, d_rope
        B, self.B = len(lens), len(lens)
        g = torch.Generator().manual_seed(seed)
        n = lambda *s, dtype=F32, scale=1.0: (torch.randn(*s, generator=g) * scale).to(dtype).to(DEV)
        used = max([0] + [p + 1 for r in rows for p in r])
        self.nb = used + 2
        ids = torch.randperm(self.nb, generator=g)
        mb = max([1] + [len(r) for r in rows])
        table = torch.full((max(B, 1), mb), -1, dtype=I32)
        for s, r in enumerate(rows):
            if r:
                table[s, :len(r)] = ids[torch.tensor(r)].to(I32)
        self.table = table
        self.geom = lla.Geometry(T, H, D, rk, rv)
        self.pool = n(self.nb, H, BLOCK * (rk + rv), dtype=BF16)
        self.planes = n(self.nb, BLOCK * max(d_rope, 1), dtype=BF16)
        if garbage:  # what lies behind a sequence's last token is not read
            nan = float("nan")
            for s, L in enumerate(lens):
                if L % BLOCK:
                    b = int(table[s, L // BLOCK])
                    page = self.pool[b]
                    page[:, :BLOCK * rk].view(H, rk // 8, BLOCK, 8)[:, :, L % BLOCK:] = nan
                    page[:, BLOCK * rk:].view(H, BLOCK, rv)[:, L % BLOCK:] = nan
                    if d_rope:
                        self.planes[b].view(d_rope // 8, BLOCK, 8)[:, L % BLOCK:] = nan
        self.wk, self.wv = n(H, T, D, rk, dtype=BF16, scale=rk ** -0.5), n(H, T, D, rv, dtype=BF16, scale=rv ** -0.5)
        self.mk, self.mv = (n(H, T * D), n(H, T * D)) if mu else (None, None)
        down = torch.zeros(16, dtype=BF16, device=DEV)
        self.codec = lla.Codec(down, down, self.wk, self.wv, self.mk, self.mv)
        self.cache = lla.Cache(self.pool, self.nb, table.to(DEV), mb)
        self.lens_t, self.max_ctx = dev(lens), mb * BLOCK
        self.q, self.ck, self.cv = n(B, H, D, dtype=io, scale=sigma), n(B, H, D, dtype=io), n(B, H, D, dtype=io)
        self.qr, self.ckr = n(B, H, max(d_rope, 1), dtype=io), n(B, max(d_rope, 1), dtype=io)
        self.pos = torch.randint(0, 70000, (3, B), generator=g, dtype=I32).to(DEV)
        self.rope = lla.RopeAxes(10000.0, lla.LLA_ROPE_HALF, (d_rope // 2 - 2 * (d_rope // 8), d_rope // 8, d_rope // 8), lla.LLA_AXES_INTERLEAVED)
        self.plan = lla.Prefix.empty(B)
        self.replan()
        self.ws = torch.full((lla.lla_decode_prefix_workspace_size(self.geom, B, d_rope),), 0xA5, dtype=torch.uint8, device=DEV)

    def replan(self, min_pages=1):
        self.lla.lla_prefix_plan(self.cache, self.lens_t, self.max_ctx, self.plan, min_pages=min_pages)

    def decode(self, loop=1, pass1=True, pos=True, **kw):
        out = torch.full((self.B, self.H, D), 7.0, dtype=self.io, device=DEV)
        cur = (self.ck, self.cv) if pass1 else (None, None)
        if self.dr:
            self.lla.lla_decode_attn_prefix_decoupled(self.geom, self.codec, self.cache, self.plan, self.planes, self.dr, self.rope,
                                                      self.pos if pos else None, self.lens_t, self.max_ctx, loop, self.q, self.qr, *cur,
                                                      self.ckr if pass1 else None, out, self.ws, **kw)
        else:
            self.lla.lla_decode_attn_prefix(self.geom, self.codec, self.cache, self.plan, self.lens_t, self.max_ctx, loop, self.q, *cur, out,
                                            self.ws, **kw)
        return out

    def turned(self, b, h, pass1, pos):
        """rot(q^R) of one query, pair by pair."""
        hp, x = self.dr // 2, f64(self.qr[b, h])
        at = f64(self.pos[:, b]) if pos else np.full(3, self.lens[b] - (0 if pass1 else 1))
        z = x[:hp] + 1j * x[hp:]
        axis = [j % 3 if j // 3 < self.rope.pairs[j % 3] else 0 for j in range(hp)]
        z = z * np.exp(1j * np.array([at[a] for a in axis]) * 10000.0 ** (-np.arange(hp) / hp))
        return np.concatenate([z.real, z.imag])

    def exact(self, b, h, loop=1, pass1=True, pos=True):
        L, q = self.lens[b], f64(self.q[b, h])
        if not hasattr(self, "_u8"):
            self._u8 = self.pool.cpu().contiguous().view(torch.uint8).reshape(-1)
            self._planes = self.planes.cpu()
        ck, cv = unpack_head(self._u8, self.H, self.rk, self.rv, "bf16", self.table[b], L, h)
        K, V = ck @ f64(self.wk[h, loop]).T, cv @ f64(self.wv[h, loop]).T
        if self.mk is not None:
            K, V = K + f64(self.mk[h]).reshape(T, D)[loop], V + f64(self.mv[h]).reshape(T, D)[loop]
        s = K @ q
        if self.dr:
            kr = [f64(self._planes[int(b)]).reshape(self.dr // 8, BLOCK, 8).transpose(1, 0, 2).reshape(BLOCK, self.dr)
                  for b in self.table[b, :-(-L // BLOCK)]]
            s = s + (np.concatenate(kr)[:L] @ self.turned(b, h, pass1, pos) if kr else 0.0)
        if pass1:
            s = np.append(s, q @ f64(self.ck[b, h]) + (f64(self.qr[b, h]) @ f64(self.ckr[b]) if self.dr else 0.0))
            V = np.concatenate([V, f64(self.cv[b, h])[None]])
        s = s / math.sqrt(D)
        p = np.exp(s - s.max())
        return (p @ V) / p.sum()

    def check(self, out, pairs=None, tol=2e-4, **kw):
        got = f64(out)
        r = random.Random(3)
        pairs = pairs or [(b, r.randrange(self.H)) for b in range(self.B)]
        for b, h in pairs:
            want = self.exact(b, h, **kw)
            err = np.linalg.norm(got[b, h] - want) / np.linalg.norm(want)
            assert err <= tol + (2.0 ** -8 if self.io == BF16 else 0.0), (b, h, err)


def shared(P, W, prompt, own, system=0, seed=0, branch=0):
    """P prompts of `prompt` full pages behind `system` ones, W sequences each (every two share `branch` pages more) with up to
    `own` tokens of their own."""
    r, nxt, rows, lens = random.Random(seed), 0, [], []

    def new(n):
        nonlocal nxt
        nxt += n
        return list(range(nxt - n, nxt))

    top = new(system)
    for _ in range(P):
        p = top + new(r.randint(max(0, prompt - 2), prompt))
        for w in range(W):
            if w % 2 == 0:
                br = p + new(branch)
            n = r.randint(0, own)
            rows.append(br + new(-(-n // BLOCK)))
            lens.append(len(br) * BLOCK + n)
    return rows, lens


@pytest.mark.parametrize("W", [1, 2, 7, 8, 9, 31, 32, 33, 40, 63, 64, 65, 130])
def test_group_sizes(lla, W):
    x = Batch(lla, *shared(1, W, 5, 150, seed=W), seed=W)
    x.check(x.decode())


@pytest.mark.parametrize("rk, rv", [(96, 160), (128, 128), (72, 120)])
@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("pass1", [True, False])
def test_shapes_types_and_passes(lla, rk, rv, io, pass1):
    rows, lens = shared(3, 6, 9, 200, system=3, branch=2, seed=4)
    x = Batch(lla, rows, [max(1, n) for n in lens], H=5, rk=rk, rv=rv, io=io, mu=True, garbage=True)
    for loop in (0, 3):
        x.check(x.decode(loop, pass1), loop=loop, pass1=pass1)


@pytest.mark.parametrize("d_rope", [32, 64, 96])
@pytest.mark.parametrize("io, pass1, pos", [(F32, True, True), (F32, False, True), (BF16, True, False), (F32, False, False)])
def test_rotary_branch(lla, d_rope, io, pass1, pos):
    x = Batch(lla, *shared(2, 37, 4, 130, system=1, seed=d_rope), d_rope=d_rope, io=io, garbage=True, H=2)
    x.check(x.decode(2, pass1, pos), pairs=[(b, b % 2) for b in range(0, x.B, 5)], loop=2, pass1=pass1, pos=pos)


@pytest.mark.parametrize("H", [1, 16, 40])
def test_heads(lla, H):
    x = Batch(lla, *shared(2, 5, 7, 70), H=H)
    x.check(x.decode())


def test_nothing_shared_and_empty_sequences(lla):
    """Every sequence on its own: lengths around a page, none (pass 1 gives the current value), all of one page."""
    lens, rows, n = [0, 1, 63, 64, 65, 127, 128, 129, 0, 777], [], 0
    for L in lens:
        rows.append(list(range(n, n + -(-L // BLOCK))))
        n += len(rows[-1])
    x = Batch(lla, rows, lens, garbage=True)
    assert x.plan.num_groups.item() == 0
    out = x.decode()
    x.check(out)
    assert torch.equal(out[0], x.cv[0]) and torch.equal(out[8], x.cv[8])


def test_nothing_of_their_own(lla):
    """Sequences that end with the pages that they share, in groups of every class, and one page in all."""
    for B in (2, 9, 33, 70):
        x = Batch(lla, [[0]] * B, [64] * B, H=2, seed=B)
        assert x.plan.own_page.tolist() == [1] * B
        x.check(x.decode())
        x.check(x.decode(pass1=False), pass1=False)


def test_many_short_runs_of_all_classes(lla):
    """Groups of 2 to 64 members with one or two pages each, beside sequences of one page: every role is a run ahead."""
    r, rows, lens, n = random.Random(1), [], [], 0
    for size in [2, 33, 1, 9, 64, 3, 34, 8, 1, 50, 10, 2, 2, 40]:
        pages = list(range(n, n + r.randint(1, 2)))
        n += len(pages)
        for _ in range(size):
            own = r.choice([0, 1, 64, 100])
            rows.append(pages + list(range(n, n + -(-own // BLOCK))))
            lens.append(len(pages) * BLOCK + own)
            n += -(-own // BLOCK)
    x = Batch(lla, rows, lens, H=4)
    first = x.decode()
    x.check(first)
    for _ in range(20):
        assert torch.equal(x.decode(), first)


def test_maxima_that_grow_late(lla):
    """Scores that rise along the pages, so that what has been summed is scaled again and again, for all classes."""
    for W in (3, 20, 50):
        x = Batch(lla, *shared(1, W, 12, 90, seed=W), H=2, sigma=0.5, seed=W)
        order = x.table[0]
        for i, b in enumerate(order[:12].tolist()):
            x.pool[b] *= 2.0 ** (i / 2 - 1)
        x.check(x.decode(), tol=2e-3)  # (scores up to 32 times as large: ten times the tolerance at least)


def test_one_long_prompt(lla):
    """Far more pages than CTAs for one unit, and so a run of each CTA."""
    x = Batch(lla, *shared(1, 3, 900, 64), H=1)
    x.check(x.decode())


def test_a_nan_stays_with_the_sequences_that_read_it(lla):
    rows, lens = shared(1, 12, 3, 100, seed=2)
    x = Batch(lla, rows, lens, H=2)
    own = x.plan.own_page.tolist()
    s = next(i for i, n in enumerate(lens) if n > own[i] * BLOCK)
    clean = x.decode()
    x.q[s] = float("nan")
    out = x.decode()
    keep = [i for i in range(x.B) if i != s]
    assert torch.isnan(out[s]).all() and torch.equal(out[keep], clean[keep])
    x.q[s] = 0.25
    x.pool[int(x.table[s, own[s]]), :, :8] = float("inf")  # latents of a page that only s reads
    out = x.decode()
    assert torch.equal(out[keep], clean[keep])


def test_min_pages_and_a_plan_from_before(lla):
    """A plan stays right while its sequences grow, and with groups left out."""
    rows, lens = shared(3, 10, 4, 40, system=2, seed=7)
    x = Batch(lla, rows, lens, H=2)
    for least in (1, 3, 6, 100):
        x.replan(least)
        x.check(x.decode())
    x.replan()
    for s in range(0, x.B, 3):  # a token more each, in pages that are there
        if x.lens[s] % BLOCK:
            x.lens[s] += 1
    x.lens_t.copy_(dev(x.lens))
    x.check(x.decode())


def test_as_the_decode_without_a_plan(lla):
    """The pages that nobody shares take another path through lla_decode_attn; both are the documented attention."""
    x = Batch(lla, *shared(4, 9, 11, 300, system=2, seed=9), H=16, io=F32)
    out, want = x.decode(), torch.empty(x.B, x.H, D, device=DEV)
    ws = torch.zeros(lla.lla_decode_workspace_size(x.geom, x.B), dtype=torch.uint8, device=DEV)
    lla.lla_decode_attn(x.geom, x.codec, x.cache, x.lens_t, x.max_ctx, 1, x.q, x.ck, x.cv, want, ws)
    assert (out - want).norm() <= 4e-4 * want.norm()


def test_bad_plans_and_tables_are_flagged(lla):
    rows, lens = shared(2, 6, 3, 64, seed=1)

    def word(change, pass1=True):
        x = Batch(lla, rows, lens, H=2)
        torch.cuda.synchronize()
        change(x)
        x.decode(pass1=pass1)
        w = lla.lla_get_device_error()
        lla.lla_clear_device_error()
        return w

    seq, ctx = lla.LLA_DEVERR_SEQUENCE, lla.LLA_DEVERR_CONTEXT
    at = lambda name, i, v: lambda x: getattr(x.plan, name).view(-1)[i].fill_(v)
    big = 2**31 - 1
    for name, i, v, bit in [("num_groups", 0, -1, seq), ("num_groups", 0, big, seq), ("groups", 0, -1, seq), ("groups", 0, 50, seq), ("groups", 1, big, seq),
                            ("groups", 1, 0, seq), ("groups", 2, -1, seq), ("groups", 2, big, seq), ("groups", 3, 0, seq), ("groups", 3, 65, seq),
                            ("groups", 3, big, seq), ("members", 0, -1, seq), ("members", 0, 12, seq), ("members", 1, big, seq), ("column", 0, big, seq),
                            ("column", 0, 63, seq), ("own_page", 0, -1, ctx), ("own_page", 0, big, ctx)]:
        assert word(at(name, i, v)) & bit, (name, i, v)

    def block(x):
        x.cache.block_table[0, 0] = x.nb
    assert word(block) == lla.LLA_DEVERR_BLOCK_ID
    for L in (-1, 10**6):
        def length(x):
            x.lens_t[3] = L
        assert word(length) & ctx

    def negative(x):
        x.lens_t[2], x.plan.own_page[2] = 0, 0
        x.plan.column[:, 2] = -1
    assert word(negative, pass1=False) & lla.LLA_DEVERR_EMPTY_PASS2
    x = Batch(lla, rows, lens, H=2, d_rope=32)
    x.pos[1, 4] = -5
    x.decode()
    assert lla.lla_get_device_error() == ctx
    lla.lla_clear_device_error()


def test_a_small_workspace_is_refused(lla):
    x = Batch(lla, *shared(1, 2, 1, 5))
    x.ws = x.ws[:-256]
    with pytest.raises(lla.LLAError, match="WORKSPACE"):
        x.decode()


def test_captured_replayed_and_on_another_stream(lla):
    x = Batch(lla, *shared(2, 20, 6, 100, branch=1), H=4, d_rope=64)
    want = x.decode()
    out = torch.zeros_like(want)
    args = (x.geom, x.codec, x.cache, x.plan, x.planes, x.dr, x.rope, x.pos, x.lens_t, x.max_ctx, 1, x.q, x.qr, x.ck, x.cv, x.ckr, out, x.ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lla.lla_decode_attn_prefix_decoupled(*args, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):  # the plan and the decode, as a step makes them
        x.replan()
        lla.lla_decode_attn_prefix_decoupled(*args)
    x.plan.num_groups.zero_()
    for _ in range(3):
        g.replay()
    assert torch.equal(out, want)
    x.q.mul_(0.5)
    g.replay()
    x.check(out)


def test_calls_in_a_row_share_a_workspace(lla):
    """Loops and passes in a row on one workspace, as a layer makes them, without a wait between."""
    x = Batch(lla, *shared(3, 12, 8, 120, seed=5), H=8)
    outs = [x.decode(loop, p) for loop in range(T) for p in (True, False)]
    for (loop, p), out in zip([(loop, p) for loop in range(T) for p in (True, False)], outs):
        x.check(out, loop=loop, pass1=p, pairs=[(b, 0) for b in range(0, x.B, 9)])


def test_no_batch_and_the_largest(lla):
    empty = Batch(lla, [], [], H=2)
    empty.decode()
    rows, lens = shared(16, 64, 3, 64, system=1)
    x = Batch(lla, rows, lens, H=2, rk=72, rv=120)
    assert x.B == 1024
    x.check(x.decode(), pairs=[(b, b % 2) for b in range(0, 1024, 37)])


@pytest.mark.parametrize("B", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("rk, rv, d_rope", [(96, 160, 0), (128, 128, 0), (72, 120, 0), (96, 160, 96)])
def test_up_to_four_sequences_and_one_more(lla, B, rk, rv, d_rope):
    x = Batch(lla, *shared(1, B, 6, 100, system=1, branch=3, seed=B), H=5, rk=rk, rv=rv, d_rope=d_rope, mu=True, garbage=True)
    first = x.decode()
    x.check(first, pairs=[(b, h) for b in range(B) for h in range(5)])
    for _ in range(5):
        assert torch.equal(x.decode(), first)


@pytest.mark.parametrize("W", [1, 2, 3, 4, 9, 33, 64])
def test_weights_and_scores_keep_24_bits(lla, W):
    """One page, with unit vectors for latents and weights: the score of token t is q_t scale, its value the t-th unit vector, so
    that out_t / out_0 = e^(scale q_t) for q_0 = 0 >= q_t.  With |s| <= 1 in powers of two: q~ has two roundings and S two
    (truncated) additions, 2^-23 + 2^-22; the difference to the maximum 2^-24; all of them times ln 2: 3e-7.  ex2 is good to
    2^-22; and four roundings of either output, 8 2^-24.  Together 1.02e-6; weights of two bf16 parts would be off by 2^-18, and
    scores with two parts of q~ by as much."""
    x = Batch(lla, [[0]] * W, [64] * W, H=2)
    page = x.pool[int(x.table[0, 0])]
    page.zero_()
    for t in range(BLOCK):
        page[:, :BLOCK * 96].view(2, 12, BLOCK, 8)[:, t // 8, t, t % 8] = 1
        page[:, BLOCK * 96:].view(2, BLOCK, 160)[:, t, t] = 1
    x.wk.copy_(torch.eye(D, 96, dtype=BF16, device=DEV).expand_as(x.wk))
    x.wv.copy_(torch.eye(D, 160, dtype=BF16, device=DEV).expand_as(x.wv))
    g = torch.Generator().manual_seed(W)
    x.q.copy_(-torch.rand(W, 2, D, generator=g) * (math.sqrt(D) * math.log(2.0)))
    x.q[:, :, 0] = 0
    out = f64(x.decode(pass1=False))[:, :, :BLOCK]
    want = np.exp(f64(x.q)[:, :, :BLOCK] / math.sqrt(D))
    assert np.abs(out / out[:, :, :1] / want - 1).max() <= 1.1e-6


def test_a_group_of_more_members_than_sequences_is_flagged(lla):
    x = Batch(lla, *shared(1, 3, 2, 64), H=2)
    torch.cuda.synchronize()
    x.plan.groups.view(-1)[3] = 5
    x.decode()
    assert lla.lla_get_device_error() & lla.LLA_DEVERR_SEQUENCE
    lla.lla_clear_device_error()


@pytest.mark.parametrize("seed", range(16))
def test_random_batches_as_without_a_plan(lla, seed):
    """Batches of any size, from one page a sequence to many hundred, with whatever they share: as the decode that reads every
    page for itself, each within the tolerance of the 64-bit definition."""
    r = random.Random(seed)
    P, W = r.randint(1, 6), r.choice([1, 2, 3, 4, 5, 17, 40])
    prompt, own = r.choice([0, 1, 4, 30, 200]), r.choice([1, 64, 300, 3000, 20000])
    if P * W * own > 400000:
        own = 300
    d_rope = r.choice([0, 0, 32, 64, 96])
    rk, rv = (96, 160) if d_rope else r.choice([(96, 160), (128, 128), (72, 120)])
    rows, lens = shared(P, W, prompt, own, system=r.choice([0, 2]), branch=r.choice([0, 1, 3]), seed=seed)
    x = Batch(lla, rows, lens, H=r.choice([1, 2, 7]), rk=rk, rv=rv, d_rope=d_rope, mu=not d_rope, seed=seed, garbage=True)
    out, want = x.decode(pos=False), torch.empty(x.B, x.H, D, device=DEV)
    if d_rope:
        rope = lla.RopeAxes(10000.0, lla.LLA_ROPE_HALF, (d_rope // 2, 0, 0), lla.LLA_AXES_BLOCKS)
        at = x.lens_t.repeat(3, 1).contiguous()
        ws = torch.zeros(lla.lla_decode_decoupled_workspace_size(x.geom, d_rope, x.B), dtype=torch.uint8, device=DEV)
        lla.lla_decode_attn_decoupled_axes(x.geom, x.codec, x.cache, x.planes, d_rope, rope, at, x.lens_t, x.max_ctx, 1, x.q, x.qr, x.ck, x.cv,
                                           x.ckr, want, ws)
    else:
        ws = torch.zeros(lla.lla_decode_workspace_size(x.geom, x.B), dtype=torch.uint8, device=DEV)
        lla.lla_decode_attn(x.geom, x.codec, x.cache, x.lens_t, x.max_ctx, 1, x.q, x.ck, x.cv, want, ws)
    assert ((out - want).norm(dim=2) <= 4e-4 * want.norm(dim=2)).all()
    assert torch.equal(x.decode(pos=False), out)


def test_two_streams_at_once(lla):
    """Calls on two streams, each with its own workspace, in any overlap of their kernels."""
    a, b = Batch(lla, *shared(4, 12, 30, 2000, seed=1), H=8), Batch(lla, *shared(1, 3, 40, 900, seed=2), H=8, d_rope=64)
    want = [a.decode(), b.decode()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                outs.append(x.decode())
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, want[i % 2])
