"""lla_beam_select against its definition in 64 bits, and lla_beam_search over the latent cache.

What is compared, and how far it may be off.  A beam's log of the sum of exponentials is off by at most `slack` (below,
from the formula), so continuations of different beams whose exact keys are closer than two of them (and the scores' own
rounding) may change places; within a beam the order is that of the logits and exact.  So: every returned
continuation's score is the exact one of that (beam, token) within slack plus half an fp32 step; rank k's exact key is the
exact k-th best within two slacks; and the tokens of a beam come in the exact order without a gap."""
import math

import numpy as np
import pytest
import torch

import oracle
from helpers import ensure_library, f64

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, U8, F32, BF16 = torch.int32, torch.uint8, torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    m.lla_clear_device_error()
    return m


def dev(v, t=I32):
    return torch.tensor(v, dtype=t, device=DEV)


def slack(z):
    """How far log sum exp of the finite logits z (64-bit) may be off: ex2.approx is off by 2^-22; its argument
    (z - m) log2 e, with m within 60 of the maximum or on either side of it, by three roundings of 2^-24 of |z - m|, whose mean
    under the softmax is what counts (m counts once more: the terms' weights are those of the softmax); the sums carry
    their rounding errors, a tile's tree of 32 terms five roundings; expf joins the shares at 2^-22."""
    p = np.exp(z - z.max())
    p /= p.sum()
    return 2 ** -22 * 2 + 5 * 2 ** -24 + 3 * 2 ** -24 * (float((p * (z.max() - z)).sum()) + 60)


def reference(z, score, done, n, eos, alpha):
    """Every continuation of one sequence, best first: (key, beam, rank in the beam, token, score, length); and the slack
    of each beam in key and score."""
    found, off = [], []
    for w in range(z.shape[0]):
        off.append(0.0)
        s, length = float(score[w]), int(n[w])
        if not math.isfinite(s):
            continue
        if done[w]:
            found.append((s * float(max(1, length)) ** -alpha, w, 0, eos, s, length))
            continue
        ids = np.flatnonzero(np.isfinite(z[w]))
        if not len(ids):
            continue
        x = z[w][ids].astype(np.float64)
        top = x.max()
        log_sum = math.log(float(np.exp(x - top).sum()))
        off[w] = slack(x)
        scale = float(max(1, length + 1)) ** -alpha
        near = np.flatnonzero(x >= np.partition(x, -40)[-40]) if len(x) > 40 else np.arange(len(x))
        order = near[np.lexsort((ids[near], -x[near]))][:40]
        for r, i in enumerate(order):
            t = s + ((x[i] - top) - log_sum)
            found.append((t * scale, w, r, int(ids[i]), t, length + 1))
    found.sort(key=lambda f: (-f[0], f[1], f[2]))
    return found, off


class Select:
    def __init__(self, lla, z, score, K, done=None, n=None, eos=-1, alpha=0.0):
        B, W, V = z.shape
        self.args = (z, score, K, done, n, eos, alpha)
        o = self.out = dict(parents=torch.full((B, K), 99, dtype=I32, device=DEV), tokens=torch.full((B, K), 99, dtype=I32, device=DEV),
                            out_scores=torch.full((B, K), 99.0, device=DEV), out_finished=torch.full((B, K), 99, dtype=U8, device=DEV),
                            out_lengths=torch.full((B, K), 99, dtype=I32, device=DEV) if n is not None else None)
        self.ws = torch.full((lla.lla_beam_select_workspace_size(B, W, V, K, z.dtype),), 0xA5, dtype=U8, device=DEV)
        self.call = lambda stream=None: lla.lla_beam_select(
            z, score, o["parents"], o["tokens"], o["out_scores"], self.ws, finished=done, lengths=n, out_finished=o["out_finished"],
            out_lengths=o["out_lengths"], eos=eos, length_penalty=alpha, stream=stream)
        self.call()

    def check(self):
        z, score, K, done, n, eos, alpha = self.args
        B, W, V = z.shape
        got = {k: v.cpu().numpy() for k, v in self.out.items() if v is not None}
        zs, ss = f64(z), score.cpu().numpy()
        dn = np.zeros((B, W), int) if done is None else done.cpu().numpy()
        ln = np.zeros((B, W), int) if n is None else n.cpu().numpy()
        for b in range(B):
            want, off = reference(zs[b], ss[b], dn[b], ln[b], eos, alpha)
            by = {(f[1], f[3]): f for f in want}
            wide = max(off) * max([1.0] + [f[0] / f[4] for f in want if f[4]])
            seen = {}
            for k in range(K):
                at = (b, k)
                if k >= len(want):
                    assert got["parents"][at] == got["tokens"][at] == -1 and got["out_scores"][at] == -np.inf and got["out_finished"][at] == 1
                    assert n is None or got["out_lengths"][at] == 0
                    continue
                w, token = int(got["parents"][at]) - b * W, int(got["tokens"][at])
                assert (w, token) in by, (b, k, w, token, want[k])
                key, _, rank, _, total, length = by[w, token]
                assert rank == seen.get(w, 0), (b, k, w, token, rank)
                seen[w] = rank + 1
                s = float(got["out_scores"][at])
                if abs(total) < 3e38:
                    assert abs(s - total) <= off[w] + abs(total) * 2 ** -24, (b, k, s, total)
                assert abs(key - want[k][0]) <= 2 * wide + abs(key) * 1e-14, (b, k, key, want[k])
                assert got["out_finished"][at] == (bool(dn[b, w]) or token == eos)
                assert n is None or got["out_lengths"][at] == length
        return self


def logits(seed, B, W, V, dtype, pad=0, offset=0, scale=2.5):
    """[B][W][V] in rows of V + pad elements, `offset` elements into an allocation; NaN around the rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    flat = torch.full((offset + B * W * (V + pad) + 8,), math.nan, dtype=dtype, device=DEV)
    z = flat[offset:offset + B * W * (V + pad)].view(B, W, V + pad)[:, :, :V]
    z.copy_(torch.randn(B, W, V, generator=g, device=DEV) * scale)
    return z


def scores(seed, B, W):
    return -10 - 5 * torch.rand(B, W, generator=torch.Generator(device=DEV).manual_seed(seed + 77), device=DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,W,K,V,pad,offset", [
    (1, 1, 1, 1, 0, 0), (2, 3, 4, 1, 0, 0), (1, 1, 32, 7, 0, 0), (3, 2, 8, 33, 1, 1), (2, 4, 8, 1000, 0, 3), (1, 32, 32, 500, 3, 5),
    (5, 4, 4, 8192, 0, 0), (2, 4, 8, 8193, 5, 7), (1, 2, 32, 32000, 0, 0), (3, 5, 10, 50257, 0, 1), (1, 1, 5, 1 << 18, 0, 0),
    (40, 4, 8, 4097, 2, 2), (64, 16, 16, 600, 0, 0), (1024, 1, 3, 300, 1, 0)])
def test_against_the_definition(lla, dtype, B, W, K, V, pad, offset):
    Select(lla, logits(V + W, B, W, V, dtype, pad, offset), scores(V, B, W), K).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("alpha", [0.0, 0.7, -1.0, 2.0])
def test_ended_dead_and_penalised_beams(lla, dtype, alpha):
    B, W, K, V, eos = 6, 5, 10, 3001, 7
    g = torch.Generator(device=DEV).manual_seed(5)
    z, s = logits(11, B, W, V, dtype), scores(11, B, W)
    z[:, :, eos] = 9.0  # every beam is likely to end
    done = (torch.rand(B, W, generator=g, device=DEV) < 0.4).to(U8)
    n = torch.randint(0, 50, (B, W), generator=g, device=DEV).to(I32)
    s[0, 1], s[1, 2], s[2, 0] = -math.inf, math.nan, math.inf
    done[3], s[4] = 1, -math.inf  # only ended beams; none alive
    z[5] = -math.inf              # nothing to continue with but the ended
    n[0, 0] = -3
    n[0, 3] = 2 ** 31 - 1
    x = Select(lla, z, s, K, done, n, eos, alpha).check()
    assert x.out["parents"][4].tolist() == [-1] * K


def test_no_optional_arguments(lla):
    z, s = logits(3, 2, 3, 999, BF16), scores(3, 2, 3)
    x = Select(lla, z, s, 4).check()
    o = {k: torch.zeros_like(v) for k, v in x.out.items() if v is not None}
    lla.lla_beam_select(z, s, o["parents"], o["tokens"], o["out_scores"], x.ws)
    for k in ("parents", "tokens", "out_scores"):
        assert torch.equal(o[k], x.out[k])


KINDS = ["equal", "zeros of both signs", "rising", "falling", "few finite", "lowest", "not finite", "huge", "denormal", "late block", "two values",
         "late rise"]


def test_rows_of_every_kind_in_many_tiles(lla):
    """The same with so many rows that a CTA has a whole row of nine tiles (of five in bf16), not one tile of it."""
    for what in KINDS:
        for dtype in (BF16, F32):
            rows_of_a_kind(lla, what, 33000, dtype, B=39, W=16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [100, 8192, 70000])
@pytest.mark.parametrize("what", KINDS)
def test_rows_of_every_kind(lla, what, V, dtype):
    rows_of_a_kind(lla, what, V, dtype, B=2, W=3)


def rows_of_a_kind(lla, what, V, dtype, B, W):
    K = 12
    z = logits(V, B, W, V, dtype, pad=3, offset=1)
    ramp = torch.arange(V, device=DEV, dtype=torch.float32)
    big = torch.finfo(dtype).max
    if what == "equal":
        z[:] = 1.5
    elif what == "zeros of both signs":
        z[:] = torch.where(ramp % 3 == 0, -0.0, 0.0)
        z[:, :, 40:60] = -1.0
    elif what == "rising":
        z[:] = (ramp / V * 20).to(dtype)
    elif what == "falling":
        z[:] = (-ramp / V * 20).to(dtype)
    elif what == "few finite":
        keep = z[:, :, [3, 50, V - 1]].clone()
        z[:] = -math.inf
        z[:, :, [3, 50, V - 1]] = keep
    elif what == "lowest":
        z[:] = torch.where(ramp % 5 == 1, z, -big)
        z[0, 0] = -big  # masked whole: as good as any
    elif what == "not finite":
        z[:] = torch.where(ramp % 7 == 2, math.nan, z)
        z[:] = torch.where(ramp % 11 == 3, math.inf, z)
        z[1, 1] = math.nan
        z[1, 2] = math.inf
    elif what == "huge":
        z[:] = z * 1e30
        z[0, 0, 5], z[0, 1, V - 1], z[0, 2] = big, -big, z[0, 2] * 1e7
    elif what == "denormal":
        z[:] = z * torch.finfo(dtype).tiny / 4
    elif what == "late block":
        z[:, :, :V * 3 // 4] = -math.inf
    elif what == "two values":
        z[:] = torch.where(ramp % 101 == 5, 2.0, 1.0)
    elif what == "late rise":
        z[:, :, V * 2 // 3:] += 200
    Select(lla, z, scores(V, B, W), K).check()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [1, 2, 6, 21, 22, 31, 32])
def test_ties_of_every_number(lla, K, dtype):
    """Rounded logits: from row to row another number of logits share the K-th best value, a handful or thousands."""
    B, W, V = 16, 4, 9000
    g = torch.Generator(device=DEV).manual_seed(K)
    step = 2.0 ** (torch.arange(B * W, device=DEV).view(B, W, 1) / 7 - 7)
    z = (torch.round(torch.randn(B, W, V, generator=g, device=DEV) / step) * step).to(dtype)
    z[0, :, 300:] = -math.inf  # few finite ones, equal in part
    Select(lla, z, scores(K, B, W), K).check()


def test_the_same_beam_twice(lla):
    """Equal beams tie everywhere: the lower beam first, then the lower token."""
    z = logits(4, 1, 1, 5000, BF16).expand(1, 4, 5000).contiguous()
    x = Select(lla, z, torch.full((1, 4), -3.0, device=DEV), 8)
    x.check()
    order = x.out["tokens"][0].tolist()
    top = torch.sort(z[0, 0].float(), descending=True, stable=True)
    want = [(w, int(t)) for _, w, t in sorted((-float(v), w, int(t)) for v, t in zip(top.values[:8], top.indices[:8]) for w in range(4))][:8]
    assert list(zip(x.out["parents"][0].tolist(), order)) == want


def test_repeats_bit_for_bit(lla):
    z, s = logits(8, 16, 4, 50000, BF16), scores(8, 16, 4)
    x = Select(lla, z, s, 8)
    first = {k: v.clone() for k, v in x.out.items() if v is not None}
    for _ in range(20):
        x.call()
        assert all(torch.equal(first[k], x.out[k]) for k in first)


@pytest.mark.parametrize("how", ["stream", "graph"])
def test_another_stream_and_a_captured_graph(lla, how):
    xs = [Select(lla, logits(s, 3, 4, 9000, BF16), scores(s, 3, 4), 8) for s in (1, 2)]
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in x.out.items() if v is not None} for x in xs]
    for x in xs:
        for v in x.out.values():
            if v is not None:
                v.fill_(7)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    if how == "stream":
        for x in xs:
            x.call(side)
        side.synchronize()
    else:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for x in xs:
                x.call(side)
        g.replay()
        g.replay()
        torch.cuda.synchronize()
    for x, w in zip(xs, want):
        assert all(torch.equal(w[k], x.out[k]) for k in w)


def test_both_marshallings(lla, monkeypatch):
    z, s = logits(9, 2, 4, 3000, F32, pad=5), scores(9, 2, 4)
    n = torch.full((2, 4), 5, dtype=I32, device=DEV)
    real, took = lla._native(), []

    class Spy:
        def beam_select(self, *a):
            took.append(real.beam_select(*a))
            return took[-1]

    monkeypatch.setattr(lla, "_native_module", Spy())
    a = Select(lla, z, s, 6, n=n, alpha=0.5)
    assert took == [0]
    monkeypatch.setattr(lla, "_native_module", lla._Absent())
    b = Select(lla, z, s, 6, n=n, alpha=0.5)
    assert all(torch.equal(a.out[k], b.out[k]) for k in a.out)


def test_wrong_tensors_are_refused(lla):
    z, s = logits(9, 2, 4, 3000, F32), scores(9, 2, 4)
    x = Select(lla, z, s, 6)
    o = x.out

    def call(z=z, s=s, **kw):
        a = dict(parents=o["parents"], tokens=o["tokens"], out_scores=o["out_scores"], workspace=x.ws)
        a.update(kw)
        lla.lla_beam_select(z, s, a.pop("parents"), a.pop("tokens"), a.pop("out_scores"), a.pop("workspace"), **a)

    call()
    for bad, why in ((dict(z=z.transpose(1, 2)), "dense"), (dict(z=z[:, :3]), "one distance"), (dict(z=z.cpu()), "CUDA"), (dict(z=z.half()), "dtype"),
                     (dict(s=s.double()), "float32"), (dict(s=s[:1]), "shape"), (dict(tokens=o["tokens"].long()), "int32"),
                     (dict(finished=torch.zeros(2, 4, dtype=I32, device=DEV)), "uint8"), (dict(parents=o["parents"][0]), "B"),
                     (dict(workspace=x.ws.cpu()), "CUDA")):
        with pytest.raises(ValueError, match=why):
            call(**bad)
    for bad, why in ((dict(workspace=x.ws[:16]), "WORKSPACE"), (dict(eos=3000), "INVALID"), (dict(eos=-2), "INVALID"),
                     (dict(length_penalty=0.5), "INVALID"), (dict(length_penalty=math.nan), "INVALID"),
                     (dict(z=z[:, :1].expand(2, 4, 3000)), "INVALID|one distance")):
        with pytest.raises((lla.LLAError, ValueError), match=why):
            call(**bad)


# ------------------------------------------------------------------------------------------------ the search

class Model:
    """A model with one looped attention layer over the latent cache (pass 1, loop 1): a token is its keys, values
    and queries, and the attention output gives the logits."""
    T, H, d, r_k, r_v, V, LOOP = 2, 2, 128, 96, 160, 61, 1

    def __init__(self, lla, seed, eos):
        from paper_2607_15456_gb300 import workloads as W
        self.lla = lla
        self.geom = lla.Geometry(self.T, self.H, self.d, self.r_k, self.r_v)
        self.weights = W.codec_tensors(self.T, self.H, self.d, self.r_k, self.r_v, seed, 0, device=DEV)
        self.codec = lla.Codec(**self.weights)
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(BF16)
        self.xk, self.xv = rnd(self.T, self.V, self.H, self.d), rnd(self.T, self.V, self.H, self.d)
        self.q = rnd(self.V, self.H, self.d)
        self.out_w = torch.randn(self.H * self.d, self.V, generator=g, device=DEV) * 0.35
        if eos >= 0:
            self.out_w[:, eos] *= 3

    def encode(self, pool, num_blocks, tokens, slots):
        t = tokens.long()
        cache = self.lla.Cache(pool, num_blocks, None, 1)
        self.lla.lla_encode(self.geom, self.codec, cache, self.xk[:, t].contiguous(), self.xv[:, t].contiguous(), slots)

    def attend(self, pool, num_blocks, table, lens, tokens, ws):
        t = tokens.long()
        out = torch.empty(len(t), self.H, self.d, dtype=torch.float32, device=DEV)
        cache = self.lla.Cache(pool, num_blocks, table, table.shape[1])
        q, k, v = self.q[t].float(), self.xk[self.LOOP, t].float(), self.xv[self.LOOP, t].float()
        self.lla.lla_decode_attn(self.geom, self.codec, cache, lens, table.shape[1] * 64, self.LOOP, q, k, v, out, ws)
        return out

    def logits(self, out):
        # one row at a time: the same arithmetic for a row wherever it stands in the batch
        return (out.reshape(len(out), -1)[:, :, None] * self.out_w).sum(1)


@pytest.mark.parametrize("eos,alpha", [(-1, 0.0), (9, 0.8)])
def test_search_over_shared_pages(lla, eos, alpha):
    """Two prompts, four beams, 70 steps, so that every beam's pages end and fork many times.  Each step's logits equal, bit for
    bit, those of the same hypotheses on pages of their own, encoded from their tokens anew; every selection is checked against
    the definition; the last step's attention against the oracle; and no page is lost."""
    lla.lla_clear_device_error()
    B, W, steps = 2, 4, 70
    m = Model(lla, 3, eos)
    S, V, mb, nb = B * W, m.V, 4, 64
    bb = lla.lla_cache_block_bytes(m.geom)
    pool = torch.full((nb * bb,), 0xFF, dtype=U8, device=DEV)
    pools = lla.Pools([lla.lla_cache_pool(m.geom, pool)])
    ref = torch.zeros(nb, dtype=I32, device=DEV)
    prompts = [torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n)).tolist() for n in (60, 131)]
    # the prompts without their last tokens, encoded once, then forked into their beams
    first = lla.Pages(ref, torch.full((B, mb), -1, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV))
    a, b = (lla.Pages(ref, torch.full((S, mb), -1, dtype=I32, device=DEV), torch.zeros(S, dtype=I32, device=DEV)) for _ in range(2))
    ews = torch.empty(lla.lla_pages_extend_workspace_size(S), dtype=U8, device=DEV)
    lens = [len(p) - 1 for p in prompts]
    slots = torch.zeros(sum(lens), dtype=torch.int64, device=DEV)
    lla.lla_pages_extend(first, pools, slots, ews, cu_new=dev(np.cumsum([0] + lens).tolist()))
    m.encode(pool, nb, dev(sum((p[:-1] for p in prompts), [])), slots)
    lla.lla_pages_fork(first, a, dev([i // W for i in range(S)]))

    tokens, lengths = (torch.zeros(steps + 1, B, W, dtype=I32, device=DEV) for _ in range(2))
    finished, parents = torch.zeros(steps + 1, B, W, dtype=U8, device=DEV), torch.zeros(steps, B, W, dtype=I32, device=DEV)
    score = torch.full((steps + 1, B, W), -math.inf, device=DEV)
    score[0, :, 0] = 0
    tokens[0] = dev([[p[-1]] * W for p in prompts])
    dws = torch.zeros(lla.lla_decode_workspace_size(m.geom, S), dtype=U8, device=DEV)
    seen, kept = [], []

    def step(i, pages, before, toks, step_slots):
        before, toks = before.clone(), toks.reshape(-1)
        out = m.attend(pool, nb, pages.block_table, before, toks, dws)
        m.encode(pool, nb, toks, step_slots)
        seen.append((before, out))
        kept.append(m.logits(out).view(B, W, V))
        return kept[-1]

    ws = torch.empty(lla.lla_beam_search_workspace_size(B, W, V, F32), dtype=U8, device=DEV)
    lla.lla_beam_search(a, b, pools, V, step, tokens, score, finished, lengths, parents, ws, dtype=F32, eos=eos, length_penalty=alpha)
    assert lla.lla_get_device_error() == 0

    # the ledger: every block is held as often as tables hold it
    last = a if steps % 2 == 0 else b
    count = [0] * nb
    for s in range(S):
        for j in range(-(-int(last.context_lens[s]) // 64)):
            count[int(last.block_table[s, j])] += 1
    assert ref.tolist() == count

    # the same hypotheses on pages of their own
    tk, pr, fn = tokens.cpu(), parents.cpu(), finished.cpu()
    history = [prompts[s // W][:] for s in range(S)]
    own_nb = S * mb
    table = torch.arange(own_nb, dtype=I32, device=DEV).view(S, mb)
    for i in range(steps):
        before, out = seen[i]
        assert before.tolist() == [len(h) - 1 for h in history], i
        if i % 9 == 0 or i == steps - 1:
            own = torch.full((own_nb * bb,), 0xFF, dtype=U8, device=DEV)
            # in the batches in which the search encoded them: the prompts together, then a token of each beam at a time
            n_prompt = [len(prompts[s // W]) - 1 for s in range(S)]
            for s0 in range(0, W):
                toks = dev(sum((history[v * W + s0][:n_prompt[v * W]] for v in range(B)), []))
                own_slots = [(v * W + s0) * mb * 64 + p for v in range(B) for p in range(n_prompt[v * W])]
                m.encode(own, own_nb, toks, dev(own_slots, torch.int64))
            for j in range(i):
                at = [n_prompt[s] + j for s in range(S)]
                has = [at[s] < len(history[s]) - 1 for s in range(S)]
                m.encode(own, own_nb, dev([history[s][at[s]] if has[s] else 0 for s in range(S)]),
                         dev([s * mb * 64 + at[s] if has[s] else -1 for s in range(S)], torch.int64))
            again = m.attend(own, own_nb, table, before, dev([h[-1] for h in history]), torch.zeros_like(dws))
            assert torch.equal(again, out), i
        x = Select.__new__(Select)
        x.args = (kept[i], score[i], W, finished[i], lengths[i], eos, alpha)
        x.out = dict(parents=parents[i], tokens=tokens[i + 1], out_scores=score[i + 1], out_finished=finished[i + 1], out_lengths=lengths[i + 1])
        x.check()
        new = []
        for s in range(S):
            p = int(pr[i].view(-1)[s])
            # an ended beam keeps its hypothesis (whose last token is not cached); one that goes on adds its token
            new.append(history[p][:] if fn[i].view(-1)[p] else history[p] + [int(tk[i + 1].view(-1)[s])])
        history = new
    if eos >= 0:
        assert fn.any()

    # the attention of the last step from explicitly rebuilt keys and values
    xk, xv, w = f64(m.xk), f64(m.xv), {k: f64(v) for k, v in m.weights.items() if v is not None}
    before, out = seen[-1]
    for s in (0, S - 1):
        hist = history_before(prompts, tk, pr, fn, steps - 1, s, W)
        for h in range(m.H):
            ck = oracle.encode(xk[:, hist[:-1], h], None, w["w_down_k"][h])
            cv = oracle.encode(xv[:, hist[:-1], h], None, w["w_down_v"][h])
            t = hist[-1]
            want = oracle.decode(m.LOOP, ck, cv, w["w_up_k"][h], w["w_up_v"][h], None, None, f64(m.q)[t, h], xk[m.LOOP, t, h], xv[m.LOOP, t, h],
                                 1 / math.sqrt(m.d))
            got = f64(out)[s, h]
            assert np.abs(got - want).max() <= 2e-2 and np.linalg.norm(got - want) <= 5e-3 * np.linalg.norm(want)


def history_before(prompts, tk, pr, fn, step, s, W):
    """The tokens of beam s of slab `step` (prompt first), walking back."""
    got = []
    for i in range(step, 0, -1):
        p = int(pr[i - 1].view(-1)[s])
        if not fn[i - 1].view(-1)[p]:
            got.append(int(tk[i].view(-1)[s]))
        s = p
    return prompts[s // W] + got[::-1]


@pytest.mark.parametrize("which", ["stream", "handle"])
def test_search_on_another_stream(lla, which):
    """The callback runs with the search's stream as the current one: the same hypotheses as on the default stream."""
    B, W, V, steps = 2, 3, 400, 12
    table = torch.randn(V, V, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) * 3
    results = []
    for stream in (None, torch.cuda.Stream()):
        ref = torch.zeros(40, dtype=I32, device=DEV)
        pages = [lla.Pages(ref, torch.zeros(B * W, 4, dtype=I32, device=DEV), torch.zeros(B * W, dtype=I32, device=DEV)) for _ in range(2)]
        tokens, lengths = (torch.zeros(steps + 1, B, W, dtype=I32, device=DEV) for _ in range(2))
        finished, parents = torch.zeros(steps + 1, B, W, dtype=U8, device=DEV), torch.zeros(steps, B, W, dtype=I32, device=DEV)
        score = torch.full((steps + 1, B, W), -math.inf, device=DEV)
        score[0, :, 0] = 0
        tokens[0, 1] = 7
        ws = torch.empty(lla.lla_beam_search_workspace_size(B, W, V, F32), dtype=U8, device=DEV)
        streams = []

        def step(i, pages, before, toks, slots):
            streams.append(torch.cuda.current_stream().cuda_stream)
            return table[toks.long()]

        torch.cuda.synchronize()
        lla.lla_beam_search(*pages, lla.Pools(), V, step, tokens, score, finished, lengths, parents, ws, dtype=F32, eos=5, length_penalty=0.3,
                            stream=stream.cuda_stream if stream is not None and which == "handle" else stream)
        torch.cuda.synchronize()
        assert set(streams) == {(stream or torch.cuda.current_stream()).cuda_stream}
        results.append([t.clone() for t in (tokens, parents, score, finished, lengths, ref, pages[0].context_lens)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert lla.lla_get_device_error() == 0


def test_search_stops_with_the_callback(lla):
    m = Model(lla, 3, -1)
    pages = [lla.Pages(torch.zeros(8, dtype=I32, device=DEV), torch.zeros(2, 2, dtype=I32, device=DEV), torch.zeros(2, dtype=I32, device=DEV)) for _ in range(2)]
    pages[1].ref_count = pages[0].ref_count
    slab = lambda t, n=4: torch.zeros(n, 1, 2, dtype=t, device=DEV)
    ws = torch.empty(lla.lla_beam_search_workspace_size(1, 2, m.V, F32), dtype=U8, device=DEV)
    calls = []

    def step(i, *_):
        calls.append(i)
        if i == 1:
            raise KeyError("no model")
        return torch.zeros(1, 2, m.V, device=DEV)

    args = (slab(I32), slab(F32), slab(U8), slab(I32), slab(I32, 3), ws)
    with pytest.raises(KeyError, match="no model"):
        lla.lla_beam_search(*pages, lla.Pools(), m.V, step, *args, dtype=F32)
    assert calls == [0, 1]
    with pytest.raises(ValueError, match="logits"):
        lla.lla_beam_search(*pages, lla.Pools(), m.V, lambda *_: torch.zeros(1, 2, 5, device=DEV), *args, dtype=F32)
    with pytest.raises(lla.LLAError, match="WORKSPACE"):
        lla.lla_beam_search(*pages, lla.Pools(), m.V, step, *args[:-1], ws[:32], dtype=F32)
    lla.lla_clear_device_error()
