"""Beam search over the paged latent cache, measured: the selection of the next beams, and the pages
of the sequences as they fork, grow, end and are moved together.

A case is a dict of plain values.  `op` names the operator:

  select   the best K continuations of W beams over a vocabulary of V tokens, for B sequences
  fork     block tables of new sequences from their parents' (a parent may have several children or none)
  extend   pages and slots for new tokens; a last page that others hold too is copied before it is written
  free     the pages of sequences that have ended
  compact  the live pages moved to the front of the pools, tables and references renamed

Page cases have P prompts of W beams each.  The beams of a prompt share its pages and the pages of their
common past; `lens` draws the lengths ("fixed:n", "uniform:lo:hi", "log:lo:hi") from `shape_seed`, which also
draws who shares what, so that the work of a case does not depend on the seed of its inputs.  That seed
draws the block ids (a page is anywhere in the pool), the pools' contents, the logits and the scores.  A pass
over pages starts from the same references and lengths each time (one small copy, in both forms).

With `own` false, run() computes in elementary torch operations; with `own` true it calls the library.
"""
import math
import random

import torch

own = False

BLOCK = 64
F32, F64, BF16, I32, I64 = torch.float32, torch.float64, torch.bfloat16, torch.int32, torch.int64
DEV = "cuda"


# ---------------------------------------------------------------------------------------------- cases

def _select(name, B, W, K, V, dtype, pad=0, done=0.0, banned=0.0, alpha=0.0):
    c = dict(op="select", B=B, W=W, K=K, V=V, dtype=dtype, pad=pad, done=done, banned=banned, alpha=alpha, shape_seed=5)
    return dict(c, name=name) if name else c


def _pages(name, op, P, W, lens, kind="heads", ranks="96x160", H=16, storage="bf16", layers=0, spare=0.25,
           new="fixed:1", skip=0.0, drop=0.0, shape_seed=1):
    c = dict(op=op, P=P, W=W, lens=lens, kind=kind, ranks=ranks, H=H, storage=storage, layers=layers, spare=spare, new=new,
             skip=skip, drop=drop, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, four beams, twice as many candidates as beams: latency
        _select("select_one", 1, 4, 8, 32000, "bf16"),
        # a serving batch: fp32 logits of an odd vocabulary in padded rows, ended beams, banned tokens, a length penalty
        _select("select_batch", 16, 4, 8, 50257, "fp32", pad=47, done=0.1, banned=0.1, alpha=0.6),
        # wide beams, a large vocabulary, the largest batch of the library: every logit is read once
        _select("select_wide", 64, 16, 16, 131072, "bf16"),
        # the headline batch's contexts with four beams each, after a selection
        _pages("fork_beams", "fork", 16, 4, "uniform:2048:4096", drop=0.02),
        # the largest batch, long contexts
        _pages("fork_long", "fork", 256, 4, "uniform:8192:32768", drop=0.02, shape_seed=4),
        # a step of the headline model's 24 layers: one token for each beam, shared last pages copied (short contexts, so
        # that the pools stay a few GB)
        _pages("extend_step", "extend", 16, 4, "uniform:64:512", layers=24, skip=0.05),
        # the same at the highest compression (4-byte granules) in 48 layers, more beams of the one prompt
        _pages("extend_low_rank", "extend", 16, 8, "log:64:1024", ranks="18x30", layers=48, skip=0.05, shape_seed=3),
        # a batch of ragged prompts before their prefill into an LLA-2D cache: only pages and slots
        _pages("extend_prompts", "extend", 64, 1, "fixed:0", kind="2d", layers=1, new="log:1:8192", shape_seed=2),
        # sequences of the headline batch that end
        _pages("free_some", "free", 16, 4, "uniform:2048:4096", drop=0.1),
        # half of the largest batch
        _pages("free_long", "free", 256, 4, "uniform:8192:32768", drop=0.5, shape_seed=4),
        # the headline model's pools, half empty: whole blocks of 24 layers move
        _pages("compact_layers", "compact", 16, 2, "uniform:64:512", layers=24, spare=1.0),
        # many small blocks (LLA-2D), three quarters of them free
        _pages("compact_2d", "compact", 64, 4, "uniform:2048:8192", kind="2d", layers=2, spare=3.0, shape_seed=2),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["select", "select", "fork", "extend", "extend", "free", "compact"])
    if op == "select":
        while True:
            W, V = rng.randint(1, 32), _log(rng, 500, 200000)
            B, dtype = _log(rng, 1, 1024 // W), rng.choice(["bf16", "fp32"])
            if B * W * V * (2 if dtype == "bf16" else 4) <= 64 * 16 * 131072 * 2:
                break
        return _select(None, B, W, min(32, rng.choice([W, 2 * W, rng.randint(1, 32)])), V, dtype, rng.choice([0, 0, rng.randint(1, 64)]),
                       rng.choice([0.0, 0.1, 0.3]), rng.choice([0.0, 0.2]), rng.choice([0.0, 0.6, 1.0]))
    seed = rng.randint(1, 1 << 20)
    if op in ("fork", "free"):
        W = rng.randint(1, 8)
        hi = _log(rng, 100, 32768)
        return _pages(None, op, _log(rng, 1, 1024 // W), W, "uniform:%d:%d" % (hi // 4, hi), drop=rng.choice([0.0, 0.1, 0.5]), shape_seed=seed)
    W = rng.randint(1, 8)
    kind = rng.choice(["heads", "heads", "2d"])
    ranks = rng.choice(["96x160", "72x120", "18x30", "128x128"] if kind == "heads" else ["96x160", "288x480"])
    storage = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    layers = rng.randint(1, 48) if kind == "heads" else rng.randint(1, 4)
    spare = rng.choice([0.25, 1.0, 3.0])
    while True:
        P, hi = _log(rng, 1, 64), _log(rng, 8, 4096)
        c = _pages(None, op, P, W, "uniform:%d:%d" % (hi // 8, hi), kind=kind, ranks=ranks, storage=storage, layers=layers, spare=spare,
                   new=rng.choice(["fixed:1", "fixed:%d" % rng.randint(2, 9), "log:1:%d" % rng.randint(2, 700)]), skip=rng.choice([0.0, 0.1]),
                   shape_seed=seed)
        s = _shape(c)
        if s["num_blocks"] * _block_bytes(c) * layers <= 3 << 30:
            return c
        layers = max(1, layers // 2)


# ---------------------------------------------------------------------------------------------- shapes

def _length(spec, rng):
    kind, *v = spec.split(":")
    v = [int(x) for x in v]
    if kind == "fixed":
        return v[0]
    return rng.randint(v[0], v[1]) if kind == "uniform" else _log(rng, max(1, v[0]), v[1])


def _row_bytes(c):
    """(pages a block has, bytes of a token's K row and V row in each)."""
    rk, rv = (int(x) for x in c["ranks"].split("x"))
    es = 2 if c["storage"] == "bf16" else 4
    return (c["H"] if c["kind"] == "heads" else 1), rk * es, rv * es


def _block_bytes(c):
    pages, k, v = _row_bytes(c)
    return pages * BLOCK * (k + v)


def _up(n):
    return -(-n // BLOCK)


def _shape(c):
    """Who holds which page: per sequence a list of numbers of pages (not yet block ids) and a length; the parents of a
    fork, the sequences of a free, the growth of an extend."""
    rng = random.Random(c["shape_seed"])
    rows, lens, total = [], [], 0
    for _ in range(c["P"]):
        L = _length(c["lens"], rng)
        n = _up(L)
        # the beams continue some of the last step's beams, which went their own ways some pages ago
        last = [rng.randrange(c["W"]) for _ in range(c["W"])]
        trunk = list(range(total, total + n))
        total += n
        branch = {}
        for w in last:
            if w not in branch:
                keep = n if not branch else max(0, n - rng.randint(1, 3))
                branch[w] = trunk[:keep] + list(range(total, total + n - keep))
                total += n - keep
            rows.append(branch[w])
            lens.append(L)
    S = c["P"] * c["W"]
    s = dict(rows=rows, lens=lens, S=S)
    W = c["W"]
    s["parents"] = [-1 if rng.random() < c["drop"] else (i // W) * W + rng.randrange(W) for i in range(S)]
    ended = [i for i in range(S) if rng.random() < c["drop"]]
    rng.shuffle(ended)
    s["ended"] = ended or [S - 1]
    s["skip"] = [1 if rng.random() < c["skip"] else 0 for _ in range(S)]
    uniform = c["new"].startswith("fixed")
    s["new"] = [_length(c["new"], rng) for _ in range(S)]
    s["uniform"] = uniform
    grow = [0 if s["skip"][i] else s["new"][i] for i in range(S)]
    # what a growth needs: fresh pages, and a copy of each shared last page for all but its lowest holder that grows
    # (for that one too where another holds the page and does not grow)
    holders, growers = {}, {}
    for i in range(S):
        if lens[i] % BLOCK:
            t = rows[i][-1]
            holders[t] = holders.get(t, 0) + 1
            if grow[i]:
                growers.setdefault(t, []).append(i)
    s["fresh"] = sum(_up(lens[i] + grow[i]) - _up(lens[i]) for i in range(S))
    s["copies"] = []
    for t, g in growers.items():
        if holders[t] > 1:
            s["copies"] += [lens[i] % BLOCK for i in (g[1:] if len(g) == holders[t] else g)]
    need = (s["fresh"] + len(s["copies"])) if c["op"] == "extend" else 0
    s["live"] = total
    s["num_blocks"] = max(total + need, int(total * (1 + c["spare"])) + need + 1)
    s["max_blocks"] = max(1, max(_up(lens[i] + s["new"][i]) for i in range(S)))
    return s


def work(c):
    if c["op"] == "select":
        rows, es = c["B"] * c["W"], 2 if c["dtype"] == "bf16" else 4
        live = rows - sum(_select_done(c))
        return {"bytes": live * c["V"] * es + rows * 9 + c["B"] * c["K"] * 17, "flops": 4.0 * live * c["V"]}
    s = _shape(c)
    held = sum(len(r) for r in s["rows"])
    if c["op"] == "fork":
        out = [p for p in s["parents"] if p >= 0]
        count = {p: out.count(p) for p in set(out)} if s["S"] <= 64 else {}
        for p in (out if s["S"] > 64 else ()):
            count[p] = count.get(p, 0) + 1
        changed = sum(len(s["rows"][p]) for p in range(s["S"]) if count.get(p, 0) != 1)
        return {"bytes": 4 * sum(len(s["rows"][p]) for p in count) + 4 * sum(len(s["rows"][p]) for p in out) + 8 * changed + 12 * s["S"], "flops": 0}
    if c["op"] == "free":
        return {"bytes": 12 * sum(len(s["rows"][i]) for i in s["ended"]) + 12 * len(s["ended"]), "flops": 0}
    pages, k, v = _row_bytes(c)
    if c["op"] == "extend":
        taken = s["fresh"] + len(s["copies"])
        return {"bytes": 2 * sum(s["copies"]) * pages * (k + v) * c["layers"] + 4 * s["num_blocks"] + 8 * taken + 8 * sum(s["new"]) + 20 * s["S"],
                "flops": 0}
    # the expected moves: live pages are spread evenly, so the share of them behind the first `live` blocks
    moves = s["live"] * (s["num_blocks"] - s["live"]) / s["num_blocks"]
    return {"bytes": 2 * moves * _block_bytes(c) * c["layers"] + 8 * s["num_blocks"] + 8 * held, "flops": 0}


def _select_done(c):
    rng = random.Random(c["shape_seed"])
    done = [1 if rng.random() < c["done"] else 0 for _ in range(c["B"] * c["W"])]
    if c["W"] > 1:
        done[::c["W"]] = [0] * c["B"]  # a sequence whose every beam has ended leaves the batch
    return done


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed, *key):
    s = seed & 0x7fffffff
    for k in key:
        s = (s * 1000003 + k + 1) & 0x7fffffffffff
    return torch.Generator(device=DEV).manual_seed(s)


def prepare(c, seed):
    return _prepare_select(c, seed) if c["op"] == "select" else _prepare_pages(c, seed)


def _prepare_select(c, seed):
    B, W, K, V = c["B"], c["W"], c["K"], c["V"]
    g = _gen(seed, 1)
    ld = V + c["pad"]
    # the beams of a sequence see related logits: a common part, a part of their own, and a few likely tokens
    x = torch.empty(B, W, ld, device=DEV, dtype=BF16 if c["dtype"] == "bf16" else F32)
    for b in range(B):
        x[b] = torch.randn(1, ld, generator=g, device=DEV) * 2.0 + torch.randn(W, ld, generator=g, device=DEV)
        likely = torch.randint(0, V, (W, 12), generator=g, device=DEV)
        x[b].scatter_add_(1, likely, (4 + 8 * torch.rand(W, 12, generator=g, device=DEV)).to(x.dtype))
    if c["banned"]:
        ban = torch.rand(V, generator=g, device=DEV) < c["banned"]
        x[:, :, :V].masked_fill_(ban, -math.inf)
    if ld > V:
        x[:, :, V:] = math.nan  # what follows a row is not read
    st = dict(c=c, logits=x[:, :, :V], scores=-20 - 6 * torch.rand(B, W, generator=g, device=DEV), eos=2 % V,
              finished=torch.tensor(_select_done(c), dtype=torch.uint8, device=DEV).view(B, W),
              lengths=torch.randint(10, 40, (B, 1), generator=g, device=DEV).expand(B, W).to(I32).contiguous())
    if W > 3:
        st["scores"][::3, W - 1] = -math.inf  # a beam that found no continuation
    for n, t in (("parents", I32), ("tokens", I32), ("out_scores", F32), ("out_finished", torch.uint8), ("out_lengths", I32)):
        st[n] = torch.zeros(B, K, dtype=t, device=DEV)
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["workspace"] = torch.empty(lla.lla_beam_select_workspace_size(B, W, V, K, x.dtype), dtype=torch.uint8, device=DEV)
    return st


def _prepare_pages(c, seed):
    s = _shape(c)
    g = _gen(seed, 2)
    S, mb, nb = s["S"], s["max_blocks"], s["num_blocks"]
    ids = torch.randperm(nb, generator=g, device=DEV).to(I32).cpu()
    table = torch.full((S, mb), -1, dtype=I32)
    for i, r in enumerate(s["rows"]):
        table[i, :len(r)] = ids[torch.tensor(r, dtype=I64)] if r else table[i, :0]
    ref = torch.zeros(nb, dtype=I32)
    ref.index_add_(0, table[table >= 0].to(I64), torch.ones(int((table >= 0).sum()), dtype=I32))
    lens = torch.tensor(s["lens"], dtype=I32)
    # one buffer for what a pass changes: references, lengths, tables (each on a 16-byte boundary)
    pad = lambda n: -(-n // 4) * 4  # noqa: E731
    start = torch.zeros(pad(nb) + pad(S) + S * mb, dtype=I32)
    start[:nb], start[pad(nb):pad(nb) + S], start[pad(nb) + pad(S):] = ref, lens, table.reshape(-1)
    start = start.to(DEV)
    led = start.clone()
    st = dict(c=c, s=s, start=start, ledger=led, ref=led[:nb], lens=led[pad(nb):pad(nb) + S], table=led[pad(nb) + pad(S):].view(S, mb))
    st["uniform"] = s["uniform"]
    if c["layers"] and c["op"] in ("extend", "compact"):
        words = nb * _block_bytes(c) // 2
        st["pools"] = torch.empty(c["layers"], words, dtype=torch.int16, device=DEV)
        for l in range(c["layers"]):
            st["pools"][l] = torch.randn(words, generator=g, device=DEV, dtype=BF16).view(torch.int16)
    else:
        st["pools"] = torch.empty(0, 0, dtype=torch.int16, device=DEV)
    dev = lambda v, t=I32: torch.tensor(v, dtype=t, device=DEV)  # noqa: E731
    if c["op"] == "fork":
        st["parents"] = dev(s["parents"])
        st["to_table"], st["to_lens"] = torch.full((S, mb), -1, dtype=I32, device=DEV), torch.zeros(S, dtype=I32, device=DEV)
    elif c["op"] == "free":
        st["ended"] = dev(s["ended"])
    elif c["op"] == "extend":
        cu = [0]
        for n in s["new"]:
            cu.append(cu[-1] + n)
        st["cu_new"], st["skip"] = dev(cu), dev(s["skip"], torch.uint8)
        st["slots"] = torch.zeros(cu[-1], dtype=I64, device=DEV)
        st["before"], st["free"] = torch.zeros(S, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    else:
        st["remap"], st["live"] = torch.zeros(nb, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV)
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["pages"] = lla.Pages(st["ref"], st["table"], st["lens"])
        rk, rv = (int(x) for x in c["ranks"].split("x"))
        geom = lla.Geometry(4, c["H"], 128, rk, rv, c["storage"])
        one = lla.lla_cache_pool if c["kind"] == "heads" else lla.lla_cache_2d_pool
        st["pool_list"] = lla.Pools([one(geom, p) for p in st["pools"]])
        if c["op"] == "fork":
            st["to"] = lla.Pages(st["ref"], st["to_table"], st["to_lens"])
        elif c["op"] == "extend":
            st["workspace"] = torch.empty(lla.lla_pages_extend_workspace_size(S), dtype=torch.uint8, device=DEV)
        elif c["op"] == "compact":
            st["workspace"] = torch.empty(lla.lla_pages_compact_workspace_size(nb), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    c = st["c"]
    if c["op"] == "select":
        (_own_select if own else _plain_select)(st)
        return {n: st[n] for n in ("parents", "tokens", "out_scores", "out_finished", "out_lengths")}
    st["ledger"].copy_(st["start"])
    (_OWN if own else _PLAIN)[c["op"]](st)
    out = {n: st[n] for n in ("ref", "lens", "table")}
    for n in {"fork": ("to_table", "to_lens"), "free": (), "extend": ("pools", "slots", "before", "free"), "compact": ("pools", "remap", "live")}[c["op"]]:
        out[n] = st[n]
    return out


def _own_select(st):
    st["lla"].lla_beam_select(st["logits"], st["scores"], st["parents"], st["tokens"], st["out_scores"], st["workspace"], finished=st["finished"],
                              lengths=st["lengths"], out_finished=st["out_finished"], out_lengths=st["out_lengths"], eos=st["eos"],
                              length_penalty=st["c"]["alpha"])


def _own_fork(st):
    st["lla"].lla_pages_fork(st["pages"], st["to"], st["parents"])


def _own_extend(st):
    st["lla"].lla_pages_extend(st["pages"], st["pool_list"], st["slots"], st["workspace"], cu_new=None if st["uniform"] else st["cu_new"],
                               skip=st["skip"], lens_before=st["before"], free_blocks=st["free"])


def _own_free(st):
    st["lla"].lla_pages_free(st["pages"], st["ended"])


def _own_compact(st):
    st["lla"].lla_pages_compact(st["pages"], st["pool_list"], st["remap"], st["live"], st["workspace"])


_OWN = {"fork": _own_fork, "extend": _own_extend, "free": _own_free, "compact": _own_compact}


def _plain_select(st):
    """Continuations ranked by (score + logit - log sum exp) (length)^-alpha in 64 bits, since neighbours are close; within a beam by logit; ties go to
    the lower beam, then the lower token.  An ended beam continues as itself."""
    c, x = st["c"], st["logits"]
    B, W, K = c["B"], c["W"], c["K"]
    done = st["finished"].bool()
    dead = ~torch.isfinite(st["scores"])
    x = x.to(F32) + 0.0
    x = torch.where(torch.isfinite(x), x, -math.inf)
    top, tok = torch.sort(x, dim=-1, descending=True, stable=True)
    k = min(K, c["V"])
    top, tok = top[..., :k], tok[..., :k]
    m = torch.where(torch.isfinite(top[..., :1]), top[..., :1], 0.0).to(F64)
    log_sum = torch.log(torch.exp(x.to(F64) - m).sum(-1, keepdim=True))
    score = st["scores"].to(F64)[..., None]
    total = score + ((top.to(F64) - m) - log_sum)
    valid = torch.isfinite(top)
    first = torch.arange(k, device=x.device) == 0
    total = torch.where(done[..., None], score, total)
    valid = torch.where(done[..., None], first, valid) & ~dead[..., None]
    tok = torch.where(done[..., None], st["eos"], tok)
    length = torch.where(done, st["lengths"], st["lengths"] + 1)
    key = total * torch.clamp(length, min=1).to(F64)[..., None] ** -c["alpha"]
    key = torch.where(valid, key, -math.inf).view(B, W * k)
    n = min(K, W * k)
    best, at = torch.sort(key, dim=-1, descending=True, stable=True)
    at = at[:, :n]
    got = valid.view(B, W * k).gather(1, at)
    beam = at // k
    row = torch.arange(B, device=x.device)[:, None] * W
    tok = tok.reshape(B, W * k).gather(1, at)
    st["parents"].fill_(-1)
    st["parents"][:, :n] = torch.where(got, row + beam, -1).to(I32)
    st["tokens"].fill_(-1)
    st["tokens"][:, :n] = torch.where(got, tok, -1).to(I32)
    st["out_scores"].fill_(-math.inf)
    st["out_scores"][:, :n] = torch.where(got, total.view(B, W * k).gather(1, at), -math.inf).to(F32)
    st["out_finished"].fill_(1)
    st["out_finished"][:, :n] = (~got | (tok == st["eos"])).to(torch.uint8)
    st["out_lengths"].fill_(0)
    st["out_lengths"][:, :n] = torch.where(got, length.gather(1, beam), 0)


def _held(st):
    """[S][max_blocks]: whether the sequence holds a page there."""
    col = torch.arange(st["table"].shape[1], device=DEV)
    return col < ((st["lens"] + BLOCK - 1) // BLOCK)[:, None]


def _plain_fork(st):
    held, par = _held(st), st["parents"].to(I64)
    some = par >= 0
    p = torch.clamp(par, min=0)
    children = torch.zeros(len(st["lens"]), dtype=I32, device=DEV).index_add_(0, p, some.to(I32))
    change = torch.where(held, (children - 1)[:, None], 0)
    st["to_table"].copy_(torch.where(held[p] & some[:, None], st["table"][p], st["to_table"]))
    st["to_lens"].copy_(torch.where(some, st["lens"][p], 0))
    st["ref"].index_add_(0, torch.where(held, st["table"], 0).reshape(-1).to(I64), change.reshape(-1).to(I32))


def _plain_free(st):
    gone = torch.zeros(len(st["lens"]), dtype=torch.bool, device=DEV)
    gone[st["ended"].to(I64)] = True
    drop = _held(st) & gone[:, None]
    st["ref"].index_add_(0, torch.where(drop, st["table"], 0).reshape(-1).to(I64), -drop.reshape(-1).to(I32))
    st["lens"].masked_fill_(gone, 0)


def _planes(st):
    """The pools as [layers][block][page][granule][token][16-bit word], K-plane and V-plane."""
    c = st["c"]
    pages, k, v = _row_bytes(c)
    g = 16 if k % 16 == 0 else 4
    x = st["pools"].view(c["layers"], -1, pages, BLOCK * (k + v) // 2)
    return x[..., :BLOCK * k // 2].unflatten(-1, (k // g, BLOCK, g // 2)), x[..., BLOCK * k // 2:].unflatten(-1, (1, BLOCK, v // 2))


def _plain_extend(st):
    lens, ref, table = st["lens"], st["ref"], st["table"]
    S, mb = table.shape
    nb = ref.shape[0]
    col = torch.arange(mb, device=DEV)
    seq = torch.arange(S, device=DEV)
    asked = st["cu_new"][1:] - st["cu_new"][:-1]
    n = torch.where(st["skip"].bool(), 0, asked)
    old, new = (lens + BLOCK - 1) // BLOCK, (lens + n + BLOCK - 1) // BLOCK
    rows = lens % BLOCK
    tail = torch.where(old > 0, table.gather(1, torch.clamp(old - 1, min=0)[:, None].to(I64))[:, 0], 0).to(I64)
    part = (rows > 0) & (n > 0) & (ref[tail] > 1)
    growers = torch.zeros(nb, dtype=I32, device=DEV).index_add_(0, tail, part.to(I32))
    lowest = torch.full((nb,), S, dtype=I64, device=DEV).scatter_reduce_(0, tail, torch.where(part, seq, S), "amin")
    copy = part & ~((growers[tail] >= ref[tail]) & (lowest[tail] == seq))
    need = new - old + copy
    base = torch.cumsum(need, 0) - need
    free_first = torch.sort((ref != 0).to(I32), stable=True).indices  # free blocks, lowest first
    free = (ref == 0).sum()
    granted = need.sum() <= free
    # every page column that gets a block: the copied last page, then the fresh ones
    at = base[:, None] + torch.where(col < old[:, None], 0, copy[:, None] + col - old[:, None])
    gets = (((col >= old[:, None]) & (col < new[:, None])) | (copy[:, None] & (col == old[:, None] - 1))) & granted
    ids = free_first[torch.clamp(at, 0, nb - 1)].to(I32)
    table.copy_(torch.where(gets, ids, table))
    ref.index_add_(0, torch.where(gets, ids, 0).reshape(-1).to(I64), gets.reshape(-1).to(I32))
    ref.index_add_(0, tail, -(copy & granted).to(I32))
    st["before"].copy_(lens)
    lens.add_(torch.where(granted, n, 0))
    st["free"].copy_((ref == 0).sum().to(I32))
    who = torch.nonzero(copy & granted)[:, 0]
    if st["c"]["layers"] and len(who):
        src, dst = tail[who], table[who, (old[who] - 1).to(I64)].to(I64)
        keep = (torch.arange(BLOCK, device=DEV) < rows[who][:, None])[:, None, None, :, None]
        for plane in _planes(st):
            for x in plane:
                x[dst] = torch.where(keep, x[src], x[dst])
    i = torch.arange(len(st["slots"]), device=DEV)
    s = torch.searchsorted(st["cu_new"].to(I64), i, right=True) - 1
    pos = st["before"][s] + i - st["cu_new"][s]
    fits = (n[s] > 0) & granted
    block = table[s, torch.where(fits, pos // BLOCK, 0).to(I64)].to(I64)
    st["slots"].copy_(torch.where(fits, block * BLOCK + pos % BLOCK, -1))


def _plain_compact(st):
    ref, table, c = st["ref"], st["table"], st["c"]
    nb = ref.shape[0]
    used = ref != 0
    live = used.sum()
    ids = torch.arange(nb, device=DEV)
    src, dst = torch.nonzero(used & (ids >= live))[:, 0], torch.nonzero(~used & (ids < live))[:, 0]
    remap = torch.where(used, ids, -1)
    remap[src] = dst
    ref[dst] = ref[src]
    ref[src] = 0
    for x in (st["pools"].view(c["layers"], nb, -1) if c["layers"] else ()):
        x[dst] = x[src]
    table.copy_(torch.where(_held(st), remap[torch.clamp(table, min=0).to(I64)].to(I32), table))
    st["remap"].copy_(remap)
    st["live"].copy_(live.to(I32))


_PLAIN = {"fork": _plain_fork, "extend": _plain_extend, "free": _plain_free, "compact": _plain_compact}


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(c, seed):
    """What run() returns for a selection, from its definition, sequence by sequence in numpy's 64 bits; None for the page operators, which
    compute no numbers."""
    if c["op"] != "select":
        return None
    import numpy as np
    st = prepare(c, seed)
    B, W, K = c["B"], c["W"], c["K"]
    scores, done, length = (st[n].cpu().numpy() for n in ("scores", "finished", "lengths"))
    out = {"parents": np.full((B, K), -1, np.int32), "tokens": np.full((B, K), -1, np.int32), "out_scores": np.full((B, K), -np.inf),
           "out_finished": np.ones((B, K), np.uint8), "out_lengths": np.zeros((B, K), np.int32)}
    for b in range(B):
        found = []
        logits = st["logits"][b].to(F64).cpu().numpy()
        for w in range(W):
            if not np.isfinite(scores[b, w]):
                continue
            score, n = float(scores[b, w]), int(length[b, w])
            if done[b, w]:
                found.append((-score * float(max(n, 1)) ** -c["alpha"], w, 0, st["eos"], score, n))
                continue
            ids = np.flatnonzero(np.isfinite(logits[w]))
            if not len(ids):
                continue
            x = logits[w][ids]
            log_sum = math.log(float(np.sum(np.exp(x - np.max(x)))))
            enough = np.partition(x, -K)[-K] if len(x) > K else -np.inf
            near = np.flatnonzero(x >= enough)
            near = near[np.lexsort((ids[near], -x[near]))][:K]
            for r, i in enumerate(near):
                total = score + ((float(x[i]) - float(np.max(x))) - log_sum)
                found.append((-total * float(max(n + 1, 1)) ** -c["alpha"], w, r, int(ids[i]), total, n + 1))
        for k, (_, w, _, token, total, n) in enumerate(sorted(found)[:K]):
            out["parents"][b, k], out["tokens"][b, k], out["out_scores"][b, k] = b * W + w, token, total
            out["out_finished"][b, k], out["out_lengths"][b, k] = token == st["eos"], n
    return out
