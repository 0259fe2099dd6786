"""Many sequences over one prompt, measured: requests that share a prompt's pages, the decode that reads shared pages once for
all of their sequences, and rotary positions with several axes (time, height, width) for images and video.

A case is a dict of plain values.  `op` names the operator:

  prefix   one decode call (one layer, one loop) of a batch whose sequences share pages, each shared page read once for up to 64
           of them; with d_rope > 0 the scores have a rotary branch with positions on three axes
  plan     which sequences share which pages, worked out from the block table
  keys     rotary keys turned at positions with three axes and written into the paged rotary planes
  axes     one decode call with a rotary branch whose current tokens have positions with three axes, nothing shared
  admit    requests that keep a part of a resident sequence: their block table rows, lengths, references, copied rows and slots

Batches come as a tree: `system` tokens that all of the batch has in common, P prompts of `prompt` more tokens, each forked into W
sequences, of which every two share `branch` tokens more, and `own` tokens of each sequence.  "fixed:n", "uniform:lo:hi" and
"log:lo:hi" are drawn from `shape_seed`, so that the work of a case does not depend on the seed of its inputs.  That seed draws the
block ids (a page is anywhere in the pool), the sequences' order and the pages that some have of their own where they are
planned for, latents, queries and weights.

With `own` false, run() computes in elementary torch operations; with `own` true it calls the library.
"""
import math
import random

import torch

own = False

BLOCK, D, T = 64, 128, 4
LEVELS, MEMBERS = 3, 64
F32, F64, BF16, I32, I64 = torch.float32, torch.float64, torch.bfloat16, torch.int32, torch.int64
DEV = "cuda"
LOG_BASE = math.log(10000.0)


# ---------------------------------------------------------------------------------------------- cases

def _attn(name, op, P, W, prompt, own_, system="fixed:0", branch="fixed:0", ranks="96x160", H=16, d_rope=0, io="bf16", pass1=True,
          mu=False, interleaved=False, adjacent=False, shape_seed=1):
    c = dict(op=op, P=P, W=W, prompt=prompt, own=own_, system=system, branch=branch, ranks=ranks, H=H, d_rope=d_rope, io=io, pass1=pass1,
             mu=mu, interleaved=interleaved, adjacent=adjacent, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _plan(name, P, W, prompt, own_, system="fixed:0", branch="fixed:0", min_pages=1, shape_seed=1):
    c = dict(op="plan", P=P, W=W, prompt=prompt, own=own_, system=system, branch=branch, min_pages=min_pages, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _keys(name, N, d_rope, dtype, images, interleaved=False, adjacent=False, skip=0.0, shape_seed=1):
    c = dict(op="keys", N=N, d_rope=d_rope, dtype=dtype, images=images, interleaved=interleaved, adjacent=adjacent, skip=skip,
             shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def _admit(name, residents, lens, n, new, keep, layers, ranks="96x160", H=16, storage="bf16", room=1.0, shape_seed=1):
    c = dict(op="admit", residents=residents, lens=lens, n=n, new=new, keep=keep, layers=layers, ranks=ranks, H=H, storage=storage,
             room=room, shape_seed=shape_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, four samples of a short prompt: latency
        _attn("prefix_one", "prefix", 1, 4, "fixed:768", "uniform:1:64"),
        # the headline batch's contexts with four sequences each, up to eight pages of their own
        _attn("prefix_batch", "prefix", 16, 4, "uniform:2048:4096", "uniform:1:512"),
        # a service: a system prompt for all, documents, samples in two branches; fp32 inputs and outputs, a calibration mean, pass 2
        _attn("prefix_tree", "prefix", 8, 16, "log:1024:8192", "log:1:1024", system="fixed:1024", branch="log:64:512", ranks="72x120",
              io="fp32", pass1=False, mu=True, shape_seed=3),
        # 64 samples of each of two long videos, keys with three axes
        _attn("prefix_video", "prefix", 2, 64, "uniform:12000:16000", "log:16:1024", d_rope=64, shape_seed=2),
        # the plan of the headline batch, made again when a sequence gets a page
        _plan("plan_batch", 16, 4, "uniform:2048:4096", "uniform:1:512"),
        # the plan of the largest batch over long contexts
        _plan("plan_largest", 64, 16, "uniform:8192:32768", "log:16:4096", system="fixed:2048", branch="log:64:2048", shape_seed=4),
        # the rotary keys of a decode step
        _keys("keys_step", 64, 64, "bf16", 0.0),
        # prompts with images before their prefill: 32768 tokens, fp32 keys, the widest branch, some tokens without a slot
        _keys("keys_images", 32768, 96, "fp32", 0.8, interleaved=True, skip=0.05),
        # one user over an image and a question
        _attn("axes_one", "axes", 1, 1, "fixed:768", "fixed:9", d_rope=32),
        # the headline batch with a rotary branch
        _attn("axes_batch", "axes", 16, 1, "uniform:2048:4096", "fixed:0", d_rope=64, interleaved=True),
        # eight requests over four resident prompts, their last pages copied in 24 layers
        _admit("admit_step", 4, "uniform:256:1024", 8, "uniform:16:256", 0.8, 24),
        # a full batch over long documents (tables and slots; short requests behind long kept parts)
        _admit("admit_largest", 64, "uniform:8192:32768", 960, "log:1:4096", 0.9, 0, shape_seed=2),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prefix", "prefix", "prefix", "plan", "keys", "axes", "admit"])
    seed = rng.randint(1, 1 << 20)
    if op == "keys":
        return _keys(None, _log(rng, 1, 32768), rng.choice([16, 32, 48, 64, 96]), rng.choice(["bf16", "fp32"]), rng.choice([0.0, 0.5, 0.9]),
                     rng.random() < 0.5, rng.random() < 0.5, rng.choice([0.0, 0.1]), seed)
    if op == "admit":
        storage = rng.choice(["bf16", "bf16", "fp32"])
        ranks = rng.choice(["96x160", "72x120", "18x30", "128x128"])
        layers = rng.choice([0, 0, 1, rng.randint(2, 24)])
        residents = _log(rng, 1, 64)
        n = _log(rng, 1, LLA_ROWS - residents)
        hi = _log(rng, 16, 1024 if layers else 16384)
        new = _log(rng, 2, 512 if layers else 4096)
        while layers > 1:  # pools of a few GB at most
            c = _admit(None, residents, "log:1:%d" % hi, n, "log:1:%d" % new, 0.8, layers, ranks, 16, storage, 1.0, seed)
            if _admit_shape(c)["num_blocks"] * _block_bytes(c) * layers <= 3 << 30:
                break
            layers, n = layers // 2, max(1, n // 2)
        return _admit(None, residents, "log:1:%d" % hi, n, "log:1:%d" % new, rng.choice([0.5, 0.9]), layers, ranks, 16, storage,
                      rng.choice([1.0, 1.0, 0.7]) if layers <= 1 else 1.0, seed)
    if op == "plan":
        W, hi = rng.randint(2, 32), _log(rng, 1024, 32768)
        P = _log(rng, -(-16 // W), 1024 // W)
        return _plan(None, P, W, "log:%d:%d" % (max(512, hi // 16), hi), "log:1:%d" % _log(rng, 2, 2048),
                     rng.choice(["fixed:0", "fixed:%d" % _log(rng, 16, 4096)]), rng.choice(["fixed:0", "log:1:%d" % _log(rng, 2, 1024)]),
                     rng.choice([1, 1, 2, 4]), seed)
    io, pass1, mu = rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.6, rng.random() < 0.3
    if op == "axes":
        while True:
            P, hi = _log(rng, 1, 128), _log(rng, 64, 8192)
            if P * hi <= 64 * 4096:
                break
        return _attn(None, "axes", P, 1, "log:%d:%d" % (max(1, hi // 8), hi), "fixed:%d" % rng.randint(0, 63), H=rng.randint(1, 16),
                     d_rope=rng.choice([32, 64, 96]), io=io, pass1=pass1, mu=mu, interleaved=rng.random() < 0.5, adjacent=rng.random() < 0.5,
                     shape_seed=seed)
    d_rope = rng.choice([0, 0, 0, 32, 64, 96])
    while True:  # at most as many tokens attended to as in the largest listed case
        W = _log(rng, 1, 128)
        P, prompt, own_, system = _log(rng, 1, 64), _log(rng, 64, 16384), _log(rng, 1, 2048), rng.choice([0, 0, _log(rng, 64, 2048)])
        if P * W <= 512 and P * W * (prompt + own_ + system) <= 1200000:
            break
    return _attn(None, "prefix", P, W, "log:%d:%d" % (max(1, prompt // 4), prompt), "log:1:%d" % own_ if own_ > 1 else "fixed:1",
                 "fixed:%d" % system, rng.choice(["fixed:0", "log:1:%d" % _log(rng, 2, 512)]),
                 "96x160" if d_rope else rng.choice(["96x160", "96x160", "128x128", "72x120"]), rng.randint(1, 16), d_rope, io, pass1, mu,
                 rng.random() < 0.5, rng.random() < 0.5, seed)


# ---------------------------------------------------------------------------------------------- shapes

LLA_ROWS = 1024


def _length(spec, rng):
    kind, *v = spec.split(":")
    v = [int(x) for x in v]
    if kind == "fixed":
        return v[0]
    return rng.randint(v[0], v[1]) if kind == "uniform" else _log(rng, max(1, v[0]), v[1])


def _up(n):
    return -(-n // BLOCK)


def _ranks(c):
    return tuple(int(x) for x in c["ranks"].split("x"))


def _block_bytes(c):
    return c["H"] * BLOCK * sum(_ranks(c)) * (2 if c["storage"] == "bf16" else 4)


def _batch_shape(c):
    """Per sequence its pages (numbers, not yet block ids) and its length.  What a node of the tree has of a page that is not full is
    in the pages of those below it (each has copied it before it wrote there)."""
    rng = random.Random(c["shape_seed"])
    rows, lens, total = [], [], 0

    def grow(pages, length, tokens):
        nonlocal total
        length += tokens
        full = length // BLOCK
        new = list(range(total, total + full - len(pages)))
        total += len(new)
        return pages + new, length

    top = grow([], 0, _length(c["system"], rng))
    for _ in range(c["P"]):
        prompt = grow(*top, _length(c["prompt"], rng))
        for w in range(c["W"]):
            if w % 2 == 0:
                branch = grow(*prompt, _length(c["branch"], rng)) if c["branch"] != "fixed:0" else prompt
            pages, length = grow(*branch, _length(c["own"], rng))
            if length % BLOCK:
                pages = pages + [total]
                total += 1
            if c.get("pass1", True) is False and length == 0:
                pages, length, total = [total], 1, total + 1
            rows.append(pages)
            lens.append(length)
    return dict(rows=rows, lens=lens, B=len(rows), unique=total, num_blocks=total + 1 + total // 8,
                max_blocks=max(1, max(len(r) for r in rows)), max_ctx=max(1, max(lens)))


def _admit_shape(c):
    rng = random.Random(c["shape_seed"])
    lens = [_length(c["lens"], rng) for _ in range(c["residents"])]
    S = c["residents"] + c["n"]
    free_rows = list(range(S))
    rng.shuffle(free_rows)
    home, rows = free_rows[:c["residents"]], free_rows[c["residents"]:]  # row of each resident, row of each request
    parents, keep, new = [], [], []
    for _ in range(c["n"]):
        r = rng.randrange(c["residents"])
        if rng.random() < c["keep"]:
            parents.append(home[r])
            keep.append(rng.randint(lens[r] * 3 // 4, lens[r]))
        else:
            parents.append(-1)
            keep.append(0)
        new.append(keep[-1] + _length(c["new"], rng))
    need = sum(_up(a) - k // BLOCK for a, k in zip(new, keep))
    held = sum(_up(x) for x in lens)
    tokens = sum(a - k for a, k in zip(new, keep))
    return dict(lens=lens, home=home, rows=rows, parents=parents, keep=keep, new=new, S=S, need=need, held=held, tokens=tokens,
                copied=sum(k % BLOCK for k in keep), shared=sum(k // BLOCK for k in keep),
                num_blocks=held + max(1, int(need * c["room"])) + 3, max_blocks=max(1, max(_up(x) for x in lens + new)))


def work(c):
    if c["op"] in ("prefix", "axes"):
        s = _batch_shape(c)
        rk, rv = _ranks(c)
        es, H, B, dr = (2 if c["io"] == "bf16" else 4), c["H"], s["B"], c["d_rope"]
        # tokens whose latents have to be read: each full page once, and the rows in use of the others
        tokens = s["unique"] * BLOCK - sum(-n % BLOCK for n in s["lens"])
        io = B * H * (4 if c["pass1"] else 2) * D * es + (B * (H + 1) * dr * es if dr else 0)
        return {"bytes": tokens * (H * (rk + rv) + dr) * 2 + H * D * (rk + rv) * 2 + io + 4 * s["unique"],
                "flops": 2.0 * sum(s["lens"]) * H * (rk + rv + dr) + 2.0 * B * H * D * (rk + rv)}
    if c["op"] == "plan":
        s = _batch_shape(c)
        return {"bytes": 4 * sum(len(r) for r in s["rows"]) + 4 * s["B"] * (2 + 2 * LEVELS) + 16 * LEVELS * max(1, s["B"] // 2), "flops": 0}
    if c["op"] == "keys":
        N, d = c["N"], c["d_rope"]
        return {"bytes": N * (d * (2 if c["dtype"] == "bf16" else 4) + d * 2 + 12 + 8), "flops": 3.0 * N * d}
    s = _admit_shape(c)
    row = c["H"] * sum(_ranks(c)) * (2 if c["storage"] == "bf16" else 4) * c["layers"]
    return {"bytes": 2 * s["copied"] * row + 4 * s["num_blocks"] + 16 * s["shared"] + 8 * s["need"] + 8 * s["tokens"] + 24 * c["n"], "flops": 0}


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed, *key):
    s = seed & 0x7fffffff
    for k in key:
        s = (s * 1000003 + k + 1) & 0x7fffffffffff
    return torch.Generator(device=DEV).manual_seed(s)


def _pairs(d_rope):
    """Rotation pairs of the three axes: about a half for time, the rest for height and width."""
    third = d_rope // 2 * 3 // 8 // 2 * 2
    return d_rope // 2 - 2 * third, third, third


def _axis_of(d_rope, interleaved):
    """The axis of each pair: one axis after the other, or the axes in turn (the first one where another has no pairs left)."""
    p = _pairs(d_rope)
    if not interleaved:
        return [0] * p[0] + [1] * p[1] + [2] * p[2]
    return [j % 3 if j // 3 < p[j % 3] else 0 for j in range(d_rope // 2)]


def _positions(rng, N, images):
    """[3][N]: text has one position on all axes, an image one time and its row and column."""
    out, pos = [], rng.randint(0, 50000)
    while len(out) < N:
        if rng.random() < images:
            h, w = rng.randint(4, 40), rng.randint(4, 40)
            out += [(pos, pos + y, pos + x) for y in range(h) for x in range(w)]
            pos += max(h, w)
        else:
            n = rng.randint(1, 200)
            out += [(pos + i,) * 3 for i in range(n)]
            pos += n
    return torch.tensor(out[:N], dtype=I32).t().contiguous().to(DEV)


def _rope(st, c):
    lla = st["lla"]
    return lla.RopeAxes(10000.0, lla.LLA_ROPE_ADJACENT if c["adjacent"] else lla.LLA_ROPE_HALF, _pairs(c["d_rope"]),
                        lla.LLA_AXES_INTERLEAVED if c["interleaved"] else lla.LLA_AXES_BLOCKS)


def prepare(c, seed):
    st = {"prefix": _prepare_attn, "axes": _prepare_attn, "plan": _prepare_plan, "keys": _prepare_keys, "admit": _prepare_admit}[c["op"]](c, seed)
    st["c"] = c
    return st


def _table(s, seed):
    ids = torch.randperm(s["num_blocks"], generator=_gen(seed, 1), device=DEV).to(I32).cpu()
    table = torch.full((len(s["rows"]), s["max_blocks"]), -1, dtype=I32)
    for i, r in enumerate(s["rows"]):
        if r:
            table[i, :len(r)] = ids[torch.tensor(r, dtype=I64)]
    return table.to(DEV), torch.tensor(s["lens"], dtype=I32, device=DEV)


def _plan_buffers(B):
    return dict(num_groups=torch.zeros(1, dtype=I32, device=DEV), groups=torch.zeros(LEVELS * max(1, B // 2), 4, dtype=I32, device=DEV),
                members=torch.zeros(LEVELS * B, dtype=I32, device=DEV), column=torch.zeros(LEVELS, B, dtype=I32, device=DEV),
                own_page=torch.zeros(B, dtype=I32, device=DEV))


def _prepare_plan(c, seed):
    s = _batch_shape(c)
    rng = random.Random(seed)
    order = list(range(s["B"]))
    rng.shuffle(order)  # requests have come in any order
    rows, lens, nb = [list(s["rows"][i]) for i in order], [s["lens"][i] for i in order], s["num_blocks"]
    for r in rows:  # some came while their prompt was still being encoded: from a page on, theirs are their own
        if len(r) > 1 and rng.random() < 0.3:
            cut = rng.randrange(1, len(r))
            r[cut:] = range(nb, nb + len(r) - cut)
            nb += len(r) - cut
    s = dict(s, rows=rows, lens=lens, num_blocks=nb)
    table, lens = _table(s, seed)
    st = dict(s=s, table=table, lens=lens, **_plan_buffers(s["B"]))
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["plan"] = lla.Prefix(*(st[n] for n in ("num_groups", "groups", "members", "column", "own_page")))
    return st


def _prepare_attn(c, seed):
    s = _batch_shape(c)
    rk, rv = _ranks(c)
    B, H, nb, dr = s["B"], c["H"], s["num_blocks"], c["d_rope"]
    io = BF16 if c["io"] == "bf16" else F32
    g = _gen(seed, 2)
    normal = lambda *shape, dtype=io, scale=1.0: (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)  # noqa: E731
    table, lens = _table(s, seed)
    st = dict(s=s, table=table, lens=lens, pool=torch.randn(nb, H, BLOCK * (rk + rv), generator=g, device=DEV, dtype=BF16),
              w_up_k=normal(H, T, D, rk, dtype=BF16, scale=rk ** -0.5), w_up_v=normal(H, T, D, rv, dtype=BF16, scale=rv ** -0.5),
              mu_k=normal(H, T * D, dtype=F32) if c["mu"] else None, mu_v=normal(H, T * D, dtype=F32) if c["mu"] else None,
              loop=seed % T, q=normal(B, H, D), cur_k=normal(B, H, D) if c["pass1"] else None, cur_v=normal(B, H, D) if c["pass1"] else None,
              out=torch.zeros(B, H, D, dtype=io, device=DEV))
    if dr:
        rng = random.Random(seed)
        st["planes"] = torch.randn(nb, BLOCK * dr, generator=g, device=DEV, dtype=BF16)
        st["q_rope"], st["cur_k_rope"] = normal(B, H, dr), normal(B, dr) if c["pass1"] else None
        # the next token behind images stands nearer than its index
        st["positions"] = torch.tensor([[max(0, n - rng.randint(0, n // 2)) for n in s["lens"]] for _ in range(3)], dtype=I32, device=DEV)
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["geom"] = lla.Geometry(T, H, D, rk, rv, "bf16")
        down = torch.zeros(16, dtype=BF16, device=DEV)  # (the encode's weights: a decode does not read them)
        st["codec"] = lla.Codec(down, down, st["w_up_k"], st["w_up_v"], st["mu_k"], st["mu_v"])
        st["cache"] = lla.Cache(st["pool"], nb, table, s["max_blocks"])
        if dr:
            st["rope"] = _rope(st, c)
        if c["op"] == "prefix":
            st["plan"] = lla.Prefix(*_plan_buffers(B).values())
            lla.lla_prefix_plan(st["cache"], lens, s["max_ctx"], st["plan"])
            size = lla.lla_decode_prefix_workspace_size(st["geom"], B, dr)
        else:
            size = lla.lla_decode_decoupled_workspace_size(st["geom"], dr, B)
        st["workspace"] = torch.zeros(size, dtype=torch.uint8, device=DEV)
    return st


def _prepare_keys(c, seed):
    N, dr = c["N"], c["d_rope"]
    g = _gen(seed, 3)
    rng = random.Random(c["shape_seed"] * 7919 + seed)
    nb = _up(N) + 1 + _up(N) // 4
    slots = torch.randperm(nb, generator=g, device=DEV)[:_up(N)].repeat_interleave(BLOCK)[:N] * BLOCK + torch.arange(N, device=DEV) % BLOCK
    if c["skip"]:
        slots = torch.where(torch.rand(N, generator=g, device=DEV) < c["skip"], -1, slots)
    st = dict(nb=nb, slots=slots, positions=_positions(rng, N, c["images"]),
              keys=torch.randn(N, dr, generator=g, device=DEV).to(BF16 if c["dtype"] == "bf16" else F32),
              planes=torch.randn(nb, BLOCK * dr, generator=g, device=DEV, dtype=BF16))
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["rope"] = _rope(st, c)
    return st


def _prepare_admit(c, seed):
    s = _admit_shape(c)
    g = _gen(seed, 4)
    S, mb, nb, n = s["S"], s["max_blocks"], s["num_blocks"], c["n"]
    ids = torch.randperm(nb, generator=g, device=DEV).to(I32).cpu()
    table, ref, lens, at = torch.full((S, mb), -1, dtype=I32), torch.zeros(nb, dtype=I32), torch.zeros(S, dtype=I32), 0
    for length, row in zip(s["lens"], s["home"]):
        k = _up(length)
        table[row, :k], lens[row] = ids[at:at + k], length
        ref[ids[at:at + k].to(I64)] = 1
        at += k
    pad = lambda k: -(-k // 4) * 4  # noqa: E731
    # one buffer for what a pass changes: references, lengths, tables (each on a 16-byte boundary)
    start = torch.zeros(pad(nb) + pad(S) + S * mb, dtype=I32)
    start[:nb], start[pad(nb):pad(nb) + S], start[pad(nb) + pad(S):] = ref, lens, table.reshape(-1)
    start = start.to(DEV)
    led = start.clone()
    dev = lambda v: torch.tensor(v, dtype=I32, device=DEV)  # noqa: E731
    st = dict(s=s, start=start, ledger=led, ref=led[:nb], lens=led[pad(nb):pad(nb) + S], table=led[pad(nb) + pad(S):].view(S, mb),
              rows=dev(s["rows"]), parents=dev(s["parents"]), keep=dev(s["keep"]), new=dev(s["new"]),
              slots=torch.zeros(max(1, s["tokens"]), dtype=I64, device=DEV), cu_new=torch.zeros(n + 1, dtype=I32, device=DEV),
              admitted=torch.zeros(n, dtype=torch.uint8, device=DEV), free=torch.zeros(1, dtype=I32, device=DEV))
    words = nb * _block_bytes(c) // 2
    st["pools"] = torch.empty(c["layers"], words if c["layers"] else 0, dtype=torch.int16, device=DEV)
    for layer in range(c["layers"]):
        st["pools"][layer] = torch.randn(words, generator=g, device=DEV, dtype=BF16).view(torch.int16)
    if own:
        from paper_2607_15456_gb300 import lla
        st["lla"] = lla
        st["pages"] = lla.Pages(st["ref"], st["table"], st["lens"])
        geom = lla.Geometry(T, c["H"], D, *_ranks(c), c["storage"])
        st["pool_list"] = lla.Pools([lla.lla_cache_pool(geom, p) for p in st["pools"]])
        st["workspace"] = torch.empty(lla.lla_pages_admit_workspace_size(n), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(st):
    op = st["c"]["op"]
    if op == "admit":
        st["ledger"].copy_(st["start"])
    (_OWN if own else _PLAIN)[op](st)
    if op in ("prefix", "axes"):
        return st["out"]
    if op == "keys":
        return st["planes"]
    return {n: st[n] for n in (("num_groups", "groups", "members", "column", "own_page") if op == "plan" else
                               ("ref", "lens", "table", "pools", "slots", "cu_new", "admitted", "free"))}


def _own_attn(st):
    c, lla, s = st["c"], st["lla"], st["s"]
    if c["op"] == "axes":
        lla.lla_decode_attn_decoupled_axes(st["geom"], st["codec"], st["cache"], st["planes"], c["d_rope"], st["rope"], st["positions"], st["lens"],
                                           s["max_ctx"], st["loop"], st["q"], st["q_rope"], st["cur_k"], st["cur_v"], st["cur_k_rope"],
                                           st["out"], st["workspace"])
    elif c["d_rope"]:
        lla.lla_decode_attn_prefix_decoupled(st["geom"], st["codec"], st["cache"], st["plan"], st["planes"], c["d_rope"], st["rope"],
                                             st["positions"], st["lens"], s["max_ctx"], st["loop"], st["q"], st["q_rope"], st["cur_k"],
                                             st["cur_v"], st["cur_k_rope"], st["out"], st["workspace"])
    else:
        lla.lla_decode_attn_prefix(st["geom"], st["codec"], st["cache"], st["plan"], st["lens"], s["max_ctx"], st["loop"], st["q"],
                                   st["cur_k"], st["cur_v"], st["out"], st["workspace"])


def _own_plan(st):
    st["lla"].lla_prefix_plan(_cache_of(st), st["lens"], st["s"]["max_ctx"], st["plan"], min_pages=st["c"]["min_pages"])


def _cache_of(st):
    # a plan reads the block table alone
    return st["lla"].Cache(None, st["s"]["num_blocks"], st["table"], st["s"]["max_blocks"])


def _own_keys(st):
    st["lla"].lla_encode_rope_keys_axes(st["c"]["d_rope"], st["rope"], st["planes"], st["nb"], st["keys"], st["positions"], st["slots"])


def _own_admit(st):
    st["lla"].lla_pages_admit(st["pages"], st["pool_list"], st["rows"], st["parents"], st["keep"], st["new"], st["slots"], st["cu_new"],
                              st["admitted"], st["workspace"], free_blocks=st["free"])


_OWN = {"prefix": _own_attn, "axes": _own_attn, "plan": _own_plan, "keys": _own_keys, "admit": _own_admit}


def _turns(c, positions, dtype=F64):
    """cos and sin of every pair at positions [3][N]: angles in 64 bits, since positions are far."""
    hp = c["d_rope"] // 2
    axis = torch.tensor(_axis_of(c["d_rope"], c["interleaved"]), device=DEV)
    theta = torch.exp(torch.arange(hp, device=DEV, dtype=F64) * (-LOG_BASE / hp))
    a = positions.to(F64)[axis].t() * theta
    return torch.cos(a).to(dtype), torch.sin(a).to(dtype)


def _turn(c, x, cos, sin):
    """x [..., d_rope] with its pairs turned."""
    hp = c["d_rope"] // 2
    if c["adjacent"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    a, b = x[..., :hp], x[..., hp:]
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def _plane(x, r):
    """[n][64 r] in granules of 8 columns as [n][64][r]."""
    return x.view(*x.shape[:-1], r // 8, BLOCK, 8).transpose(-3, -2).reshape(*x.shape[:-1], BLOCK, r)


def _plain_attn(st):
    """Absorbed attention of every sequence over its own table row, in 32 bits, a few sequences at a time."""
    c, s = st["c"], st["s"]
    rk, rv = _ranks(c)
    dr, B, H = c["d_rope"], s["B"], c["H"]
    t, scale = st["loop"], D ** -0.5
    q = st["q"].to(F32)
    wk, wv = st["w_up_k"][:, t].to(F32), st["w_up_v"][:, t].to(F32)  # [H][D][r]
    qt = torch.einsum("bhd,hdr->bhr", q, wk)
    beta = (q * st["mu_k"].view(H, T, D)[:, t]).sum(-1) if c["mu"] else torch.zeros(B, H, device=DEV)
    if dr:
        cos, sin = _turns(c, st["positions"], F32)
        qr = _turn(c, st["q_rope"].to(F32), cos[:, None], sin[:, None])
    lens = s["lens"]
    b0 = 0
    while b0 < B:
        b1, top = b0 + 1, _up(lens[b0])
        while b1 < B and (b1 + 1 - b0) * max(top, _up(lens[b1])) * BLOCK * H * (rk + rv) <= 1 << 30:
            top = max(top, _up(lens[b1]))
            b1 += 1
        n, N = b1 - b0, top * BLOCK
        parts = []
        if N:
            ids = torch.clamp(st["table"][b0:b1, :top], min=0).reshape(-1).to(I64)
            page = st["pool"][ids]
            ck = _plane(page[..., :BLOCK * rk], rk).view(n, top, H, BLOCK, rk).transpose(1, 2).reshape(n, H, N, rk).to(F32)
            cv = page[..., BLOCK * rk:].view(n, top, H, BLOCK, rv).transpose(1, 2).reshape(n, H, N, rv).to(F32)
            x = (ck @ qt[b0:b1, :, :, None])[..., 0] + beta[b0:b1, :, None]
            if dr:
                kr = _plane(st["planes"][ids], dr).view(n, 1, N, dr).to(F32)
                x = x + (kr @ qr[b0:b1, :, :, None])[..., 0]
            hold = torch.arange(N, device=DEV) < st["lens"][b0:b1, None]
            parts.append(torch.where(hold[:, None], x * scale, -math.inf))
        if c["pass1"]:
            now = (q[b0:b1] * st["cur_k"][b0:b1].to(F32)).sum(-1)
            if dr:  # both stand at one position
                now = now + (st["q_rope"][b0:b1].to(F32) * st["cur_k_rope"][b0:b1, None].to(F32)).sum(-1)
            parts.append(now[..., None] * scale)
        x = torch.cat(parts, -1)
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        o = torch.zeros(n, H, D, device=DEV)
        if N:
            cv = torch.where(hold[:, None, :, None], cv, 0.0)
            o = torch.einsum("bhr,hdr->bhd", (p[..., None, :N] @ cv)[..., 0, :], wv)
            if c["mu"]:
                o = o + p[..., :N].sum(-1, keepdim=True) * st["mu_v"].view(H, T, D)[:, t]
        if c["pass1"]:
            o = o + p[..., -1:] * st["cur_v"][b0:b1].to(F32)
        st["out"][b0:b1] = o.to(st["out"].dtype)
        b0 = b1


def _plain_plan(st):
    """Level by level: the sequences of a set (at first all) that have the same block in the set's next full page form a set of
    their own, whose pages go on as long as all of them agree.  One of two sequences and min_pages pages at least becomes groups of at
    most 64 members, evenly; sets are ordered by their lowest sequence, members by number."""
    table, lens, c = st["table"], st["lens"], st["c"]
    B, MB = table.shape
    seq, col = torch.arange(B, device=DEV), torch.arange(MB, device=DEV)
    full = torch.div(lens, BLOCK, rounding_mode="floor")
    alive, lead, page = torch.ones(B, dtype=torch.bool, device=DEV), torch.zeros(B, dtype=I64, device=DEV), torch.zeros(B, dtype=I64, device=DEV)
    groups, members = torch.zeros_like(st["groups"]), torch.full_like(st["members"], -1)
    num, filled = torch.zeros((), dtype=I64, device=DEV), torch.zeros((), dtype=I64, device=DEV)
    for level in range(LEVELS):
        alive = alive & (full > page)
        block = torch.where(alive, table.gather(1, torch.clamp(page, max=MB - 1)[:, None])[:, 0], -1)
        same = alive[:, None] & alive & (lead[:, None] == lead) & (block[:, None] == block)
        n = same.sum(1)
        lead_new = torch.where(alive, same.to(I32).argmax(1), seq)
        both = torch.minimum(full, full[lead_new])
        differ = (col >= page[:, None]) & ((table != table[lead_new]) | (col >= both[:, None]))
        end = torch.where(differ.any(1), differ.to(I32).argmax(1), MB)
        end = torch.full((B,), MB, dtype=I64, device=DEV).scatter_reduce_(0, lead_new, end, "amin")[lead_new]
        ok = alive & (n >= 2) & (end - page >= c["min_pages"])
        rank = (same & (seq[None, :] < seq[:, None])).sum(1)
        k = torch.div(n + MEMBERS - 1, MEMBERS, rounding_mode="floor")
        first = ok & (lead_new == seq)
        k_lead, n_lead = torch.where(first, k, 0), torch.where(first, n, 0)
        group0 = num + (torch.cumsum(k_lead, 0) - k_lead)[lead_new]
        member0 = filled + (torch.cumsum(n_lead, 0) - n_lead)[lead_new]
        part = torch.div((rank + 1) * k - 1, torch.clamp(n, min=1), rounding_mode="floor")
        begin = torch.div(part * n, torch.clamp(k, min=1), rounding_mode="floor")
        size = torch.div((part + 1) * n, torch.clamp(k, min=1), rounding_mode="floor") - begin
        group = group0 + part
        st["column"][level] = torch.where(ok, group * MEMBERS + rank - begin, -1).to(I32)
        who = torch.nonzero(ok)[:, 0]
        members[(member0 + rank)[who]] = who.to(I32)
        groups[group[who]] = torch.stack((page, end, member0 + begin, size), 1)[who].to(I32)
        num, filled = num + k_lead.sum(), filled + n_lead.sum()
        page = torch.where(ok, end, page)
        alive, lead = ok, lead_new
    st["own_page"].copy_(page)
    st["groups"].copy_(groups)
    st["members"].copy_(members)
    st["num_groups"].copy_(num)


def _plain_keys(st):
    c, slots = st["c"], st["slots"]
    cos, sin = _turns(c, st["positions"], F32)
    x = _turn(c, st["keys"].to(F32), cos, sin).to(BF16)
    who = torch.nonzero(slots >= 0)[:, 0]
    planes = st["planes"].view(st["nb"], c["d_rope"] // 8, BLOCK, 8)
    planes[torch.div(slots[who], BLOCK, rounding_mode="floor"), :, slots[who] % BLOCK] = x[who].view(-1, c["d_rope"] // 8, 8)


def _plain_admit(st):
    """Requests in order as long as their blocks (the free ones of the lowest numbers) and their tokens find room."""
    c, s, ref, table, lens = st["c"], st["s"], st["ref"], st["table"], st["lens"]
    n, mb, nb = c["n"], s["max_blocks"], s["num_blocks"]
    up = lambda x: torch.div(x + BLOCK - 1, BLOCK, rounding_mode="floor")  # noqa: E731
    rows, par, keep, new = (st[k].to(I64) for k in ("rows", "parents", "keep", "new"))
    shared, copied = keep // BLOCK, keep % BLOCK
    need = up(new) - shared
    free = (ref == 0).sum()
    ok = (torch.cumsum(need, 0) <= free) & (torch.cumsum(new - keep, 0) <= len(st["slots"]))
    need, tokens = torch.where(ok, need, 0), torch.where(ok, new - keep, 0)
    base = torch.cumsum(need, 0) - need
    free_first = torch.sort((ref != 0).to(I32), stable=True).indices
    col = torch.arange(mb, device=DEV)
    fresh = free_first[torch.clamp(base[:, None] + col - shared[:, None], 0, nb - 1)].to(I32)
    kept = table[torch.clamp(par, min=0)]
    is_kept = ok[:, None] & (col < shared[:, None])
    is_fresh = ok[:, None] & (col >= shared[:, None]) & (col < up(new)[:, None])
    mine = torch.where(is_kept, kept, torch.where(is_fresh, fresh, table[rows]))
    table[rows] = mine
    got = is_kept | is_fresh
    ref.index_add_(0, torch.where(got, mine, 0).reshape(-1).to(I64), got.reshape(-1).to(I32))
    lens[rows] = torch.where(ok, new, lens[rows].to(I64)).to(I32)
    who = torch.nonzero(ok & (copied > 0))[:, 0]
    if c["layers"] and len(who):
        rk, rv = _ranks(c)
        es = 1 if c["storage"] == "bf16" else 2  # 16-bit words of an element
        src, dst = kept[who, shared[who]].to(I64), mine[who, shared[who]].to(I64)
        hold = (torch.arange(BLOCK, device=DEV) < copied[who, None])[:, None, None, :, None]
        gk = 8 if rk * es % 8 == 0 else 2  # words of a granule
        x = st["pools"].view(c["layers"], nb, c["H"], -1)
        for layer in x:
            k = layer[..., :BLOCK * rk * es].unflatten(-1, (rk * es // gk, BLOCK, gk))
            v = layer[..., BLOCK * rk * es:].unflatten(-1, (1, BLOCK, rv * es))
            for y in (k, v):
                y[dst] = torch.where(hold, y[src], y[dst])
    st["cu_new"][0] = 0
    st["cu_new"][1:] = torch.cumsum(tokens, 0)
    st["admitted"].copy_(ok)
    st["free"].copy_(free - need.sum())
    i = torch.arange(len(st["slots"]), device=DEV)
    r = torch.clamp(torch.searchsorted(st["cu_new"].to(I64), i, right=True) - 1, max=n - 1)
    pos = keep[r] + i - st["cu_new"][r]
    fits = i < st["cu_new"][n]
    block = mine[r, torch.where(fits, pos // BLOCK, 0)].to(I64)
    st["slots"].copy_(torch.where(fits, block * BLOCK + pos % BLOCK, -1))


_PLAIN = {"prefix": _plain_attn, "axes": _plain_attn, "plan": _plain_plan, "keys": _plain_keys, "admit": _plain_admit}


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(c, seed):
    """What run() returns, from the definition in 64 bits: keys and values rebuilt for every token, sequence by sequence; None for the
    operators that compute no numbers."""
    if c["op"] in ("plan", "admit"):
        return None
    st = prepare(c, seed)
    hp = c["d_rope"] // 2
    axis = _axis_of(c["d_rope"], c["interleaved"]) if hp else []

    def rotate(x, where):  # x [..., d_rope] as complex numbers, `where` [3]
        z = torch.complex(x[..., 0::2], x[..., 1::2]) if c["adjacent"] else torch.complex(x[..., :hp], x[..., hp:])
        angle = torch.stack([where[a].to(F64) * 10000.0 ** (-j / hp) for j, a in enumerate(axis)], -1)
        z = z * torch.polar(torch.ones_like(angle), angle)
        return torch.view_as_real(z).flatten(-2) if c["adjacent"] else torch.cat((z.real, z.imag), -1)

    if c["op"] == "keys":
        out = st["planes"].to(F64)
        rows = out.view(st["nb"], c["d_rope"] // 8, BLOCK, 8).permute(0, 2, 1, 3).reshape(st["nb"] * BLOCK, -1)
        hold = st["slots"] >= 0
        rows[st["slots"][hold]] = rotate(st["keys"].to(F64), st["positions"])[hold]
        return rows.view(st["nb"], BLOCK, c["d_rope"] // 8, 8).permute(0, 2, 1, 3).reshape(out.shape)
    rk, rv = _ranks(c)
    s, H, t = st["s"], c["H"], st["loop"]
    if 2.0 * sum(s["lens"]) * H * D * (rk + rv) > 4e12:
        return None
    out = torch.zeros(st["out"].shape, dtype=F64, device=DEV)
    wk, wv = (st[w][:, t].to(F64) for w in ("w_up_k", "w_up_v"))
    for b, n in enumerate(s["lens"]):
        q = st["q"][b].to(F64)
        scores, values = [], []
        if n:
            ids = st["table"][b, :_up(n)].to(I64)
            page = st["pool"][ids].to(F64)  # [pages][H][64 (rk + rv)]
            ck = page[..., :BLOCK * rk].view(-1, H, rk // 8, BLOCK, 8).permute(1, 0, 3, 2, 4).reshape(H, -1, rk)[:, :n]
            cv = page[..., BLOCK * rk:].view(-1, H, BLOCK, rv).permute(1, 0, 2, 3).reshape(H, -1, rv)[:, :n]
            key, val = ck @ wk.transpose(1, 2), cv @ wv.transpose(1, 2)
            if c["mu"]:
                key, val = (x + st[m].to(F64).view(H, T, 1, D)[:, t] for x, m in ((key, "mu_k"), (val, "mu_v")))
            x = (key @ q[:, :, None])[..., 0]
            if hp:
                kr = st["planes"][ids].to(F64).view(-1, 2 * hp // 8, BLOCK, 8).permute(0, 2, 1, 3).reshape(-1, 2 * hp)[:n]
                x = x + rotate(st["q_rope"][b].to(F64), st["positions"][:, b]) @ kr.t()
            scores.append(x)
            values.append(val)
        if c["pass1"]:
            x = (q * st["cur_k"][b].to(F64)).sum(-1, keepdim=True)
            if hp:
                x = x + st["q_rope"][b].to(F64) @ st["cur_k_rope"][b].to(F64)[:, None]
            scores.append(x)
            values.append(st["cur_v"][b].to(F64)[:, None])
        p = torch.softmax(torch.cat(scores, -1) / math.sqrt(D), -1)
        out[b] = (p[:, None] @ torch.cat(values, 1))[:, 0]
    return out
