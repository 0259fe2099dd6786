"""lla_beam_search: what the model's callback is given and what becomes of the search where a beam dies or pages run out."""
import gc
import math
import weakref

import pytest
import torch

from helpers import ensure_library
from paper_2607_15456_gb300 import workloads

pytestmark = pytest.mark.gpu

DEV = "cuda"
I32, I64, U8, F32 = torch.int32, torch.int64, torch.uint8, torch.float32


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


@pytest.fixture(autouse=True)
def no_error_left(lla):
    lla.lla_clear_device_error()
    yield
    assert lla.lla_get_device_error() == 0


class Search:
    """Page sets, slabs and workspace of a search without pools."""

    def __init__(self, lla, B, W, V, steps, blocks=64, max_blocks=4):
        self.lla, self.B, self.W, self.V, self.steps = lla, B, W, V, steps
        S = B * W
        self.ref = torch.zeros(blocks, dtype=I32, device=DEV)
        self.pages = [lla.Pages(self.ref, torch.full((S, max_blocks), -1, dtype=I32, device=DEV), torch.zeros(S, dtype=I32, device=DEV)) for _ in range(2)]
        self.tokens, self.lengths = (torch.zeros(steps + 1, B, W, dtype=I32, device=DEV) for _ in range(2))
        self.finished = torch.zeros(steps + 1, B, W, dtype=U8, device=DEV)
        self.parents = torch.zeros(steps, B, W, dtype=I32, device=DEV)
        self.scores = torch.full((steps + 1, B, W), -math.inf, device=DEV)
        self.scores[0, :, 0] = 0
        self.ws = torch.full((lla.lla_beam_search_workspace_size(B, W, V, F32),), 0xA5, dtype=U8, device=DEV)

    def run(self, step, pools=None, **kw):
        self.lla.lla_beam_search(*self.pages, pools or self.lla.Pools(), self.V, step, self.tokens, self.scores, self.finished, self.lengths, self.parents,
                                 self.ws, dtype=F32, **kw)
        return self

    def prompt(self, lens):
        """Every sequence's prompt of lens[b] cached tokens, forked into its beams."""
        first = self.lla.Pages(self.ref, torch.full((self.B, self.pages[0].block_table.shape[1]), -1, dtype=I32, device=DEV),
                               torch.zeros(self.B, dtype=I32, device=DEV))
        ws = torch.empty(self.lla.lla_pages_extend_workspace_size(self.B), dtype=U8, device=DEV)
        cu = torch.tensor([0] + lens, dtype=I32, device=DEV).cumsum(0).to(I32)
        self.lla.lla_pages_extend(first, self.lla.Pools(), torch.zeros(sum(lens), dtype=I64, device=DEV), ws, cu_new=cu)
        self.lla.lla_pages_fork(first, self.pages[0], (torch.arange(self.B * self.W, device=DEV) // self.W).to(I32))
        return self

    def last(self):
        return self.pages[self.steps % 2]

    def check_ledger(self):
        """Every block is held as often as the last set's tables hold it."""
        count, last = [0] * len(self.ref), self.last()
        table = last.block_table.tolist()
        for s, n in enumerate(last.context_lens.tolist()):
            for b in table[s][:-(-n // 64)]:
                count[b] += 1
        assert self.ref.tolist() == count


def test_logits_of_earlier_steps_are_let_go(lla):
    """Each step's logits are needed until its selection is enqueued: at most the last step's are alive in the callback, and
    the memory that the search takes does not grow with its steps."""
    s = Search(lla, 4, 8, 50000, 30)  # 6.4 MB a step
    base = torch.randn(s.B, s.W, s.V, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    refs, alive = [], []

    def step(i, *_):
        gc.collect()
        alive.append(sum(r() is not None for r in refs))
        z = base + float(i)
        refs.append(weakref.ref(z))
        return z

    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    s.run(step)
    assert max(alive) <= 1
    assert torch.cuda.max_memory_allocated() - before <= 4 * base.numel() * 4


def test_logits_from_another_stream(lla):
    """The memory of logits that were made on a stream of the model's own is not handed out again before the selection has read
    it: the hypotheses are those of logits that are all kept."""
    side = torch.cuda.Stream()
    results = []
    for keep in (True, False):
        s, kept = Search(lla, 4, 8, 50000, 20), []
        base = torch.randn(s.B, s.W, s.V, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
        torch.cuda.synchronize()

        def step(i, *_):
            here = torch.cuda.current_stream()
            with torch.cuda.stream(side):
                z = base.roll(i * 977, 2)
                here.wait_stream(side)
                if keep:
                    kept.append(z)
            return z

        s.run(step)
        torch.cuda.synchronize()
        results.append((s.tokens, s.parents, s.scores))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def masked(s, step, open_tokens, seed=5):
    """Logits with only the tokens open_tokens[b] finite."""
    g = torch.Generator(device=DEV).manual_seed(seed * 1000 + step)
    z = torch.full((s.B, s.W, s.V), -math.inf, device=DEV)
    for b, ids in enumerate(open_tokens):
        z[b][:, ids] = torch.randn(s.W, len(ids), generator=g, device=DEV)
    return z


def test_dead_beams(lla):
    """Sequence 0 has two continuations a beam in the first two steps, so two of its four beams die in the first and come back
    in the second; sequence 1 has none at step 2 and is dead from there on; sequence 2 is as usual.  The model is
    given a token of the vocabulary and a sequence that is not empty for every beam, dead ones too, and its decode reports
    nothing; a dead beam keeps the pages that it had and does not grow."""
    B, W, V, steps = 3, 4, 50, 6
    s = Search(lla, B, W, V, steps).prompt([5, 63, 128])
    allowed = lambda i: [[3, 7] if i < 2 else list(range(V)), list(range(V)) if i != 2 else [], list(range(V))]
    geom = lla.Geometry(1, 1, 128, 96, 160)
    g = torch.Generator(device=DEV).manual_seed(1)
    rnd = lambda *n: torch.randn(*n, generator=g, device=DEV)
    codec = lla.Codec(**workloads.codec_tensors(1, 1, 128, 96, 160, 3, 0, device=DEV))
    pool = torch.zeros(len(s.ref) * lla.lla_cache_block_bytes(geom), dtype=U8, device=DEV)
    dws = torch.zeros(lla.lla_decode_workspace_size(geom, B * W), dtype=U8, device=DEV)
    seen = []

    def step(i, pages, before, toks, slots):
        seen.append([t.clone() for t in (toks, before, pages.context_lens, slots)])
        out = torch.empty(B * W, 1, 128, dtype=F32, device=DEV)
        cache = lla.Cache(pool, len(s.ref), pages.block_table, 4)
        lla.lla_decode_attn(geom, codec, cache, pages.context_lens, 256, 0, rnd(B * W, 1, 128), None, None, out, dws)  # pass 2
        assert torch.isfinite(out).all()
        return masked(s, i, allowed(i))

    s.run(step, pools=[lla.lla_cache_pool(geom, pool)])
    assert lla.lla_get_device_error() == 0
    tokens, parents, finished, lengths = (t.tolist() for t in (s.tokens, s.parents, s.finished, s.lengths))
    # dead where there is no continuation: two in sequence 0 at the first step; all of sequence 1 from step 2 on
    dead = [[[p < 0 for p in row] for row in slab] for slab in parents]
    assert [sum(d) for d in dead[0]] == [2, 0, 0] and [sum(d) for d in dead[1]] == [0, 0, 0]
    assert [[sum(d) for d in slab] for slab in dead[2:]] == [[0, 4, 0]] * (steps - 2)
    for i in range(steps):
        toks, before, lens, slots = (t.view(B, W).tolist() for t in seen[i])
        for b in range(B):
            for w in range(W):
                was_dead = i > 0 and dead[i - 1][b][w]
                if was_dead:  # the slabs say so; the model gets a token that it can look up
                    assert tokens[i][b][w] == -1 and finished[i][b][w] == 1 and lengths[i][b][w] == 0 and s.scores[i, b, w] == -math.inf
                    # the pages of its last step, as they are
                    assert toks[b][w] == 0 and slots[b][w] == -1 and lens[b][w] == before[b][w] == seen[i - 1][2].view(B, W)[b, w]
                else:
                    assert toks[b][w] == tokens[i][b][w] and slots[b][w] >= 0 and lens[b][w] == before[b][w] + 1
                assert lens[b][w] > 0
    s.check_ledger()
    lla.lla_pages_free(s.last(), torch.arange(B * W, dtype=I32, device=DEV))
    assert not s.ref.any()


def test_ended_beams_without_an_ending_token(lla):
    """With eos = -1 a beam that the caller marks as ended has token -1 in the slabs; the model is given one that it can look up."""
    s = Search(lla, 1, 3, 40, 3).prompt([10])
    s.finished[0, 0, 1] = 1
    s.scores[0, 0, 1] = 1.0
    seen = []

    def step(i, pages, before, toks, slots):
        seen.append(toks.clone())
        return masked(s, i, [list(range(s.V))])

    s.run(step)
    assert (s.tokens[1:, 0, 0] == -1).all() and (s.parents[1:, 0, 0] == 0).all()
    assert all((t >= 0).all() and (t < s.V).all() for t in seen)


@pytest.mark.parametrize("why", ["pages", "context"])
def test_growth_that_fails(lla, why):
    """A beam whose token finds no room has no continuation, so that no hypothesis with a hole goes on: from the step that fails
    only the beam that has ended is left, and the first slab of parents with -1 says which step that was."""
    B, W, V, steps, eos = 1, 3, 30, 5, 4
    if why == "pages":  # 64 cached tokens: each beam takes a block in step 0, the other two of the four are free in step 1, until one is taken
        s, error = Search(lla, B, W, V, steps, blocks=4).prompt([64]), lla.LLA_DEVERR_PAGES
    else:               # a row of one page: step 0 fills it
        s, error = Search(lla, B, W, V, steps, blocks=8, max_blocks=1).prompt([63]), lla.LLA_DEVERR_CONTEXT
    seen = []

    def step(i, pages, before, toks, slots):
        seen.append([t.clone() for t in (slots, pages.context_lens, toks)])
        z = masked(s, i, [list(range(V))])
        if i == 0:
            z[:, :, eos] = 9.0  # the best continuation ends
            if why == "pages":
                s.ref[3] += 1   # another user of the pool
        return z

    s.run(step, eos=eos)
    assert lla.lla_get_device_error() == error
    lla.lla_clear_device_error()
    assert s.parents[0].tolist() == [[0, 0, 0]] and s.finished[1].tolist() == [[1, 0, 0]]
    for i in range(1, steps):
        assert s.parents[i].tolist() == [[0, -1, -1]], i
        assert s.tokens[i + 1].tolist() == [[eos, -1, -1]] and s.finished[i + 1].tolist() == [[1, 1, 1]]
        assert s.scores[i + 1].tolist() == [[s.scores[1, 0, 0].item(), -math.inf, -math.inf]]
        assert seen[i][0].tolist() == [-1] * 3
        assert seen[i][1].tolist() == seen[1][1].tolist()
        assert (seen[i][2] >= 0).all()
    if why == "pages":
        s.ref[3] -= 1
    s.check_ledger()
    lla.lla_pages_free(s.last(), torch.arange(B * W, dtype=I32, device=DEV))
    assert not s.ref.any()


def test_in_pieces(lla):
    """Two steps and then four give what six give; and no more blocks are held at any step than the documented number."""
    B, W, V, prompts = 2, 4, 50, [130, 62]
    allowed = [[3, 7], list(range(V))]  # sequence 0 has dead beams at first
    bound = sum(P // 64 + W * (-(-(P + 6) // 64) - P // 64) for P in prompts)

    def run(steps, start=None, first=0):
        s = Search(lla, B, W, V, steps, blocks=bound)
        if start is None:
            s.prompt(prompts)
        else:
            s.ref, s.pages = start.ref, start.pages
            for name in ("tokens", "scores", "finished", "lengths"):
                getattr(s, name)[0] = getattr(start, name)[-1]
            s.tokens[0].clamp_(min=0)

        def step(i, pages, before, toks, slots):
            z = masked(s, i + first, allowed if i + first < 2 else [allowed[1]] * 2)
            z[:, :, 9] += 1.5
            return z + toks[:, :, None] / 100

        return s.run(step, eos=9, length_penalty=0.4)

    whole, one = run(6), run(2)
    assert lla.lla_get_device_error() == 0
    two = run(4, one, 2)
    for name in ("tokens", "scores", "finished", "lengths"):
        a, b = getattr(whole, name), getattr(two, name)
        assert torch.equal(a[3:], b[1:]) and torch.equal(a[:3], getattr(one, name)), name
    assert torch.equal(whole.parents, torch.cat([one.parents, two.parents]))
    assert torch.equal(whole.ref, two.ref) and torch.equal(whole.last().context_lens, two.last().context_lens)
    two.check_ledger()
    assert whole.finished.any()


def test_captured_and_replayed(lla):
    """A whole search with dead beams in a CUDA graph, replayed on other prompts and scores: what the same calls give outside."""
    B, W, V, steps = 2, 4, 60, 8
    table = torch.randn(V, V, generator=torch.Generator(device=DEV).manual_seed(8), device=DEV)
    table[:, 5:50][table[:, 5:50] < 1.2] = -math.inf  # few continuations a token

    def step(i, pages, before, toks, slots):
        return table[toks.long()].masked_fill(torch.arange(V, device=DEV) > (2 if i < 1 else V), -math.inf)

    def fresh():
        return Search(lla, B, W, V, steps, blocks=40).prompt([70, 3])

    def start(s, like, first):
        for a, b in zip([s.ref, s.pages[0].block_table, s.pages[0].context_lens], [like.ref, like.pages[0].block_table, like.pages[0].context_lens]):
            a.copy_(b)
        s.tokens[0] = first

    begin, s, plain = fresh(), fresh(), fresh()
    s.run(step, eos=9)  # once outside
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run(step, eos=9, stream=side)
    for first in (0, 17, 44):
        start(s, begin, first)
        graph.replay()
        start(plain, begin, first)
        plain.run(step, eos=9)
        torch.cuda.synchronize()
        for name in ("tokens", "parents", "scores", "finished", "lengths", "ref"):
            assert torch.equal(getattr(s, name), getattr(plain, name)), (first, name)
        assert torch.equal(s.last().block_table, plain.last().block_table) and torch.equal(s.last().context_lens, plain.last().context_lens)
        s.check_ledger()
    assert (s.parents < 0).any() and lla.lla_get_device_error() == 0


def test_the_largest_batch(lla):
    """32 sequences of 32 beams, all but a few dead at first."""
    B, W, V, steps = 32, 32, 300, 4
    s = Search(lla, B, W, V, steps, blocks=4096).prompt([40 + 3 * b for b in range(B)])
    allowed = lambda i: [list(range(1 + b % 7)) if i < 2 else list(range(V)) for b in range(B)]
    seen = []

    def step(i, pages, before, toks, slots):
        seen.append((toks.clone(), pages.context_lens.clone()))
        return masked(s, i, allowed(i))

    s.run(step)
    alive = [(s.parents[i] >= 0).sum(1).tolist() for i in range(steps)]
    assert alive[0] == [min(W, 1 + b % 7) for b in range(B)]
    assert alive[1] == [min(W, (1 + b % 7) ** 2) for b in range(B)]
    assert alive[2] == alive[3] == [W] * B
    assert all((t >= 0).all() and (t < V).all() and (n > 0).all() for t, n in seen)
    s.check_ledger()
