"""lla_decode_attn_decoupled_axes refuses arrays of another type or shape than its queries', like the calls beside it."""
import pytest
import torch

from helpers import ensure_library

B, H, D, DR = 3, 2, 128, 64
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
NAMES = ("positions", "context_lens", "q", "q_rope", "cur_k", "cur_v", "cur_k_rope", "out")


@pytest.fixture(scope="module")
def lla():
    ensure_library()
    from paper_2607_15456_gb300 import lla as m
    return m


def arrays(device, io=F32):
    x = lambda *s: torch.zeros(*s, dtype=io, device=device)
    return dict(positions=torch.zeros(3, B, dtype=I32, device=device), context_lens=torch.zeros(B, dtype=I32, device=device), q=x(B, H, D),
                q_rope=x(B, H, DR), cur_k=x(B, H, D), cur_v=x(B, H, D), cur_k_rope=x(B, DR), out=x(B, H, D))


def call(lla, device, a, table=None, workspace=None):
    w = torch.zeros(64, dtype=BF16, device=device)
    table = torch.zeros(B, 2, dtype=I32, device=device) if table is None else table
    cache = lla.Cache(w, 1, table, 2)
    lla.lla_decode_attn_decoupled_axes(lla.Geometry(4, H, D, 96, 160), lla.Codec(w, w, w, w), cache, w, DR, lla.RopeAxes(1e4, 0, (16, 8, 8)),
                                       a["positions"], a["context_lens"], 128, 0, a["q"], a["q_rope"], a["cur_k"], a["cur_v"], a["cur_k_rope"],
                                       a["out"], torch.zeros(1, dtype=torch.uint8, device=device) if workspace is None else workspace)


def wrong(device, io):
    """(name, an array that the call refuses)"""
    a = arrays(device, io)
    other = BF16 if io == F32 else F32
    for name in NAMES[3:]:
        yield name, a[name].to(other)
    yield "positions", a["positions"].long()
    yield "context_lens", a["context_lens"].long()
    for name in NAMES:
        if name != "q":
            yield name, a[name][..., :-1].contiguous()
            yield name, torch.cat((a[name], a[name]))
            yield name, a[name].reshape(-1)[:0]
    yield "q", a["q"][:, :, :64].contiguous()
    yield "q", a["q"][:, :1].contiguous()
    yield "q", a["q"].view(B, H * D)


@pytest.mark.parametrize("io", [F32, BF16])
def test_python_refuses(lla, io, monkeypatch):
    """On the host, with arrays that stand in for the device's: nothing reaches the library."""
    class Nothing:
        def __getattr__(self, name):
            def enqueue(*args):
                raise AssertionError("enqueued")
            return enqueue
    monkeypatch.setattr(lla, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(lla, "_stream", lambda s: None)
    monkeypatch.setattr(lla, "library", Nothing)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)  # that of a host tensor
    with pytest.raises(AssertionError, match="enqueued"):  # what is right gets there
        call(lla, "cpu", arrays("cpu", io))
    cur = dict(arrays("cpu", io), cur_k=None, cur_v=None, cur_k_rope=None)
    with pytest.raises(AssertionError, match="enqueued"):
        call(lla, "cpu", cur)
    for name, bad in wrong("cpu", io):
        with pytest.raises(ValueError):
            call(lla, "cpu", dict(arrays("cpu", io), **{name: bad}))
    for table in (torch.zeros(B - 1, 2, dtype=I32), torch.zeros(B, 3, dtype=I32), torch.zeros(B, 2, dtype=I64), torch.zeros(2 * B, dtype=I32)):
        with pytest.raises(ValueError):
            call(lla, "cpu", arrays("cpu", io), table=table)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [F32, BF16])
def test_the_native_call_refuses(lla, io):
    """The same through the native marshalling; a right call is refused for its small workspace alone."""
    with pytest.raises(lla.LLAError, match="WORKSPACE"):
        call(lla, "cuda", arrays("cuda", io))
    for name, bad in wrong("cuda", io):
        with pytest.raises(ValueError):
            call(lla, "cuda", dict(arrays("cuda", io), **{name: bad}))
