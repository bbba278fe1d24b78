"""Which stream the sequence operators' memory belongs to, on the host: torch's allocator and streams are stood in for,
and the library by one that accepts every call (no GPU needed)."""
import contextlib

import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, name, handle, device=None):
        self.name, self.cuda_stream, self.device = name, handle, device or torch.device("cpu")


class Library:
    """Answers every size query with 4096 bytes, records the calls' arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 4096 if name.endswith("_bytes") else B.WM_OK
        return call


@pytest.fixture
def world(monkeypatch):
    class World:
        main, side = Stream("main", 1), Stream("side", 2)
        now, lib, born, recorded = [main], Library(), [], []
        device = None                        # the current one; the CPU tensors' index is None too

        @staticmethod
        @contextlib.contextmanager
        def stream(s):
            World.now.append(s)
            yield
            World.now.pop()
    w = World
    empty = torch.empty

    def new(*a, **k):
        t = empty(*a, **k)
        w.born.append((w.now[-1].name, t))
        return t
    monkeypatch.setattr(B, "load_library", lambda: w.lib)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    monkeypatch.setattr(torch, "empty", new)
    monkeypatch.setattr(torch.cuda, "stream", w.stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: w.now[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: w.device)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.recorded.append((t.data_ptr(), s.name)), raising=False)
    return w


def all_calls():
    q, k = torch.zeros(4, 2, 64), torch.zeros(9, 1, 64)
    lse = torch.zeros(4, 2)
    x, off, wt = torch.zeros(4, 8), torch.tensor([0, 4], dtype=torch.int32), torch.zeros(8, 4)
    A, b = torch.zeros(8, 16), torch.zeros(4, 16)
    kept = torch.zeros(4096, dtype=torch.uint8)
    return {
        "cross_attention": ((q, k, k, [0, 4], [0, 9]), dict(need_lse=True)),
        "cross_attention_grad": ((q, q, k, k, q, lse, [0, 4], [0, 9]), {}),
        "causal_conv": ((x, off, wt), dict(T_max=4, need_state=True)),
        "causal_conv_grad": ((x, x, off, wt), dict(T_max=4, need_dstate=True)),
        "selective_scan": ((x, x, A, b, b, off), dict(T_max=4, need_state=True, need_checkpoints=True)),
        "selective_scan_grad": ((x, x, x, A, b, b, off, kept), dict(T_max=4, need_dh0=True)),
    }


@pytest.mark.parametrize("name", list(all_calls()))
def test_given_stream_owns_what_a_call_allocates(world, name):
    """All memory made in a call comes from the given stream's pool, so that none of it is handed to other work
    before the stream is past the call; results are kept from that pool's reuse while the caller's stream uses them, and
    the caller's tensors from their own pool's."""
    args, kw = all_calls()[name]
    r = getattr(wm, name)(*args, stream=world.side, **kw)
    assert world.born and {s for s, _ in world.born} == {"side"}
    launch = [c for c in world.lib.calls if not c[0].endswith("_bytes")]
    assert len(launch) == 1 and launch[0][1][-1] == 2                        # the kernels' stream
    for t in r.values():
        if t is not None:
            assert (t.data_ptr(), "main") in world.recorded
    for t in args:
        if isinstance(t, torch.Tensor):
            assert (t.data_ptr(), "side") in world.recorded


@pytest.mark.parametrize("name", list(all_calls()))
@pytest.mark.parametrize("given", [False, True])
def test_current_stream(world, name, given):
    """Without a stream, or with the current one, there is nothing to record."""
    args, kw = all_calls()[name]
    getattr(wm, name)(*args, **kw, **({"stream": world.main} if given else {}))
    assert {s for s, _ in world.born} == {"main"} and not world.recorded
    assert [c[1][-1] for c in world.lib.calls if not c[0].endswith("_bytes")] == [1]
