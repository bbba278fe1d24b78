"""What the binding of the sequence operators asks of a workspace and of kept states that the caller passes: device
memory beside the tensors, dense; and of a stream: the tensors' device (no GPU needed)."""
import pytest

import paper_2606_09312_amd as wm
from test_sequence_streams import Library, Stream, all_calls, torch, world  # noqa: F401

WITH_WS = [n for n in all_calls() if n != "causal_conv"]
META = torch.device("meta")


@pytest.mark.parametrize("name", WITH_WS)
@pytest.mark.parametrize("ws", [torch.zeros(8192, dtype=torch.uint8, device=META),       # another device than the tensors'
                                torch.zeros(8192, 2, dtype=torch.uint8)[:, 0]], ids=["device", "strided"])
def test_workspace(world, name, ws):  # noqa: F811
    args, kw = all_calls()[name]
    with pytest.raises(ValueError, match="ws must be dense"):
        getattr(wm, name)(*args, ws=ws, **kw)
    assert not [c for c in world.lib.calls if not c[0].endswith("_bytes")]
    getattr(wm, name)(*args, ws=torch.zeros(8192, dtype=torch.uint8), **kw)


@pytest.mark.parametrize("kept", [torch.zeros(8192, dtype=torch.uint8, device=META),
                                  torch.zeros(8192, 2, dtype=torch.uint8)[:, 0], torch.zeros(4095, dtype=torch.uint8)],
                         ids=["device", "strided", "short"])
def test_checkpoints(world, kept):  # noqa: F811
    (x, _, A, b, _, off), _ = all_calls()["selective_scan"]
    with pytest.raises(ValueError, match="checkpoints"):
        wm.selective_scan(x, x, A, b, b, off, T_max=4, checkpoints=kept)
    with pytest.raises(ValueError, match="checkpoints"):
        wm.selective_scan_grad(x, x, x, A, b, b, off, kept, T_max=4)
    assert not [c for c in world.lib.calls if not c[0].endswith("_bytes")]


@pytest.mark.parametrize("name", list(all_calls()))
def test_tensors_on_another_device_than_the_current_one(world, monkeypatch, name):  # noqa: F811
    """The tensors' device is current for the launch, and only for it."""
    current = []

    class Device:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.was, world.device = world.device, self.dev.index

        def __exit__(self, *_):
            world.device = self.was
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(world, "device", 3)
    monkeypatch.setattr(Library, "__getattr__", lambda lib, n: lambda *a: current.append((n, world.device)) or
                        (4096 if n.endswith("_bytes") else 0))
    args, kw = all_calls()[name]
    getattr(wm, name)(*args, **kw)
    assert [d for n, d in current if not n.endswith("_bytes")] == [None]           # the tensors' index here
    assert world.device == 3


@pytest.mark.parametrize("name", list(all_calls()))
def test_stream_of_another_device(world, name):  # noqa: F811
    args, kw = all_calls()[name]
    with pytest.raises(ValueError, match="stream is on"):
        getattr(wm, name)(*args, stream=Stream("there", 9, torch.device("cuda", 1)), **kw)
    assert not world.lib.calls
