"""Which stream the memory of evaluate, rollout_loss and encode_text belongs to when they are given one, on the host with
stand-ins for torch's streams and the library (no GPU needed)."""
import pytest

import paper_2606_09312_amd as wm
from test_sequence_streams import torch, world  # noqa: F401


class Evaluator(wm.Model):                 # without the library's objects behind them
    handle, norm, dims = 1, "none", dict(d=8, e=4, H=16, n_kinds=3, n_params=2)

    def __init__(self):
        pass

    def __del__(self):
        pass


class Encoder(wm.TextModel):
    handle, w = 1, type("W", (), dict(d=8))

    def __init__(self):
        pass

    def __del__(self):
        pass


def all_calls():
    m, t = Evaluator(), Encoder()
    z0, types, params = torch.zeros(1, 8), torch.zeros(4, 5, dtype=torch.int32), torch.zeros(4, 5, 2)
    lens, hw, tgt = torch.zeros(4, dtype=torch.int32), torch.zeros(2, 3), torch.zeros(4, 5, 8)
    neg, tokens = torch.zeros(4, 5, 2, 8), torch.zeros(9, dtype=torch.int32)
    return {"evaluate": ((m, z0, [0, 4], types, params, lens, hw, 2), dict(scores=torch.zeros(2, 4))),
            "rollout_loss": ((m, z0, [0, 4], types, params, lens, tgt, neg, 0.5, 0.3), dict(out={"w1": torch.zeros(16, 12)})),
            "encode_text": ((t, tokens, [0, 9]), {})}


@pytest.mark.parametrize("name", list(all_calls()))
@pytest.mark.parametrize("given", [True, False])
def test_given_stream_owns_what_a_call_allocates(world, monkeypatch, name, given):  # noqa: F811
    zeros = torch.zeros

    def new(*a, **k):
        t = zeros(*a, **k)
        world.born.append((world.now[-1].name, t))
        return t
    args, kw = all_calls()[name]
    monkeypatch.setattr(torch, "zeros", new)
    r = getattr(wm, name)(*args, **kw, **({"stream": world.side} if given else {}))
    assert len(world.born) >= 2 and {s for s, _ in world.born} == {"side" if given else "main"}
    launch = [c for c in world.lib.calls if not c[0].endswith(("_bytes", "_chunks", "_destroy"))]
    assert len(launch) == 1 and launch[0][1][-1].value == (2 if given else 1)
    wanted = [(t.data_ptr(), "main") for t in r.values() if t is not None]
    wanted += [(t.data_ptr(), "side") for v in (*args, *kw.values()) for t in (v.values() if isinstance(v, dict) else [v])
               if isinstance(t, torch.Tensor)]
    assert set(wanted) == set(world.recorded) if given else not world.recorded


def test_encode_text_takes_the_stream_by_place(world):  # noqa: F811
    args, _ = all_calls()["encode_text"]
    wm.encode_text(*args, None, None, world.side)
    assert [c[1][-1].value for c in world.lib.calls if c[0] == "wm_encode_text"] == [2]
