"""Gradient outputs that prefix_attention_grad refuses and takes, before anything reaches a device (no GPU needed)."""
import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B

torch = pytest.importorskip("torch")


def good():
    q, k, pk, off = torch.zeros(4, 4, 64), torch.zeros(4, 2, 64), torch.zeros(9, 2, 64), torch.tensor([0, 4], dtype=torch.int32)
    return dict(do=q, q=q, k=k, v=k, pk=pk, pv=pk, o=q, lse=torch.zeros(4, 4), off=off, q_off=[0, 4], p_off=[0, 9], T_max=4)


@pytest.fixture
def launched(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    calls = []
    monkeypatch.setattr(B, "_launch", lambda fn, dev, *args: calls.append(args))
    return calls


@pytest.mark.parametrize("name,shape", [("dq", (4, 4, 64)), ("dk", (4, 2, 64)), ("dv", (4, 2, 64)), ("dpk", (9, 2, 64)), ("dpv", (9, 2, 64))])
def test_gradient_outputs(launched, name, shape):
    rows, heads, dim = shape
    for t in (torch.zeros(rows - 1, heads, dim), torch.zeros(rows, heads, dim, dtype=torch.bfloat16), torch.zeros(rows, heads + 1, dim),
              torch.zeros(rows, dim, heads).transpose(1, 2)):
        with pytest.raises(ValueError):
            wm.prefix_attention_grad(**good(), **{name: t})
    assert not launched
    t = torch.zeros(rows, heads + 3, dim)[:, 1:heads + 1]
    r = wm.prefix_attention_grad(**good(), **{name: t})
    g = launched[0][6]
    assert r[name] is t and getattr(g, name) == t.data_ptr() and getattr(g, "ld_" + name) == (heads + 3) * dim
    assert all(r[n] is not None for n in ("dq", "dk", "dv", "dpk", "dpv"))
