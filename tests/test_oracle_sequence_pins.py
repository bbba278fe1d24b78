"""The float64 definitions of the sequence operators against independent forms: torch's softmax and
differentiation, closed forms by hand, and central differences of the definitions themselves."""
import math

import numpy as np
import pytest

from oracle import sequence as Q

torch = pytest.importorskip("torch")


def _attn(seed=0, hidden=True):
    r = np.random.default_rng(seed)
    q_off, k_off = [0, 3, 3, 7, 9], [0, 5, 9, 9, 12]      # a segment without rows, one without keys
    q, k, v = r.normal(size=(9, 4, 8)), r.normal(size=(12, 2, 8)), r.normal(size=(12, 2, 8))
    mask = (r.random(12) > 0.3).astype(np.uint8) if hidden else None
    if hidden:
        mask[9:] = 0                                       # a segment whose keys are all hidden
        mask[0] = 1
    return q, k, v, q_off, k_off, 0.7, mask


def _scan(seed=1, gate=True):
    r = np.random.default_rng(seed)
    off = [0, 4, 4, 5, 11]
    n, C, N = 11, 3, 4
    a = dict(u=r.normal(size=(n, C)), delta=r.normal(size=(n, C)), A=-np.exp(r.normal(size=(C, N))), Bm=r.normal(size=(n, N)),
             Cm=r.normal(size=(n, N)), D=r.normal(size=C), z=r.normal(size=(n, C)) if gate else None,
             delta_bias=r.normal(size=C), h0=r.normal(size=(4, C, N)))
    return a, off, r.normal(size=(n, C)), r.normal(size=(4, C, N))


def _differences(f, x, eps=1e-5):
    """Central differences of a scalar function of the array x."""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        y = x.copy()
        y[i] += eps
        hi = f(y)
        y[i] -= 2 * eps
        g[i] = (hi - f(y)) / (2 * eps)
    return g


@pytest.mark.parametrize("hidden", [False, True])
def test_attention_equals_torch_softmax(hidden):
    q, k, v, q_off, k_off, scale, mask = _attn(hidden=hidden)
    o, lse = Q.attention(q, k, v, q_off, k_off, scale, mask)
    for s in range(4):
        keys = [j for j in range(k_off[s], k_off[s + 1]) if mask is None or mask[j]]
        for i in range(q_off[s], q_off[s + 1]):
            for h in range(4):
                if not keys:
                    assert (o[i, h] == 0).all() and lse[i, h] == -math.inf
                    continue
                sc = torch.tensor(scale * (k[keys, h // 2] @ q[i, h]))
                np.testing.assert_allclose(o[i, h], (torch.softmax(sc, 0).numpy() @ v[keys, h // 2]), rtol=1e-12, atol=1e-13)
                assert abs(lse[i, h] - torch.logsumexp(sc, 0).item()) < 1e-12


@pytest.mark.parametrize("hidden", [False, True])
def test_attention_gradient_equals_differences(hidden):
    q, k, v, q_off, k_off, scale, mask = _attn(3, hidden)
    do = np.random.default_rng(4).normal(size=q.shape)
    got = Q.attention_grad(do, q, k, v, q_off, k_off, scale, mask)
    loss = lambda q, k, v: (Q.attention(q, k, v, q_off, k_off, scale, mask)[0] * do).sum()  # noqa: E731
    for g, want in zip(got, (_differences(lambda x: loss(x, k, v), q), _differences(lambda x: loss(q, x, v), k),
                             _differences(lambda x: loss(q, k, x), v))):
        np.testing.assert_allclose(g, want, rtol=1e-6, atol=1e-7)


def test_conv_by_hand_and_differences():
    # two taps, identity: y_t = w0 x_{t-1} + w1 x_t + b
    x, w = np.array([[1.0], [2.0], [4.0]]), np.array([[10.0, 1.0]])
    y, out = Q.conv(x, [0, 1, 3], w, np.array([0.5]), silu=False, state=np.array([[[3.0]], [[0.0]]]))
    np.testing.assert_array_equal(y[:, 0], [31.5, 2.5, 24.5])
    np.testing.assert_array_equal(out[:, 0, 0], [1.0, 4.0])
    r = np.random.default_rng(5)
    off = [0, 1, 1, 6, 8]                                    # shorter than the taps, empty, longer
    x, w, b, st = r.normal(size=(8, 2)), r.normal(size=(2, 4)), r.normal(size=2), r.normal(size=(4, 3, 2))
    dy, ds = r.normal(size=(8, 2)), r.normal(size=(4, 3, 2))

    def loss(x, w, b, st):
        y, out = Q.conv(x, off, w, b, True, st)
        return (y * dy).sum() + (out * ds).sum()
    got = Q.conv_grad(dy, x, off, w, b, True, st, ds)
    for g, want in zip(got, (_differences(lambda a: loss(a, w, b, st), x), _differences(lambda a: loss(x, a, b, st), w),
                             _differences(lambda a: loss(x, w, a, st), b), _differences(lambda a: loss(x, w, b, a), st))):
        np.testing.assert_allclose(g, want, rtol=1e-6, atol=1e-7)


def test_conv_equals_torch_conv1d():
    r = np.random.default_rng(6)
    x, w, b = r.normal(size=(9, 5)), r.normal(size=(5, 4)), r.normal(size=5)
    y, _ = Q.conv(x, [0, 9], w, b, True)
    t = torch.nn.functional.conv1d(torch.tensor(x.T)[None], torch.tensor(w)[:, None], torch.tensor(b), padding=3, groups=5)
    np.testing.assert_allclose(y, torch.nn.functional.silu(t[0, :, :9]).T.numpy(), rtol=1e-12, atol=1e-13)


def test_scan_closed_form():
    # constant dt and B, no input after the first step: h decays as exp(A dt) per step
    T, dt, A = 5, math.log(2.0), -1.5                      # softplus(0) = log 2
    u = np.array([[3.0]] + [[0.0]] * (T - 1))
    y, hT = Q.scan(u, np.zeros((T, 1)), np.array([[A]]), np.ones((T, 1)), np.full((T, 1), 2.0), [0, T])
    want = 2.0 * dt * 3.0 * np.exp(A * dt * np.arange(T))
    np.testing.assert_allclose(y[:, 0], want, rtol=1e-14)
    np.testing.assert_allclose(hT[0, 0, 0], want[-1] / 2.0, rtol=1e-14)


@pytest.mark.parametrize("gate", [False, True])
def test_scan_gradient_equals_differentiation_and_differences(gate):
    a, off, dy, dhT = _scan(gate=gate)
    got = Q.scan_grad(dy, off=off, dhT=dhT, **a)

    def loss(**kw):
        y, hT = Q.scan(off=off, **{**a, **kw})
        return (y * dy).sum() + (hT * dhT).sum()
    names = {"u": "du", "delta": "ddelta", "A": "dA", "Bm": "dB", "Cm": "dC", "D": "dD", "delta_bias": "ddelta_bias", "h0": "dh0"}
    if gate:
        names["z"] = "dz"
    for n, g in names.items():
        np.testing.assert_allclose(got[g], _differences(lambda x: loss(**{n: x}), a[n]), rtol=2e-6, atol=1e-7)
    # the same by torch, with its own softplus, sigmoid and differentiation
    t = {n: torch.tensor(x, requires_grad=True) for n, x in a.items() if x is not None}
    total = 0.0
    for s in range(4):
        h = t["h0"][s]
        for i in range(off[s], off[s + 1]):
            d = torch.nn.functional.softplus(t["delta"][i] + t["delta_bias"], threshold=1e3)
            h = torch.exp(d[:, None] * t["A"]) * h + (d * t["u"][i])[:, None] * t["Bm"][i]
            y = h @ t["Cm"][i] + t["D"] * t["u"][i]
            if gate:
                y = y * torch.nn.functional.silu(t["z"][i])
            total = total + (y * torch.tensor(dy[i])).sum()
        total = total + (h * torch.tensor(dhT[s])).sum()
    total.backward()
    for n, g in names.items():
        np.testing.assert_allclose(got[g], t[n].grad.numpy(), rtol=1e-10, atol=1e-12)


def test_scan_split_in_two_equals_whole():
    a, _, _, _ = _scan(7)
    y, hT = Q.scan(off=[0, 11], **{**a, "h0": a["h0"][:1]})
    first = {n: (x[:6] if n in ("u", "delta", "Bm", "Cm", "z") else x) for n, x in a.items()}
    rest = {n: (x[6:] if n in ("u", "delta", "Bm", "Cm", "z") else x) for n, x in a.items()}
    y1, h1 = Q.scan(off=[0, 6], **{**first, "h0": a["h0"][:1]})
    y2, h2 = Q.scan(off=[0, 5], **{**rest, "h0": h1})
    np.testing.assert_allclose(np.concatenate([y1, y2]), y, rtol=1e-13)
    np.testing.assert_allclose(h2, hT, rtol=1e-13)
