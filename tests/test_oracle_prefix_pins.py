"""The float64 definitions of the operators over a shared prefix against independent forms: complex
multiplication, a dense softmax over all keys at once, central differences."""
import numpy as np
import pytest

from oracle import prefix as Q
from oracle import sequence as S


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    x, f = rnd(0, 7, 2, 10), np.array([1.0, 0.3, 0.01, 2.0])
    pos = np.array([0, 1, 5, 1000, 1 << 23, 3, 17])
    y = Q.rotate(x, pos, f, interleaved)
    a, b = (slice(0, 8, 2), slice(1, 8, 2)) if interleaved else (slice(0, 4), slice(4, 8))
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, None, None] * f)
    assert np.allclose(y[..., a], z.real, atol=1e-8) and np.allclose(y[..., b], z.imag, atol=1e-8)
    assert (y[..., 8:] == x[..., 8:]).all() and (y[0] == x[0]).all()
    assert np.allclose(Q.rotate(y, pos, f, interleaved, inverse=True), x)


def test_rotation_back_is_the_gradient():
    x, dy, f, pos = rnd(1, 3, 1, 6), rnd(2, 3, 1, 6), np.array([0.7, 0.1]), np.array([2, 9, 4])
    dx = Q.rotate(dy, pos, f, inverse=True)
    for i in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[i] = 1e-5
        d = ((Q.rotate(x + e, pos, f) - Q.rotate(x - e, pos, f)) * dy).sum() / 2e-5
        assert abs(d - dx[i]) < 1e-8


def test_append_puts_rows_where_the_table_says():
    k, v, q = rnd(3, 5, 2, 4), rnd(4, 5, 2, 4), rnd(5, 5, 4, 4)
    kc, vc = rnd(6, 4, 2, 16, 4), rnd(7, 4, 2, 16, 4)
    pages, lens, off = np.array([[2, 0], [3, -1]]), [18, 2], [0, 3, 5]
    q2, k2, v2 = Q.append(k, v, kc, vc, pages, lens, off, first=[10, 0], freq=[0.5], q=q)
    where = [(2, 15), (0, 0), (0, 1), (3, 0), (3, 1)]
    pos = np.array([25, 26, 27, 0, 1])
    assert np.allclose(q2, Q.rotate(q, pos, [0.5]))
    for r, (p, j) in enumerate(where):
        assert np.allclose(k2[p, :, j], Q.rotate(k, pos, [0.5])[r]) and (v2[p, :, j] == v[r]).all()
        kc[p, :, j], vc[p, :, j] = k2[p, :, j], v2[p, :, j]
    assert (k2 == kc).all() and (v2 == vc).all()


def packed():
    off, q_off, p_off = [0, 3, 3, 7, 9], [0, 7, 9], [0, 5, 6]
    return (rnd(10, 9, 4, 6), rnd(11, 9, 2, 6), rnd(12, 9, 2, 6), rnd(13, 6, 2, 6), rnd(14, 6, 2, 6), off, q_off, p_off)


@pytest.mark.parametrize("mask", [None, [1, 0, 1, 1, 0, 0]])
def test_prefix_is_one_softmax_over_both_kinds_of_keys(mask):
    q, k, v, pk, pv, off, q_off, p_off = packed()
    o, lse = Q.prefix(q, k, v, pk, pv, off, q_off, p_off, 0.4, mask)
    for p, a, b in ((0, 0, 3), (0, 3, 7), (1, 7, 9)):
        shown = [j for j in range(p_off[p], p_off[p + 1]) if mask is None or mask[j]]
        for i in range(a, b):
            for h in range(4):
                keys = np.concatenate([pk[shown, h // 2], k[a:i + 1, h // 2]])
                w = np.exp(0.4 * keys @ q[i, h])
                assert np.allclose(o[i, h], w @ np.concatenate([pv[shown, h // 2], v[a:i + 1, h // 2]]) / w.sum())
                assert np.isclose(lse[i, h], np.log(w.sum()))


def test_prefix_without_own_history_is_cross_attention():
    """Sequences of one row with an own key that weighs nothing: cross attention to the program's keys."""
    q, k, v, pk, pv, _, q_off, p_off = packed()
    off = list(range(10))
    o, lse = Q.prefix(q, -1e3 * np.repeat(q[:, ::2], 1, 1), v, pk, pv, off, q_off, p_off, 0.4)
    want, wl = S.attention(q, pk, pv, q_off, p_off, 0.4)
    assert np.allclose(o[:, ::2], want[:, ::2]) and np.allclose(lse[:, ::2], wl[:, ::2])


def test_prefix_gradient_by_differences():
    args = list(packed())
    mask = [1, 1, 0, 1, 1, 1]
    do = rnd(20, 9, 4, 6)
    grads = Q.prefix_grad(do, *args, 0.4, mask)
    r = np.random.default_rng(3)
    for n, g in enumerate(grads):
        for _ in range(12):
            i = tuple(r.integers(0, d) for d in args[n].shape)
            e = np.zeros(args[n].shape)
            e[i] = 1e-5
            up, down = ([*args[:n], args[n] + s * e, *args[n + 1:]] for s in (1, -1))
            d = ((Q.prefix(*up, 0.4, mask)[0] - Q.prefix(*down, 0.4, mask)[0]) * do).sum() / 2e-5
            assert abs(d - g[i]) < 1e-7, (n, i)


def test_cached_reads_pages_as_prefix_reads_rows():
    """The same sequences through page tables: chunks of 2, 1 and 3 new rows of longer sequences."""
    page, P, L, T = 16, [5, 20], [18, 4, 33], [2, 1, 3]
    per = [0, 2, 3]
    kc, vc = rnd(30, 9, 2, page, 6), rnd(31, 9, 2, page, 6)
    pages = np.array([[4, 1, -1], [7, -1, -1], [0, 8, 2]])
    ppages = np.array([[3, -1], [6, 5]])
    off = [0, 2, 3, 6]
    q = rnd(32, 6, 4, 6)
    o, lse = Q.cached(q, kc, vc, pages, L, off, 0.5, per, ppages, P)
    whole = [0, *np.cumsum(L)]
    k, v = (np.concatenate([Q.keys_of(c, t, n) for t, n in zip(pages, L)]) for c in (kc, vc))
    pk, pv = (np.concatenate([Q.keys_of(c, t, n) for t, n in zip(ppages, P)]) for c in (kc, vc))
    qq = rnd(33, whole[-1], 4, 6)
    rows = np.concatenate([np.arange(whole[s + 1] - T[s], whole[s + 1]) for s in range(3)])
    qq[rows] = q
    want, wl = Q.prefix(qq, k, v, pk, pv, whole, [whole[i] for i in per], [0, 5, 25], 0.5)
    assert np.allclose(o, want[rows]) and np.allclose(lse, wl[rows])


def test_cached_row_without_keys():
    q = rnd(40, 3, 2, 4)
    o, lse = Q.cached(q, rnd(41, 2, 1, 16, 4), rnd(42, 2, 1, 16, 4), np.array([[0], [1]]), [1, 0], [0, 2, 3], 1.0)
    assert (o[0] == 0).all() and (lse[0] == -np.inf).all() and np.isfinite(lse[1]).all()
    assert (o[2] == 0).all() and (lse[2] == -np.inf).all()
