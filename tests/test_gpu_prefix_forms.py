"""Forms of the kernels over a shared prefix that only larger calls take: several rows per workgroup of the rotation and the append,
and what is not finite in keys or rows that only some see, where loops are split."""
import numpy as np
import pytest

from oracle import prefix as Q
from prefix_util import ATTN, LSE, TURN, Pool, close, dt, frequencies, host, i32, offsets, same_bits
from test_gpu_prefix import check_cached, make_prefix, status

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def wm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_09312_amd as wm
    wm.load_library()
    return wm


def lengths(n, seed):
    """Sequences of 0 to 59 rows, `n` together."""
    out, r = [], np.random.default_rng(seed)
    while sum(out) < n:
        out.append(int(min(r.integers(0, 60), n - sum(out))))
    return out


# ---- several rows per workgroup ------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,rot", [(2049, 64), (2050, 20), (4099, 6)])
def test_rotate_many_rows(wm, dtype, interleaved, n, rot):
    lens = lengths(n, rot)
    off, first = offsets(lens), np.random.default_rng(rot).integers(0, 1 << 23, len(lens))
    x = torch.randn((n, 3, 64), device="cuda").to(dt(dtype))[:, :2]
    f, st = frequencies(rot), status()
    y = torch.full((n, 4, 64), 7.0, device="cuda").to(dt(dtype))
    kw = dict(T_max=59, first=i32(first), interleaved=interleaved)
    wm.rotate(x, i32(off), f, y=y[:, 1:3], status=st, **kw)
    wm.device_status(st)
    close("y", y[:, 1:3], Q.rotate(host(x), Q.positions(off, first), host(f), interleaved), TURN[dtype])
    assert (y[:, 0] == 7.0).all() and (y[:, 3] == 7.0).all(), "what is not y changed"
    back = wm.rotate(x, i32(off), f, inverse=True, **kw)["y"]
    close("back", back, Q.rotate(host(x), Q.positions(off, first), host(f), interleaved, True), TURN[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,dh,rot,page", [(2049, 64, 64, 16), (2051, 32, 20, 32), (4099, 128, 6, 64)])
def test_append_many_rows(wm, dtype, interleaved, n, dh, rot, page):
    """Borders of sequences and ends of pages among a workgroup's rows; with and without rotation and queries."""
    lens = lengths(n, dh)
    r = np.random.default_rng(dh)
    off, before, first = offsets(lens), r.integers(0, 40, len(lens)), r.integers(0, 1 << 20, len(lens))
    total = [int(a + b) for a, b in zip(lens, before)]
    pool = Pool(dtype, page, 1, dh, total, seed=page, wide=1)
    qkv = torch.randn((n, 4, dh), device="cuda").to(dt(dtype))
    q, k, v = qkv[:, :2], qkv[:, 2:3], qkv[:, 3:]
    f = frequencies(rot)
    for turn in (True, False):
        kc, vc, st = pool.k.clone(), pool.v.clone(), status()
        kw = dict(first=i32(first), freq=f, interleaved=interleaved, q=q) if turn else {}
        got = wm.cache_append(k, v, kc, vc, i32(pool.pages), i32(total), i32(off), T_max=max(lens), status=st, **kw)
        wm.device_status(st)
        kw = (first, host(f), interleaved, host(q)) if turn else ()
        want = Q.append(host(k), host(v), host(pool.k), host(pool.v), pool.pages, total, off, *kw)
        if turn:
            close("q", got["q"], want[0], TURN[dtype])
            close("k_cache", kc, want[1], TURN[dtype])
        else:
            assert np.array_equal(host(kc), want[1], equal_nan=True)
        assert np.array_equal(host(vc), want[2], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,rot,interleaved", [(9, 64, False), (9, 20, True), (2051, 64, True), (2051, 6, False)])
def test_append_turns_queries_in_place(wm, dtype, n, rot, interleaved):
    lens = lengths(n, n)
    off, total = offsets(lens), [x + 5 for x in lens]
    pool = Pool(dtype, 32, 1, 64, total, seed=n)
    qkv = torch.randn((n, 4, 64), device="cuda").to(dt(dtype))
    q, k, v = qkv[:, :2], qkv[:, 2:3], qkv[:, 3:]
    f, before = frequencies(rot), qkv.clone()
    kw = dict(T_max=max(lens), freq=f, interleaved=interleaved)
    want = wm.cache_append(k, v, pool.k.clone(), pool.v.clone(), i32(pool.pages), i32(total), i32(off), q=q, **kw)["q"]
    r = wm.cache_append(k, v, pool.k, pool.v, i32(pool.pages), i32(total), i32(off), q=q, q_out=q, **kw)
    assert r["q"] is q and same_bits(q, want) and same_bits(qkv[:, 2:], before[:, 2:])


# ---- values that are not finite, in split loops ----------------------------------------
def split(wm, c, grad):
    """Whether a call's loops have parts (workspaces beyond the gradient's own, 12 bytes for every row of a head)."""
    from paper_2606_09312_amd import binding as B
    a = B._prefix(*[c[n] for n in ("q", "k", "v", "pk", "pv")], i32(c["off"]), c["q_off"], c["p_off"], c["T_max"], None, None, None)
    own = 12 * c["q"].shape[0] * c["q"].shape[1] + 1024 if grad else 256
    return wm.load_library().wm_prefix_attention_workspace_bytes(a, grad) > own


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("G,n,P", [(2, 1500, 0), (3, 1100, 200)])
def test_split_causal_loops(wm, dtype, dh, G, n, P):
    """One long sequence behind a short one: what rows do not see yet does not reach them, what they see does."""
    c = make_prefix(dtype, [2], [30, n], [P], G, 1, dh, seed=dh)
    assert split(wm, c, 0) and split(wm, c, 1)
    names, N = ("q", "k", "v", "pk", "pv"), n + 30
    x, where = {m: c[m] for m in names}, (i32(c["off"]), c["q_off"], c["p_off"])
    clean = [host(x[m]) for m in names]
    place = (c["off"], c["q_off"], c["p_off"], dh ** -0.5)
    o, lse = Q.prefix(*clean, *place)
    row = np.arange(N)

    # forward: parts of values, and a key
    a, b, z = 30 + n // 2, 30 + n - 200, 30 + n - 90
    v, k = x["v"].clone(), x["k"].clone()
    v[a, :, 3:5] = float("nan")
    v[b, :, 6] = float("inf")
    k[z] = float("nan")
    f = wm.prefix_attention(x["q"], k, v, x["pk"], x["pv"], *where, T_max=n, need_lse=True)
    want, wl = o.copy(), lse.copy()
    want[a:, :, 3:5], want[b:, :, 6], want[z:], wl[z:] = np.nan, np.inf, np.nan, np.nan
    close("o", f["o"], want, ATTN[dtype])
    close("lse", f["lse"], wl, LSE)

    # gradient: a row's do, a key's value
    f = wm.prefix_attention(*x.values(), *where, T_max=n, need_lse=True)
    given = host(f["o"])
    want = dict(zip(("dq", "dk", "dv"), Q.prefix_grad(host(c["do"]), *clean, *place, o=given)))
    spread = dict(zip(("dq", "dk", "dv"), Q.grad_spread(host(c["do"]), *clean, *place, None, given)))
    own = row >= 30
    for what in ("do", "v"):
        do, v = c["do"].clone(), x["v"].clone()
        (do if what == "do" else v)[a] = float("nan")
        got = wm.prefix_attention_grad(do, x["q"], x["k"], v, x["pk"], x["pv"], f["o"], f["lse"], *where, T_max=n)
        nan = dict(dq=row == a, dk=own & (row <= a), dv=own & (row <= a)) if what == "do" else dict(dq=row >= a, dk=row == a, dv=row < 0)
        for m in want:
            w = want[m].copy()
            w[nan[m]] = np.nan
            close(f"{what}: {m}", got[m], w, ATTN[dtype], spread[m])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("T,shared", [([200], []), ([5], []), ([130, 3], [900]), ([4, 9], [2000])])
def test_split_chunks(wm, dtype, dh, T, shared):
    """Chunks over long caches, whose last rows alone see what is not finite."""
    own = [3000 + t for t in T]
    pool = Pool(dtype, 32, 1, dh, own, shared, seed=dh)
    for s, t in enumerate(T):
        for slot, x in ((own[s] - t // 2 - 1, float("nan")), (own[s] - 2, float("inf"))):
            pool.v[pool.pages[s][slot // 32], :, slot % 32, 3 + (x > 0):6] = x
        pool.k[pool.pages[s][(own[s] - 1) // 32], :, (own[s] - 1) % 32] = float("nan")
    check_cached(wm, dtype, pool, offsets(T), [len(T)] if shared else None, 2, 1, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("G", [1, 3])
def test_products_that_overflow_elsewhere(wm, dtype, dh, G):
    """Finite values whose products are not: they stay in their sequence, its rows before them are as without them."""
    c = make_prefix(dtype, [4], [20, 33, 7, 60], [0], 2 * G, 2, dh, seed=dh)
    names, place = ("q", "k", "v", "pk", "pv"), (c["off"], c["q_off"], c["p_off"], dh ** -0.5)
    x, where = {m: c[m] for m in names}, (i32(c["off"]), c["q_off"], c["p_off"])
    clean = [host(x[m]) for m in names]
    f = wm.prefix_attention(*x.values(), *where, T_max=60, need_lse=True)
    given = host(f["o"])
    want = dict(zip(("dq", "dk", "dv"), Q.prefix_grad(host(c["do"]), *clean, *place, o=given)))
    spread = dict(zip(("dq", "dk", "dv"), Q.grad_spread(host(c["do"]), *clean, *place, None, given)))
    a, b = c["off"][1] + 10, c["off"][2]
    for what in ("q", "do", "v", "k"):
        y = {**x, "do": c["do"]}
        y[what] = y[what].clone()
        y[what][a:b] = torch.where(torch.randn(y[what][a:b].shape, device="cuda") > 0, 3e38, -3e38).to(dt(dtype))
        got = wm.prefix_attention_grad(y["do"], *[y[m] for m in names], f["o"], f["lse"], *where, T_max=60)
        for m in want:
            # rows that see none of them; keys that none of the sequence's rows see (a row's weights and the mean of its score gradients
            # bring what it sees to all of its keys)
            far = np.ones(c["off"][-1], bool)
            far[(a if m == "dq" else c["off"][1]):b] = False
            t = torch.tensor(far, device="cuda")
            close(f"{what}: {m}", got[m][t], want[m][far], ATTN[dtype], spread[m][far])
        if what in "qk":
            finite = bool(torch.isfinite(got["dq"][a:b].float()).all())
            assert not finite, what


def test_steps_that_are_not_finite_end_soon(wm):
    """A training step whose values are NaN, or one row's of them: sums that are formed again end where they are NaN, and are formed again
    only where what some rows do not see can have spoilt them (up to 130 times a finite step's time without both, 4 to 17 with them)."""
    n, Hq, Hk, dh = 6000, 32, 8, 128
    off = i32(range(0, n + 1, 1500))
    q, k, v, do = (torch.randn((n, h, dh), device="cuda").bfloat16() for h in (Hq, Hk, Hk, Hq))
    none = torch.zeros((0, Hk, dh), device="cuda").bfloat16()

    def step(do, q, k, v):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f = wm.prefix_attention(q, k, v, none, none, off, [0, n], [0, 0], T_max=1500, need_lse=True)
        wm.prefix_attention_grad(do, q, k, v, none, none, f["o"], f["lse"], off, [0, n], [0, 0], T_max=1500)
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b)

    def row(x):
        x = x.clone()
        x[n // 2 + 700] = float("nan")
        return x
    nan = lambda x: torch.full_like(x, float("nan"))  # noqa: E731
    clean = min(step(do, q, k, v) for _ in range(5))
    for name, x in (("all", (nan(do), nan(q), nan(k), nan(v))), ("do", (nan(do), q, k, v)), ("a row of do", (row(do), q, k, v)),
                    ("a row of q", (do, row(q), k, v)), ("a row of v", (do, q, k, row(v)))):
        t = min(step(*x) for _ in range(3))
        print(f"[not finite] {name}: {t:.2f} ms of {clean:.2f}", flush=True)
        assert t <= 25 * clean, f"{name}: {t} ms of {clean}"
