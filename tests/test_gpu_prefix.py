"""GPU parity of the operators over a shared prefix (rotation, paged append, cached attention, prefix attention and
its gradient) against the float64 oracle on the values that the kernels are given; tolerances in prefix_util."""
import numpy as np
import pytest

from oracle import prefix as Q
from prefix_util import ATTN, LSE, TURN, Pool, close, dt, frequencies, host, i32, offsets, same_bits

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def wm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_09312_amd as wm
    wm.load_library()
    return wm


def status():
    return torch.zeros(64, dtype=torch.int32, device="cuda")


# ---- rotation ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,dh,rot", [(3, 64, 64), (2, 128, 96), (1, 32, 20), (5, 40, 6), (2, 512, 512)])
def test_rotate(wm, dtype, interleaved, H, dh, rot):
    print(f"[rotate] {dtype} heads={H} dim={dh} rot={rot} interleaved={interleaved}", flush=True)
    lens = [5, 0, 1, 70, 3]
    off, first = offsets(lens), [0, 7, 1 << 23, 1000003, 300]
    n = off[-1]
    g = torch.Generator(device="cuda").manual_seed(rot)
    wide = torch.randn((n + 2, H + 1, dh), generator=g, device="cuda").to(dt(dtype))
    x = wide[:n, :H]                                   # a larger row stride
    f = frequencies(rot)
    kw = dict(T_max=70, first=i32(first), interleaved=interleaved)
    st = status()
    y = wm.rotate(x, i32(off), f, status=st, **kw)["y"]
    wm.device_status(st)
    pos = Q.positions(off, first)
    close("y", y, Q.rotate(host(x), pos, host(f), interleaved), TURN[dtype])
    back = wm.rotate(y, i32(off), f, inverse=True, **kw)["y"]
    close("back", back, Q.rotate(host(y), pos, host(f), interleaved, True), TURN[dtype])
    again = wide.clone()
    wm.rotate(again[:n, :H], i32(off), f, y=again[:n, :H], **kw)
    assert same_bits(again[:n, :H], y), "in place"
    assert same_bits(again[n:], wide[n:]) and same_bits(again[:, H], wide[:, H]), "what is not x changed"


def test_rotate_many_rows(wm):
    """Enough rows that a workgroup takes four."""
    lens = list(np.random.default_rng(1).integers(0, 60, 200))
    off = offsets(lens)
    x = torch.randn((off[-1], 2, 64), device="cuda")
    assert off[-1] > 4096 and off[-1] % 4
    f = frequencies(64)
    y = wm.rotate(x, i32(off), f, T_max=59)["y"]
    close("y", y, Q.rotate(host(x), Q.positions(off), host(f)), TURN["f32"])


# ---- append --------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,Hq,Hk,dh,rot,lens,before", [
    (16, 4, 2, 64, 64, [1, 1, 1], [0, 15, 16]),             # a step each: first slot, a page's last and first
    (32, 3, 3, 32, 20, [40, 0, 7, 33], [0, 5, 25, 31]),     # over page ends, odd rotation, no rows
    (64, 8, 1, 128, 128, [130], [1]),
    (256, 2, 2, 64, 32, [300, 2], [0, 255]),
])
def test_append(wm, dtype, page, Hq, Hk, dh, rot, lens, before):
    print(f"[append] {dtype} page={page} heads={Hq}/{Hk} dim={dh} rot={rot} rows={lens} before={before}", flush=True)
    off, total = offsets(lens), [a + b for a, b in zip(lens, before)]
    pool = Pool(dtype, page, Hk, dh, total, seed=page, wide=1)
    n = off[-1]
    qkv = torch.randn((n + 1, Hq + 2 * Hk, dh), device="cuda").to(dt(dtype))
    q, k, v = qkv[:n, :Hq], qkv[:n, Hq:Hq + Hk], qkv[:n, Hq + Hk:]
    first = [3, 5, 1 << 20, 9][:len(lens)]
    f = frequencies(rot)
    for interleaved in (False, True):
        kc, vc = pool.k.clone(), pool.v.clone()
        want = Q.append(host(k), host(v), host(kc), host(vc), pool.pages, total, off, first, host(f), interleaved, host(q))
        st = status()
        r = wm.cache_append(k, v, kc, vc, i32(pool.pages), i32(total), i32(off), T_max=max(lens), first=i32(first), freq=f,
                            interleaved=interleaved, q=q, status=st)
        wm.device_status(st)
        assert r["k_cache"] is kc and r["v_cache"] is vc
        close("q", r["q"], want[0], TURN[dtype])
        close("k_cache", kc, want[1], TURN[dtype])
        assert np.array_equal(host(vc), want[2], equal_nan=True)
    # without rotation: copies, other slots as they were
    kc, vc = pool.k.clone(), pool.v.clone()
    r = wm.cache_append(k, v, kc, vc, i32(pool.pages), i32(total), i32(off), T_max=max(lens))
    _, kw, vw = Q.append(host(k), host(v), host(pool.k), host(pool.v), pool.pages, total, off)
    assert r["q"] is None and np.array_equal(host(kc), kw, equal_nan=True) and np.array_equal(host(vc), vw, equal_nan=True)


# ---- cached attention ----------------------------------------------------------------
def check_cached(wm, dtype, pool, off, per, Hq, Hk, dh, seed=0, scale=None, bounds=True, extra=0):
    n = off[-1]
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn((n + extra, Hq + 1, dh), generator=g, device="cuda").to(dt(dtype))[:, :Hq]
    o = torch.full((n + extra, Hq, dh), 7.0, device="cuda", dtype=q.dtype)
    lse = torch.full((n + extra, Hq), 7.0, device="cuda")
    lens = np.diff(off)
    kw = dict(T_max=int(lens.max()), o=o, lse=lse, scale=scale)
    shared = {}
    if per is not None:
        shared = dict(seg_off=offsets(per), prefix_pages=i32(pool.prefix_pages), prefix_lens=i32(pool.shared))
        if bounds:
            shared["prefix_max"] = max(pool.shared)
    if bounds:
        kw["len_max"] = max(pool.own)
    st = status()
    wm.cached_attention(q, pool.k, pool.v, i32(pool.pages), i32(pool.own), i32(off), status=st, **kw, **shared)
    if not extra:
        wm.device_status(st)
    want = Q.cached(host(q[:n]), host(pool.k), host(pool.v), pool.pages, pool.own, off, dh ** -0.5 if scale is None else scale,
                    *((offsets(per), pool.prefix_pages, pool.shared) if per is not None else ()))
    close("o", o[:n], want[0], ATTN[dtype])
    close("lse", lse[:n], want[1], LSE)
    assert (o[n:] == 7.0).all() and (lse[n:] == 7.0).all(), "rows behind the last sequence changed"
    o2 = torch.empty_like(o)
    wm.cached_attention(q, pool.k, pool.v, i32(pool.pages), i32(pool.own), i32(off), **{**kw, "o": o2}, **shared)
    assert same_bits(o[:n], o2[:n]), "another result the second time"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("page,per,T,own,shared,Hq,Hk", [
    (16, [3, 0, 2], [1] * 5, [1, 17, 16, 40, 5], [33, 8, 200], 4, 2),      # a step each; a program without sequences
    (32, [2, 3], [1] * 5, [3, 64, 31, 130, 2], [0, 70], 8, 1),             # a program without tokens
    (64, [2, 2], [33, 1, 65, 40], [33, 90, 65, 41], [129, 64], 2, 2),      # chunks, some of them the first
    (16, [1, 1], [5, 2], [70, 2], [300, 17], 6, 3),
    (128, None, [1, 1, 4], [300, 1, 129], [], 4, 4),                       # nothing shared
])
def test_cached(wm, dtype, dh, page, per, T, own, shared, Hq, Hk):
    print(f"[cached] {dtype} dim={dh} page={page} per={per} T={T} own={own} shared={shared} heads={Hq}/{Hk}", flush=True)
    pool = Pool(dtype, page, Hk, dh, own, shared, seed=dh + page)
    check_cached(wm, dtype, pool, offsets(T), per, Hq, Hk, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_long(wm, dtype):
    """Split keys, own and shared; loose bounds; rows behind the last sequence."""
    pool = Pool(dtype, 64, 1, 64, [4000, 5, 1000], [3001], seed=2, wide=7)
    check_cached(wm, dtype, pool, [0, 1, 2, 3], [3], 4, 1, 64, extra=2)
    check_cached(wm, dtype, pool, [0, 1, 2, 3], [3], 4, 1, 64, bounds=False)
    check_cached(wm, dtype, pool, [0, 1, 2, 3], None, 4, 1, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per", [None, [2, 2]])
def test_cached_rows_without_keys(wm, dtype, per):
    """Sequences with fewer keys than rows, and none: with nothing shared a row that sees no key has o = 0, lse = -inf."""
    own, shared = [0, 2, 0, 5], [0, 9] if per else []
    pool = Pool(dtype, 16, 2, 32, own, shared, seed=3, wide=1)
    check_cached(wm, dtype, pool, offsets([1, 3, 2, 5]), per, 4, 2, 32, bounds=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_values_that_are_not_finite(wm, dtype):
    """A key that a row does not see yet may hold anything; one that it sees counts."""
    T, own = [40, 3], [50, 3]
    pool = Pool(dtype, 16, 1, 32, own, [20], seed=4)
    for slot, x in ((30, float("nan")), (45, float("inf"))):
        pool.v[pool.pages[0][slot // 16], :, slot % 16, 3:5] = x
    pool.k[pool.pages[0][49 // 16], :, 49 % 16] = float("nan")
    check_cached(wm, dtype, pool, offsets(T), [2], 2, 1, 32)


# ---- prefix attention ----------------------------------------------------------------
def make_prefix(dtype, per, T, P, Hq, Hk, dh, hidden=0.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    off = offsets(T)
    n, seg = off[-1], offsets(per)
    qkv, pkv = rnd(n, Hq + 2 * Hk, dh).to(dt(dtype)), rnd(sum(P), 2, Hk, dh).to(dt(dtype))
    mask = (torch.rand(sum(P), generator=g, device="cuda") >= hidden).to(torch.uint8) if hidden else None
    return dict(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hk], v=qkv[:, Hq + Hk:], pk=pkv[:, 0], pv=pkv[:, 1], off=off,
                q_off=[off[i] for i in seg], p_off=offsets(P), mask=mask, do=rnd(n, Hq, dh).to(dt(dtype)), T_max=max(T))


def run_prefix(wm, c, scale=None, grad=True, st=None):
    x = [c[n] for n in ("q", "k", "v", "pk", "pv")]
    where = (i32(c["off"]), c["q_off"], c["p_off"])
    kw = dict(T_max=c["T_max"], kv_mask=c["mask"], scale=scale, status=st)
    f = wm.prefix_attention(*x, *where, need_lse=True, **kw)
    out = {"o": f["o"], "lse": f["lse"]}
    if grad:
        b = wm.prefix_attention_grad(c["do"], *x, f["o"], f["lse"], *where, **kw)
        out.update({n: b[n] for n in ("dq", "dk", "dv", "dpk", "dpv")})
    return out


def check_prefix(wm, dtype, c, scale=None, poison=True, tol=None):
    tol = ATTN[dtype] if tol is None else tol
    sc = c["q"].shape[2] ** -0.5 if scale is None else scale
    clean = [host(c[n]) for n in ("q", "k", "v", "pk", "pv")]
    if c["mask"] is not None and poison:                # what hidden keys hold is never used
        for n in ("pk", "pv"):
            c[n] = c[n].clone()
            c[n][c["mask"] == 0] = float("nan")
    m = None if c["mask"] is None else c["mask"].cpu().numpy()
    st = status()
    got = run_prefix(wm, c, scale, st=st)
    wm.device_status(st)
    where = (c["off"], c["q_off"], c["p_off"], sc, m)
    o, lse = Q.prefix(*clean, *where)
    close("o", got["o"], o, tol)
    close("lse", got["lse"], lse, LSE)
    # The gradient call is given o as the forward stored it, so its oracle is too; rows of few keys do without it (ds = P (dP - sum P dP),
    # the same where o is exact), so a result may be off by what o's rounding changes.  Against the gradient of the exact o a bfloat16
    # o adds to do . o up to 2^-8 of every term: the change of the oracle's results when each of them moves by that.
    true, given = (Q.prefix_grad(host(c["do"]), *clean, *where, o=x) for x in (None, host(got["o"])))
    moved = Q.prefix_grad(host(c["do"]), *clean, *where, o=o + 2.0 ** -8 * np.abs(o) * np.sign(host(c["do"])))
    spread = Q.grad_spread(host(c["do"]), *clean, *where, o=host(got["o"]))
    for n, t, g, m, s in zip(("dq", "dk", "dv", "dpk", "dpv"), true, given, moved, spread):
        close(n, got[n], g, tol, s)
        if dtype == "bf16":
            d, norm = np.linalg.norm(host(got[n]) - t), np.linalg.norm(t)
            assert d <= tol * max(norm, 1.0) + np.linalg.norm(m - t), f"{n}: {d} of {norm}"
    again = run_prefix(wm, c, scale)
    for n in got:
        assert same_bits(got[n], again[n]), f"{n}: another result the second time"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("per,T,P,Hq,Hk", [
    ([3, 2], [30, 70, 33, 129, 1], [65, 40], 2, 2),               # sequences that end inside tiles
    ([2, 0, 1], [3, 1, 2], [300, 7, 0], 6, 2),                    # few rows, groups of 3, programs without rows or tokens
    ([1], [200], [0], 4, 1),                                      # causal alone, groups of 4
    ([40], [1 + i % 5 for i in range(40)], [90], 3, 1),           # many short sequences in a tile
    ([1, 5], [0, 0, 64, 0, 1, 63], [1, 128], 2, 1),               # empty sequences at the ends
])
def test_prefix(wm, dtype, dh, per, T, P, Hq, Hk):
    print(f"[prefix] {dtype} dim={dh} per={per} T={T[:8]} P={P} heads={Hq}/{Hk}", flush=True)
    check_prefix(wm, dtype, make_prefix(dtype, per, T, P, Hq, Hk, dh, seed=dh))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,T", [([3, 2], [30, 70, 33, 129, 1]), ([1, 2], [2, 1, 3])])
def test_prefix_hidden_keys(wm, dtype, per, T):
    c = make_prefix(dtype, per, T, [70, 200], 4, 2, 64, hidden=0.4, seed=3)
    c["mask"][:70] = 0                                  # the first program shows nothing
    check_prefix(wm, dtype, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_split_loops(wm, dtype):
    """Few rows over long keys, and one long sequence of one key head: loops are split, parts joined."""
    check_prefix(wm, dtype, make_prefix(dtype, [2], [3, 2], [3000], 2, 1, 64, seed=5))
    check_prefix(wm, dtype, make_prefix(dtype, [1], [1500], [100], 2, 1, 32, seed=6))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_large_scores(wm, dtype):
    """Scores far from 0, rising along the keys: the running maximum has to follow.  In float32 the argument of the exponential,
    score - lse, is a difference of two numbers that are rounded to 2^-24 of the largest score (70 and more here, where
    the common tolerance counts 40): a weight is off by twice that."""
    c = make_prefix(dtype, [2], [90, 40], [130], 2, 2, 32, seed=7)
    c["pk"] = (c["pk"].float() * torch.linspace(0.1, 3.0, 130, device="cuda")[:, None, None]).to(dt(dtype))
    group = torch.einsum("qhd,khd->hqk", c["q"].double(), c["pk"].double()).abs().max().item()
    check_prefix(wm, dtype, c, scale=1.0, tol=ATTN[dtype] + (2 * 2.0 ** -24 * group if dtype == "f32" else 0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefix_sequences_do_not_touch(wm, dtype):
    """What is not finite in one sequence stays there: the others have the bits they have without it, and rows before it in
    its own sequence too."""
    c = make_prefix(dtype, [4], [20, 30, 9, 50], [40], 4, 2, 32, seed=8)
    good = run_prefix(wm, c, grad=False)
    a, b = c["off"][1], c["off"][2]
    for name in ("v", "k", "q"):
        d = {**c, name: c[name].clone()}
        d[name][a + 10, :, 2:7] = float("inf") if name == "v" else float("nan")
        got = run_prefix(wm, d, grad=False)
        keep = torch.ones(c["off"][-1], dtype=torch.bool, device="cuda")
        keep[a + 10:b] = False
        if name == "q":
            keep[a + 11:b] = True
        diff = (got["o"][keep].float() - good["o"][keep].float()).abs().max().item()
        assert diff <= (2.0 ** -7 if dtype == "bf16" else 1e-5), f"{name}: {diff}"
        assert not torch.isfinite(got["o"][a + 10].float()).all()
    # gradients: a sequence that is not finite leaves the other sequences' own gradients finite and unchanged
    d = {**c, "do": c["do"].clone()}
    d["do"][a + 10] = float("nan")
    ref, got = run_prefix(wm, c), run_prefix(wm, d)
    for name in ("dq", "dk", "dv"):
        keep = torch.ones(c["off"][-1], dtype=torch.bool, device="cuda")
        keep[a:b] = False
        if name == "dq":
            keep[a:b] = True
            keep[a + 10] = False
        else:
            keep[a + 11:b] = True                        # keys behind the row
        diff = (got[name][keep].float() - ref[name][keep].float()).abs().max().item()
        assert diff <= (2.0 ** -6 if dtype == "bf16" else 1e-4), f"{name}: {diff}"
