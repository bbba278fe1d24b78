"""The operators over a shared prefix as a program uses them: whole sequences against steps through the cache, captured
steps replayed, other streams, many programs, far pages, and what the device reports.  Tolerances in prefix_util."""
import numpy as np
import pytest

from oracle import prefix as Q
from prefix_util import ATTN, LSE, TURN, Pool, close, dt, frequencies, host, i32, offsets, same_bits
from test_gpu_prefix import check_cached, check_prefix, make_prefix, run_prefix, status

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def wm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_09312_amd as wm
    wm.load_library()
    return wm


class Model:
    """One layer's rows of programs and candidates, and the cache that a rollout fills."""

    def __init__(self, dtype, P, per, T, Hq=4, Hk=2, dh=64, page=16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt(dtype))  # noqa: E731
        self.P, self.per, self.T, self.B, self.dtype = P, per, T, sum(per), dtype
        self.shape = Hq, Hk, dh, page
        self.seg = offsets(per)
        self.first = np.repeat(P, per)                                  # candidates' positions go on behind their program
        self.qkv, self.pkv = rnd(self.B * T, Hq + 2 * Hk, dh), rnd(sum(P), 2, Hk, dh)
        self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hk], self.qkv[:, Hq + Hk:]
        self.freq = frequencies(dh)

    def whole(self, wm):
        off = i32(range(0, self.B * self.T + 1, self.T))
        q, k = (wm.rotate(x, off, self.freq, T_max=self.T, first=i32(self.first))["y"] for x in (self.q, self.k))
        pk = wm.rotate(self.pkv[:, 0], i32(offsets(self.P)), self.freq, T_max=max(self.P))["y"]
        return wm.prefix_attention(q, k, self.v, pk, self.pkv[:, 1], off, [s * self.T for s in self.seg], offsets(self.P), T_max=self.T,
                                   need_lse=True)

    def start(self, wm):
        """An empty cache with the programs' keys appended."""
        Hq, Hk, dh, page = self.shape
        pool = Pool(self.dtype, page, Hk, dh, [self.T] * self.B, self.P, seed=1)
        self.pages, self.ppages, self.plens = i32(pool.pages), i32(pool.prefix_pages), i32(self.P)
        self.kc, self.vc = torch.full_like(pool.k, float("nan")), torch.full_like(pool.v, float("nan"))
        st = status()
        wm.cache_append(self.pkv[:, 0], self.pkv[:, 1], self.kc, self.vc, self.ppages, self.plens, i32(offsets(self.P)), T_max=max(self.P),
                        freq=self.freq, status=st)
        wm.device_status(st)

    def step(self, wm, q, k, v, lens, off, n, st, **kw):
        """n new rows of every candidate, lens counting them."""
        r = wm.cache_append(k, v, self.kc, self.vc, self.pages, lens, off, T_max=n, first=i32(self.first), freq=self.freq, q=q, status=st)
        return wm.cached_attention(r["q"], self.kc, self.vc, self.pages, lens, off, T_max=n, seg_off=self.seg, prefix_pages=self.ppages,
                                   prefix_lens=self.plens, need_lse=True, status=st, **kw)

    def rows(self, t, n):
        """Rows t .. t + n of every candidate, packed."""
        return lambda x: x.view(self.B, self.T, *x.shape[1:])[:, t:t + n].reshape(self.B * n, *x.shape[1:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunks", [[1] * 9, [5, 1, 3], [9]])
def test_steps_give_what_whole_sequences_give(wm, dtype, chunks):
    """Both ways round the same rotated operands; each is within the attention's tolerance of the same values, so they are within
    twice that of each other."""
    m = Model(dtype, [70, 5, 33], [3, 1, 2], 9)
    want = m.whole(wm)
    m.start(wm)
    st, t, o, lse = status(), 0, [], []
    for n in chunks:
        part = m.rows(t, n)
        lens = torch.full((m.B,), t + n, dtype=torch.int32, device="cuda")
        r = m.step(wm, part(m.q), part(m.k), part(m.v), lens, i32(range(0, m.B * n + 1, n)), n, st)
        o.append(r["o"].view(m.B, n, *r["o"].shape[1:]))
        lse.append(r["lse"].view(m.B, n, -1))
        t += n
    wm.device_status(st)
    close("o", torch.cat(o, 1).flatten(0, 1), host(want["o"]), 2 * ATTN[dtype])
    close("lse", torch.cat(lse, 1).flatten(0, 1), host(want["lse"]), 2 * LSE)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_training_through_the_rotation(wm, dtype):
    """dL/d(unrotated) = the rotation back of dL/d(rotated), against the oracle's chain."""
    m = Model(dtype, [20, 7], [2, 2], 11, seed=3)
    off, first = i32(range(0, m.B * m.T + 1, m.T)), i32(m.first)
    q, k = (wm.rotate(x, off, m.freq, T_max=m.T, first=first)["y"] for x in (m.q, m.k))
    where = (off, [s * m.T for s in m.seg], offsets(m.P))
    pk, pv = m.pkv[:, 0], m.pkv[:, 1]
    f = wm.prefix_attention(q, k, m.v, pk, pv, *where, T_max=m.T, need_lse=True)
    do = torch.randn(f["o"].shape, device="cuda").to(dt(dtype))
    b = wm.prefix_attention_grad(do, q, k, m.v, pk, pv, f["o"], f["lse"], *where, T_max=m.T)
    dq, dk = (wm.rotate(b[n], off, m.freq, T_max=m.T, first=first, inverse=True)["y"] for n in ("dq", "dk"))
    o = host(off).astype(int).tolist()
    pos = Q.positions(o, m.first)
    args = [host(t) for t in (q, k, m.v, pk, pv)] + [o, where[1], where[2], 64 ** -0.5]
    g = Q.prefix_grad(host(do), *args, o=host(f["o"]))
    for name, got, want in (("dq", dq, g[0]), ("dk", dk, g[1])):
        close(name, got, Q.rotate(want, pos, host(m.freq), inverse=True), ATTN[dtype] + TURN[dtype])


@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("T", [2, 3, 4])
def test_gradients_of_few_keys(wm, T, G):
    """Where a row sees few keys, a gradient formed with the stored bfloat16 o would be wrong by its rounding more than by anything
    else (1.4 times what is asked here, for sequences of 3).  What remains are two roundings to bfloat16, of the score gradients and
    of the results: each is spread evenly over at most half a step of 2^-8, relative to values spread over a binade 0.42 x 2^-8
    in the 2-norm; both together 0.59 x 2^-8, and a quarter more for the spread of that: 0.75 x 2^-8."""
    n = 120
    c = make_prefix("bf16", [n], [T] * n, [0], 2 * G, 2, 64, seed=T)
    got = run_prefix(wm, c)
    x = [host(c[m]) for m in ("q", "k", "v", "pk", "pv")]
    want = Q.prefix_grad(host(c["do"]), *x, c["off"], c["q_off"], c["p_off"], 64 ** -0.5)
    for name, w in zip(("dq", "dk", "dv"), want):
        close(name, got[name], w, 0.75 * 2.0 ** -8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps(wm, dtype):
    """A rollout's step captured once (append, then attention, lengths raised on the device) and replayed for every action, with
    the program's own work and synchronizations between; every replay against an eager step on a cache of its own."""
    T = 6
    eager, replayed = (Model(dtype, [40, 3], [4, 2], T, seed=5) for _ in range(2))
    eager.start(wm)
    replayed.start(wm)
    B = eager.B
    off, st = i32(range(B + 1)), status()
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    rows = [eager.rows(t, 1) for t in range(T)]
    q, k, v = (rows[0](x).contiguous() for x in (eager.q, eager.k, eager.v))
    o = torch.zeros_like(q)
    first = i32(replayed.first)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    qr = torch.empty_like(q)

    def step():
        lens.add_(1)
        wm.cache_append(k, v, replayed.kc, replayed.vc, replayed.pages, lens, off, T_max=1, first=first, freq=replayed.freq, q=q, q_out=qr, status=st)
        wm.cached_attention(qr, replayed.kc, replayed.vc, replayed.pages, lens, off, T_max=1, len_max=T, seg_off=replayed.seg,
                            prefix_pages=replayed.ppages, prefix_lens=replayed.plens, o=o, ws=ws, status=st)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    lens.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens.zero_()
    for t in range(T):
        for dst, src in ((q, eager.q), (k, eager.k), (v, eager.v)):
            dst.copy_(rows[t](src))
        o.fill_(7.0)
        graph.replay()
        want = eager.step(wm, q, k, v, torch.full((B,), t + 1, dtype=torch.int32, device="cuda"), off, 1, status(), len_max=T)["o"]
        if t % 2:
            torch.cuda.synchronize()
        assert same_bits(o, want), f"replay {t}"
    wm.device_status(st)


def test_captured_training(wm):
    """The forward and the gradient call in one graph, replayed on other values."""
    c = make_prefix("bf16", [3, 2], [30, 70, 33, 65, 1], [65, 200], 4, 2, 64, seed=11)
    off = i32(c["off"])
    x = {n: c[n].clone() for n in ("q", "k", "v", "pk", "pv", "do")}

    def go(x):
        f = wm.prefix_attention(x["q"], x["k"], x["v"], x["pk"], x["pv"], off, c["q_off"], c["p_off"], T_max=c["T_max"], need_lse=True)
        b = wm.prefix_attention_grad(x["do"], x["q"], x["k"], x["v"], x["pk"], x["pv"], f["o"], f["lse"], off, c["q_off"], c["p_off"],
                                     T_max=c["T_max"])
        return {"o": f["o"], "lse": f["lse"], **{n: b[n] for n in ("dq", "dk", "dv", "dpk", "dpv")}}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go(x)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go(x)
    for i in range(4):
        for n in x:
            x[n].copy_(c[n] * (1.0 + 0.25 * i))
        graph.replay()
        want = go({n: t.clone() for n, t in x.items()})
        if i % 2:
            torch.cuda.synchronize()
        for n in want:
            assert same_bits(out[n], want[n]), f"replay {i}: {n}"


def test_two_streams_at_once(wm):
    """Calls that share nothing but inputs, under way together on two streams."""
    a = make_prefix("bf16", [40], [64] * 40, [500], 4, 4, 64, seed=1)
    b = make_prefix("f32", [7], [30] * 7, [300], 2, 1, 32, seed=2)
    want = [run_prefix(wm, c) for c in (a, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for c, s in ((a, side), (b, None)):
        x, where = [c[n] for n in ("q", "k", "v", "pk", "pv")], (i32(c["off"]), c["q_off"], c["p_off"])
        if s is not None:
            s.wait_stream(torch.cuda.current_stream())
        kw = dict(T_max=c["T_max"], stream=s)
        f = wm.prefix_attention(*x, *where, need_lse=True, **kw)
        g = wm.prefix_attention_grad(c["do"], *x, f["o"], f["lse"], *where, **kw)
        got.append({"o": f["o"], "lse": f["lse"], **{n: g[n] for n in ("dq", "dk", "dv", "dpk", "dpv")}})
    torch.cuda.current_stream().wait_stream(side)
    for w, g in zip(want, got):
        for n in w:
            assert same_bits(w[n], g[n]), n


@pytest.mark.parametrize("per", [1, 3])
def test_many_programs(wm, per):
    """More programs than a launch's table holds, some without sequences, tokens or rows."""
    S = 300
    r = np.random.default_rng(7)
    P, counts = r.integers(0, 40, S), [per] * S
    P[5], counts[7], counts[299] = 0, 0, 0
    T = r.integers(0, 4, sum(counts))
    T[0] = 3
    check_prefix(wm, "bf16", make_prefix("bf16", counts, T, [int(p) for p in P], 2, 1, 32, seed=8))
    L = [int(t) + int(x) for t, x in zip(T, r.integers(0, 30, len(T)))]
    pool = Pool("bf16", 16, 1, 32, L, [int(p) for p in P], seed=9, wide=1)
    check_cached(wm, "bf16", pool, offsets(T), counts, 2, 1, 32)
    check_cached(wm, "bf16", pool, offsets([int(n > 0) for n in L]), counts, 2, 1, 32)         # single steps


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [5, 16, 32])
def test_wide_groups(wm, dtype, G):
    """Groups that do not divide a tile's rows, and that fill them."""
    check_prefix(wm, dtype, make_prefix(dtype, [2, 1], [3, 40, 130], [70, 5], 2 * G, 2, 32, seed=G))
    check_prefix(wm, dtype, make_prefix(dtype, [1], [70], [40], G, 1, 128, seed=G))
    pool = Pool(dtype, 32, 2, 32, [40, 5, 90], [100, 31], seed=G)
    check_cached(wm, dtype, pool, [0, 1, 3, 4], [2, 1], 2 * G, 2, 32)


def test_pages_past_32_bits(wm):
    """A pool of more than 2^32 bytes: keys in its first and its last pages."""
    Hk, dh, page, n = 8, 128, 64, 40000
    kc, vc = (torch.empty((n, Hk, page, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert kc.numel() * 2 > 1 << 32
    used = [n - 1, 0, n - 2, n // 2 + 1]
    for t in (kc, vc):
        t[used] = torch.randn((len(used), Hk, page, dh), device="cuda").bfloat16()
    tables, lens, off = i32([used[:2], used[2:]]), [100, 128], [0, 1, 2]
    qkv = torch.randn((2, 4 * Hk, dh), device="cuda").bfloat16()
    q, k, v = qkv[:, :2 * Hk], qkv[:, 2 * Hk:3 * Hk], qkv[:, 3 * Hk:]
    st = status()
    wm.cache_append(k, v, kc, vc, tables, i32(lens), i32(off), T_max=1, status=st)
    assert same_bits(kc[0, :, 35], k[0]) and same_bits(vc[n // 2 + 1, :, 63], v[1])
    o = wm.cached_attention(q, kc, vc, tables, i32(lens), i32(off), T_max=1, status=st)["o"]
    wm.device_status(st)
    at = {p: i for i, p in enumerate(used)}
    small = [host(t[used]) for t in (kc, vc)]
    pages = np.array([[at[p] for p in row] for row in (used[:2], used[2:])])
    close("o", o, Q.cached(host(q), *small, pages, lens, off, dh ** -0.5)[0], ATTN["bf16"])


def test_the_device_reports(wm):
    """Offsets, lengths and pages that do not fit are reported, and what is in the caches and behind the rows stays."""
    Hq, Hk, dh, page = 2, 1, 32, 16
    pool = Pool("f32", page, Hk, dh, [20, 5], [9], seed=1)
    q, k = torch.randn((3, Hq, dh), device="cuda"), torch.randn((3, Hk, dh), device="cuda")
    good = dict(pages=pool.pages, lens=[20, 5], off=[0, 2, 3])
    bad = [("page", dict(pages=np.array([[pool.pages[0][0], 10 ** 6], [-1, -1]]))), ("keys", dict(lens=[20, 33])), ("keys", dict(lens=[-1, 5])),
           ("offsets", dict(off=[1, 2, 3])), ("offsets", dict(off=[0, 2, 2])), ("length", dict(off=[0, 3, 2])), ("length", dict(off=[0, 0, 3]))]
    for what, kw in [("", {})] + bad:
        a = {**good, **kw}
        pages, lens, off = i32(a["pages"]), i32(a["lens"]), i32(a["off"])
        for name in ("append", "cached", "shared"):
            kc, vc, st = pool.k.clone(), pool.v.clone(), status()
            if name == "append":
                wm.cache_append(k, k, kc, vc, pages, lens, off, T_max=2, q=q, status=st)
            elif name == "cached":
                wm.cached_attention(q, kc, vc, pages, lens, off, T_max=2, status=st)
            else:
                wm.cached_attention(q, kc, vc, pages, lens, off, T_max=2, status=st, seg_off=[0, 2], prefix_pages=i32(pool.prefix_pages),
                                    prefix_lens=i32([9]))
            if not what:
                wm.device_status(st)
                continue
            with pytest.raises(wm.WMError) as e:
                wm.device_status(st)
            assert e.value.status == 5 and what in str(e.value), (name, what)
            wm.device_status(st)                                         # cleared
            if name != "append":
                assert same_bits(kc, pool.k) and same_bits(vc, pool.v)
    st = status()
    wm.cached_attention(q, pool.k, pool.v, i32(pool.pages), i32([20, 5]), i32([0, 2, 3]), T_max=2, status=st, seg_off=[0, 2],
                        prefix_pages=i32(pool.prefix_pages), prefix_lens=i32([17]))
    with pytest.raises(wm.WMError):
        wm.device_status(st)
    wm.cache_append(k, k, pool.k, pool.v, i32(pool.pages), i32([20, 5]), i32([0, 2, 2]), T_max=2, status=st)
    with pytest.raises(wm.WMError):
        wm.device_status(st)
    x = torch.randn((3, Hq, dh), device="cuda")
    for off in ([1, 2, 3], [0, 2, 2], [0, 3, 2]):
        y = torch.full_like(x, 7.0)
        wm.rotate(x, i32(off), frequencies(dh), T_max=2, y=y, status=st)
        with pytest.raises(wm.WMError):
            wm.device_status(st)
        if off == [0, 2, 2]:
            assert (y[2] == 7.0).all()
        wm.prefix_attention(x, x[:, :1], x[:, :1], x[:, :1], x[:, :1], i32(off), [0, 3], [0, 3], T_max=2, status=st)
        with pytest.raises(wm.WMError):
            wm.device_status(st)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_garbage_workspaces(wm, dtype):
    """What a workspace holds before a call does not matter."""
    c = make_prefix(dtype, [2, 2], [3, 2, 5, 200], [3000, 40], 2, 1, 64, seed=12)
    want = run_prefix(wm, c)
    x, where = [c[n] for n in ("q", "k", "v", "pk", "pv")], (i32(c["off"]), c["q_off"], c["p_off"])
    pool = Pool(dtype, 64, 1, 64, [900, 5], [3001], seed=2)
    a = (torch.randn((2, 2, 64), device="cuda").to(dt(dtype)), pool.k, pool.v, i32(pool.pages), i32(pool.own), i32([0, 1, 2]))
    kw = dict(T_max=1, seg_off=[0, 2], prefix_pages=i32(pool.prefix_pages), prefix_lens=i32(pool.shared))
    ref = wm.cached_attention(*a, **kw)["o"]
    for fill in (0, 0xFF, 0x7F):
        ws = torch.full((1 << 26,), fill, dtype=torch.uint8, device="cuda")
        f = wm.prefix_attention(*x, *where, T_max=c["T_max"], need_lse=True, ws=ws)
        ws.fill_(fill)
        b = wm.prefix_attention_grad(c["do"], *x, f["o"], f["lse"], *where, T_max=c["T_max"], ws=ws)
        for n, t in (("o", f["o"]), *((n, b[n]) for n in ("dq", "dk", "dv", "dpk", "dpv"))):
            assert same_bits(t, want[n]), f"{n}: workspace of {fill}"
        ws.fill_(fill)
        assert same_bits(wm.cached_attention(*a, ws=ws, **kw)["o"], ref), f"cached: workspace of {fill}"


def test_nothing_to_do(wm):
    """No rows, no sequences, no programs' keys."""
    x, f, e = torch.zeros((0, 2, 32), device="cuda"), frequencies(32), i32([0])
    assert wm.rotate(x, e, f, T_max=0)["y"].shape == x.shape
    kc = torch.zeros((1, 2, 16, 32), device="cuda")
    none = torch.zeros((0, 0), dtype=torch.int32, device="cuda")
    wm.cache_append(x, x, kc, kc.clone(), none, i32([]), e, T_max=0, freq=f)
    assert wm.cached_attention(x, kc, kc.clone(), none, i32([]), e, T_max=0)["o"].shape == x.shape
    o = wm.prefix_attention(x, x, x, x, x, e, [0, 0], [0, 0], T_max=0, need_lse=True)
    g = wm.prefix_attention_grad(x, x, x, x, x, x, o["o"], o["lse"], e, [0, 0], [0, 0], T_max=0)
    assert all(g[n].numel() == 0 for n in ("dq", "dk", "dv", "dpk", "dpv"))
    p = torch.randn((5, 2, 32), device="cuda")
    g = wm.prefix_attention_grad(x, x, x, x, p, p, o["o"], o["lse"], e, [0, 0], [0, 5], T_max=0)
    assert (g["dpk"] == 0).all() and (g["dpv"] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,G,P", [([11, 3], 4, [70, 5]), ([16, 0, 4], 4, [700, 3, 0]), ([50], 5, [513]), ([9, 30], 8, [17, 90])])
def test_single_steps_of_wide_beams(wm, dtype, per, G, P):
    """Programs of more rows than a tile of the single steps' kernel, on both sides of the rule that chooses their kernel."""
    lens = [1 + (7 * i) % 40 for i in range(sum(per))]
    for dh in (32, 64, 128):
        pool = Pool(dtype, 16, 2, dh, lens, P, seed=dh)
        check_cached(wm, dtype, pool, list(range(sum(per) + 1)), per, 2 * G, 2, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,T,P,Hq,Hk", [([9, 12], 40, [900, 700], 2, 2), ([3, 2], 70, [90, 17], 2, 1), ([5, 0, 6], 130, [400, 9, 0], 3, 3)])
def test_chunks_of_many_rows(wm, dtype, per, T, P, Hq, Hk):
    """Sequences of more rows than the single steps' kernel takes, on both sides of the rule whether they read their program's keys
    themselves."""
    n = [T - (11 * i) % 37 for i in range(sum(per))]
    L = [x + (13 * i) % 50 for i, x in enumerate(n)]
    for dh in (32, 64, 128):
        pool = Pool(dtype, 32, Hk, dh, L, P, seed=dh)
        check_cached(wm, dtype, pool, offsets(n), per, Hq, Hk, dh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("per,T,P,extra", [([3, 2], [30, 70, 33, 129, 1], [65, 40], 150), ([1, 1], [3, 2], [2000, 90], 2), ([1], [700], [0], 40), ([1], [0], [70], 9)])
def test_rows_behind_the_last_sequence(wm, dtype, per, T, P, extra):
    """Padding of packed rows, here NaN: its results stay, and others' results and gradients are those without it."""
    c = make_prefix(dtype, per, T, P, 4, 2, 64, seed=5)
    n = c["off"][-1]
    x = {}
    for m in ("q", "k", "v", "do"):
        x[m] = torch.full((n + extra, *c[m].shape[1:]), float("nan"), dtype=c[m].dtype, device="cuda")
        x[m][:n] = c[m]
    rows = [x["q"], x["k"], x["v"], c["pk"], c["pv"]]
    where = (i32(c["off"]), c["q_off"][:-1] + [n + extra], c["p_off"])
    o = torch.full((n + extra, 4, 64), 7.0, dtype=x["q"].dtype, device="cuda")
    lse = torch.full((n + extra, 4), 7.0, device="cuda")
    kw = dict(T_max=max(T) + extra)
    wm.prefix_attention(*rows, *where, o=o, lse=lse, **kw)
    assert (o[n:] == 7.0).all() and (lse[n:] == 7.0).all()
    g = wm.prefix_attention_grad(x["do"], *rows, o, lse, *where, **kw)
    clean = [host(c[m]) for m in ("q", "k", "v", "pk", "pv")] + [c["off"], c["q_off"], c["p_off"], 0.125]
    close("o", o[:n], Q.prefix(*clean)[0], ATTN[dtype])
    spread = Q.grad_spread(host(c["do"]), *clean, None, host(o[:n]))
    for m, want, s in zip(("dq", "dk", "dv", "dpk", "dpv"), Q.prefix_grad(host(c["do"]), *clean, o=host(o[:n])), spread):
        close(m, g[m][:n] if m in ("dq", "dk", "dv") else g[m], want, ATTN[dtype], s)
