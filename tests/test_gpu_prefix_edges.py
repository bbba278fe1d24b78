"""The operators over a shared prefix where their statements are tightest: far positions, lengths of programs that no sequence
reads, gradients of rows that see few keys, batches of sequences that differ widely,
outputs that a program gives, hidden keys in a cache."""
import numpy as np
import pytest

from oracle import prefix as Q
from prefix_util import ATTN, Pool, close, dt, frequencies, host, i32, offsets, same_bits
from test_gpu_prefix import check_cached, make_prefix, run_prefix, status

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def wm():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_09312_amd as wm
    wm.load_library()
    return wm


# ---- far positions -------------------------------------------------------------------
PI_DIGITS = 314159265358979323846264338327950288419716939937510582097494459230781640628620899


def sines(position, freq):
    """sin and cos of position x freq: whole turns are taken off in integers, from pi to 80 digits."""
    bits = 200
    per_turn = (10 ** 80 << bits) // (2 * PI_DIGITS)                   # 2^200 / (2 pi)
    out = np.zeros((len(position), len(freq), 2))
    for j, f in enumerate(np.asarray(freq, np.float32)):
        num, den = float(f).as_integer_ratio()
        for i, p in enumerate(position):
            turns = int(p) * num * per_turn % (den << bits)
            angle = 2.0 * np.pi * (turns * (1 << 60) // (den << bits)) / 2.0 ** 60
            out[i, j] = np.sin(angle), np.cos(angle)
    return out


FAR = [2 ** 31 - 1, 2 ** 31 - 54321, 2 ** 30 + 7, -2 ** 31, -2 ** 31 + 99, 2 ** 24 + 1, 0, 1, -1]


@pytest.mark.parametrize("op", ["rotate", "append"])
def test_angles_of_far_positions(wm, op):
    """A pair (1, 0) turns to (cos, sin), which float32 products leave as they are: the angle's error and the sums' of sine and cosine,
    2e-7 together at every int32 position, frequencies above 1 among them."""
    r = np.random.default_rng(3)
    at = FAR + r.integers(2 ** 30, 2 ** 31, 60).tolist() + r.integers(-2 ** 31, -2 ** 30, 30).tolist()
    n, dh = len(at), 128
    freq = np.concatenate([10000.0 ** (-np.arange(32) / 32.0), 1.0 + r.random(16), 2.0 ** r.uniform(0, 20, 16)]).astype(np.float32)
    f = torch.tensor(freq, device="cuda")
    x = torch.zeros((n, 1, dh), device="cuda")
    x[..., :dh // 2] = 1.0
    off = i32(range(n + 1))
    if op == "rotate":
        y = wm.rotate(x, off, f, T_max=1, first=i32(at))["y"]
    else:
        kc, vc = (torch.zeros((n, 1, 16, dh), device="cuda") for _ in range(2))
        first = [min(p, 2 ** 31 - 1) - 2 if p > -2 ** 31 + 2 else p for p in at]         # slot 2
        at = [p + 2 for p in first]
        wm.cache_append(x, x, kc, vc, i32(np.arange(n)[:, None]), i32([3] * n), off, T_max=1, first=i32(first), freq=f)
        y = kc[:, :, 2]
    got, want = host(y)[:, 0], sines(at, freq)
    worst = max(np.abs(got[:, :dh // 2] - want[..., 1]).max(), np.abs(got[:, dh // 2:] - want[..., 0]).max())
    assert worst <= 2e-7, worst


# ---- lengths of programs -------------------------------------------------------------
@pytest.mark.parametrize("n,T_max", [([1, 1, 1], 1), ([40, 1, 3], 40)])
@pytest.mark.parametrize("lens,pages,most", [([0, 5], 1, 0), ([0, -1], 1, 0), ([3, 0], 0, 0), ([0, 17], 1, 16), ([9, 5], 1, 8)])
def test_lengths_of_programs_are_reported(wm, n, T_max, lens, pages, most):
    """A program's length that is negative or passes prefix_max, also where that is 0, where the table has no pages, and where the
    program has no sequences."""
    off, own = offsets(n), [50, 9, 5]
    kc = torch.randn((16, 1, 16, 32), device="cuda")
    q = torch.randn((off[-1], 2, 32), device="cuda")
    table = i32(np.arange(12).reshape(3, 4))
    for seg_off in ([0, 2, 3], [0, 3, 3], [0, 0, 3]):
        for good in (True, False):
            st = status()
            wm.cached_attention(q, kc, kc, table, i32(own), i32(off), T_max=T_max, len_max=64, seg_off=seg_off,
                                prefix_pages=i32(12 + np.arange(2 * pages).reshape(2, pages)), prefix_lens=i32([min(max(x, 0), most) if good else x for x in lens]),
                                prefix_max=most, status=st)
            if good:
                wm.device_status(st)
                continue
            with pytest.raises(wm.WMError) as e:
                wm.device_status(st)
            assert e.value.status == 5 and "keys" in str(e.value), seg_off


# ---- gradients of rows that see few keys -----------------------------------------------
# Two roundings to bfloat16 remain, of the score gradients and of the results: each is spread evenly over at most half a step of
# 2^-8, relative to values spread over a binade 0.42 x 2^-8 in the 2-norm; both together 0.59 x 2^-8, and a quarter more for the
# spread of that.  The stored o's rounding would add as much again.
FEW = 0.75 * 2.0 ** -8


@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_gradients_of_few_keys_beside_many(wm, dh, G):
    """Short sequences that share a workgroup's rows with the end of a long one."""
    T = ([200] + [3] * 25) * 8
    c = make_prefix("bf16", [len(T)], T, [0], 2 * G, 2, dh, seed=dh + G)
    got = run_prefix(wm, c)
    want = Q.prefix_grad(host(c["do"]), *[host(c[m]) for m in ("q", "k", "v", "pk", "pv")], c["off"], c["q_off"], c["p_off"], dh ** -0.5)
    short = np.repeat(np.array(T) == 3, T)
    for name, w in zip(("dq", "dk", "dv"), want):
        close(name, got[name][torch.tensor(short, device="cuda")], w[short], FEW)


@pytest.mark.parametrize("hidden", [False, True])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("P", [1, 2, 3, 4])
def test_gradients_of_few_keys_with_a_program(wm, P, G, hidden):
    """Programs of few keys, some of them hidden (and NaN)."""
    S, n = 12, 10
    T = [2 + i % 3 for i in range(S * n)]
    c = make_prefix("bf16", [n] * S, T, [P] * S, 2 * G, 2, 64, seed=P)
    clean = [host(c[m]) for m in ("q", "k", "v", "pk", "pv")]
    if hidden:
        c["mask"] = torch.ones(S * P, dtype=torch.uint8, device="cuda")
        c["mask"][::3] = 0
        for m in ("pk", "pv"):
            c[m] = c[m].clone()
            c[m][::3] = float("nan")
    got = run_prefix(wm, c)
    want = Q.prefix_grad(host(c["do"]), *clean, c["off"], c["q_off"], c["p_off"], 0.125, None if c["mask"] is None else c["mask"].cpu().numpy())
    for name, w in zip(("dq", "dk", "dv", "dpk", "dpv"), want):
        close(name, got[name], w, FEW)


# ---- sequences that differ widely ------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,G,Hk", [(32, 1, 2), (64, 4, 1), (128, 3, 2)])
@pytest.mark.parametrize("T,per,shared", [
    ([300] + [1] * 20 + [0, 7, 130], None, []),                            # tiles dealt out by rows
    ([1] * 30 + [0] * 40 + [257] + [2] * 9, [10, 0, 70], [90, 5, 40]),     # programs beside them, one without sequences
    ([0] * 70 + [513, 0, 0] + [1] * 200 + [0] * 3, [100, 176], [700, 0]),  # empty ones first and last
])
def test_chunks_among_single_steps(wm, dtype, dh, G, Hk, T, per, shared):
    own = [t + (5 * i) % 23 for i, t in enumerate(T)]
    pool = Pool(dtype, 16, Hk, dh, own, shared, seed=dh, wide=1)
    check_cached(wm, dtype, pool, offsets(T), per, G * Hk, Hk, dh, extra=3)


@pytest.mark.parametrize("S", [1, 200])
def test_many_sequences_and_one_long(wm, S):
    """More workgroups than the library takes if every sequence had the longest one's; the longest comes first, in the middle and last, and
    T_max is larger than any."""
    B, n = 20000, 900
    for at in (0, B // 2, B - 1):
        T = np.ones(B, int)
        T[at] = n
        off = offsets(T)
        r = np.random.default_rng(at)
        k = torch.randn((64, 2, 16, 32), device="cuda").bfloat16()
        v = torch.randn((64, 2, 16, 32), device="cuda").bfloat16()
        pages, lens = r.integers(0, 64, (B, 60)), np.where(T > 1, T + 3, 2 + np.arange(B) % 9)
        q = torch.randn((off[-1], 32, 32), device="cuda").bfloat16()
        seg, table, plens = np.linspace(0, B, S + 1).astype(int), r.integers(0, 64, (S, 2)), np.arange(S) % 30
        st = status()
        o = wm.cached_attention(q, k, v, i32(pages), i32(lens), i32(off), T_max=40000, len_max=960, seg_off=seg, prefix_pages=i32(table),
                                prefix_lens=i32(plens), status=st)["o"]
        wm.device_status(st)
        for s in (0, 1, at - 1, at, at + 1, B - 2, B - 1):
            if not 0 <= s < B:
                continue
            p = int(np.searchsorted(seg, s, side="right")) - 1
            want = Q.cached(host(q[off[s]:off[s + 1], :4]), host(k[:, :1]), host(v[:, :1]), pages[s:s + 1], lens[s:s + 1], [0, int(T[s])], 32 ** -0.5,
                            [0, 1], table[p:p + 1], plens[p:p + 1])[0]
            close(f"o of {s}", o[off[s]:off[s + 1], :4], want, ATTN["bf16"])


def test_bad_offsets_of_chunks_are_reported(wm):
    """Offsets that decrease, pass the rows or sequences that pass T_max, where tiles are dealt out by rows: reported, the caches as they
    were, rows that no sequence has too."""
    B, n = 40, 300
    T = [1] * (B - 1) + [n - B + 1]
    good = offsets(T)
    kc, vc = (torch.randn((8, 1, 16, 32), device="cuda") for _ in range(2))
    q = torch.randn((n + 50, 2, 32), device="cuda")
    pages, lens = i32(np.arange(B * 24).reshape(B, 24) % 8), i32([t + 2 for t in T])
    keep = kc.clone(), vc.clone()
    for what, off, rows in (("", good, n), ("length", good[:20] + [0] + good[21:], n), ("offsets", [x - 5 for x in good], n), ("offsets", good, n + 50),
                            ("length", good[:-2] + [good[-1], good[-2]], n), ("length", good[:5] + [1 << 30] + good[6:], n),
                            ("length", [0] + [-(1 << 30)] * (B - 1) + [n], n)):
        st, o = status(), torch.full((n + 50, 2, 32), 7.0, device="cuda")
        wm.cached_attention(q[:rows], kc, vc, pages, lens, i32(off), T_max=n - B + 1, len_max=300, o=o[:rows], status=st)
        if what:
            with pytest.raises(wm.WMError) as e:
                wm.device_status(st)
            assert e.value.status == 5 and what in str(e.value), str(e.value)
        else:
            wm.device_status(st)
        assert (o[n:] == 7.0).all() and same_bits(kc, keep[0]) and same_bits(vc, keep[1])


# ---- outputs that a program gives ------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_outputs_of_the_caller(wm, dtype):
    """Gradients into given tensors, strided ones among them: rows behind the last sequence stay."""
    c = make_prefix(dtype, [2, 2], [30, 5, 70, 9], [40, 90], 4, 2, 64, seed=9)
    n, extra = c["off"][-1], 7
    x = {}
    for m in ("q", "k", "v", "do"):
        x[m] = torch.full((n + extra, *c[m].shape[1:]), float("nan"), dtype=c[m].dtype, device="cuda")
        x[m][:n] = c[m]
    where = (i32(c["off"]), c["q_off"][:-1] + [n + extra], c["p_off"])
    o, lse = torch.zeros_like(x["q"]), torch.zeros((n + extra, 4), device="cuda")
    rows = (x["q"], x["k"], x["v"], c["pk"], c["pv"])
    wm.prefix_attention(*rows, *where, T_max=70, o=o, lse=lse)
    want = wm.prefix_attention_grad(x["do"], *rows, o, lse, *where, T_max=70)
    dqkv = torch.full((n + extra, 8, 64), 7.0, dtype=dt(dtype), device="cuda")
    dpkv = torch.full((130, 2, 2, 64), 7.0, dtype=dt(dtype), device="cuda")
    out = dict(dq=dqkv[:, :4], dk=dqkv[:, 4:6], dv=dqkv[:, 6:], dpk=dpkv[:, 0], dpv=dpkv[:, 1])
    r = wm.prefix_attention_grad(x["do"], *rows, o, lse, *where, T_max=70, **out)
    assert (dqkv[n:] == 7.0).all()
    for m, t in out.items():
        assert r[m] is t and same_bits(*(y[:n] if m in ("dq", "dk", "dv") else y for y in (t, want[m]))), m


# ---- hidden keys -----------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hidden_keys_left_out_of_the_pages(wm, dtype):
    """Programs with hidden tokens: a mask over packed rows, and in a cache runs of shown tokens turned at their own positions.  Both
    see the same operands, so they are within twice the attention's tolerance of each other."""
    P, n, Hq, Hk, dh, page = [40, 23], 5, 4, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dt(dtype))  # noqa: E731
    pk, pv, q, k, v = rnd(sum(P), Hk, dh), rnd(sum(P), Hk, dh), rnd(2 * n, Hq, dh), rnd(2 * n, Hk, dh), rnd(2 * n, Hk, dh)
    mask = (torch.rand(sum(P), generator=g, device="cuda") > 0.4).to(torch.uint8)
    f, p_off, off = frequencies(dh), offsets(P), i32([0, n, 2 * n])
    whole = wm.rotate(pk, i32(p_off), f, T_max=max(P))["y"]
    o = wm.prefix_attention(q, k, v, whole, pv, off, [0, n, 2 * n], p_off, T_max=n, kv_mask=mask)["o"]

    shown = np.nonzero(mask.cpu().numpy())[0]
    runs = np.split(shown, np.nonzero((np.diff(shown) > 1) | np.isin(shown[1:], p_off))[0] + 1)
    at = torch.tensor(shown, device="cuda")
    first = [r[0] - p_off[int(np.searchsorted(p_off, r[0], side="right")) - 1] for r in runs]
    turned = wm.rotate(pk[at], i32(offsets([len(r) for r in runs])), f, T_max=max(len(r) for r in runs), first=i32(first))["y"]
    assert same_bits(turned, whole[at])
    lens = [int(((shown >= a) & (shown < b)).sum()) for a, b in zip(p_off, p_off[1:])]
    kc, vc = (torch.zeros((10, Hk, page, dh), dtype=dt(dtype), device="cuda") for _ in range(2))
    table, own = i32(np.arange(6).reshape(2, 3)), i32([[6], [7]])
    wm.cache_append(turned, pv[at], kc, vc, table, i32(lens), i32(offsets(lens)), T_max=max(lens))
    wm.cache_append(k, v, kc, vc, own, i32([n, n]), off, T_max=n)
    c = wm.cached_attention(q, kc, vc, own, i32([n, n]), off, T_max=n, seg_off=[0, 1, 2], prefix_pages=table, prefix_lens=i32(lens))["o"]
    close("o", c, host(o), 2 * ATTN[dtype])
