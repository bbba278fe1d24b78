"""The sequence operators where loops repeat and launches divide: gradients whose workgroups take several items, long
scans without optional inputs, more segments than a launch holds with split loops, batches that mix one-row segments with
longer ones; exact zeros, single steps and repeated calls.  Tolerances are those of test_gpu_sequence.py."""
import numpy as np
import pytest

from oracle import sequence as Q
from test_gpu_sequence import (TOL, _dt, _np, check_attn, check_scan, close, make_attn, make_conv, make_scan, offsets, torch,  # noqa: F401
                               wm)

pytestmark = pytest.mark.gpu


# ---- several items per workgroup -------------------------------------------------------
@pytest.mark.parametrize("dtype,full", [("f32", True), ("bf16", False)])
def test_scan_gradient_items(wm, dtype, full):  # noqa: F811
    """3000 sequences of up to two blocks of steps, empty ones among them, on fewer groups of workgroups."""
    lens = [int(x) for x in np.random.default_rng(80).integers(0, 13, 3000)]
    C, N = 130, 8
    a, opt, off, dy, _ = make_scan(dtype, lens, C, N, 81, full)
    s = (a["u"], a["delta"], a["A"], a["Bm"], a["Cm"], off)
    kept = wm.selective_scan(*s, T_max=max(lens), need_checkpoints=True, **opt)["checkpoints"]
    ws = wm.selective_scan_grad(dy, *s, kept, T_max=max(lens), **opt)["ws"]
    rows = 3 * sum(lens) * 2 * N * 4                     # 3 blocks of 64 channels; what is left holds the groups' sums
    groups = (ws.numel() - rows) // (C * (N + 2) * 4)
    print(f"[scan] {dtype} 3000 sequences on {groups} groups", flush=True)
    assert 0 < groups and 2 * groups < len(lens)
    check_scan(wm, dtype, lens, C, N, 81, full)


@pytest.mark.parametrize("dtype,C,W,B", [("f32", 1003, 3, 25), ("bf16", 1000, 4, 60)])
def test_conv_gradient_items(wm, dtype, C, W, B):  # noqa: F811
    lens = [0, 600] + [int(x) for x in np.random.default_rng(82).integers(0, 600, B - 2)]
    x, off, w, b, st, dy, ds = make_conv(dtype, lens, C, W, 83)
    r = wm.causal_conv_grad(dy, x, off, w, b, T_max=600, state=st, d_state_out=ds, need_dstate=True)
    groups, runs = r["ws"].numel() // ((W + 1) * C * 4), B * (600 // 16)
    print(f"[conv] {dtype} {runs} runs on {groups} groups", flush=True)
    assert 128 < groups and 2 * groups < runs            # sums of more than 128 groups are taken eight at a time
    want = Q.conv_grad(_np(dy), _np(x), offsets(lens), _np(w), _np(b), True, _np(st), _np(ds))
    for n, g, t in zip(("dx", "dweight", "dbias", "dstate"), want, (TOL[dtype], TOL["f32"], TOL["f32"], TOL[dtype])):
        close(n, r[n], g, t)


# ---- long scans without h0, dhT, gate, D and bias ------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 16, 32])
def test_scan_chunks_without_options(wm, dtype, N):  # noqa: F811
    print(f"[scan] chunks, no options, {dtype} N={N}", flush=True)
    check_scan(wm, dtype, [300, 0, 129], 20, N, 84, full=False)


# ---- attention: launches of many segments, mixed lengths -----------------------------------
def attn_bounds(do, q, k, v, qo, ko, scale, mask, eps, slop):
    """Largest error of each element of o, dq, dk, dv, from what is summed for it.  Rounded to eps of themselves: results,
    probabilities (for o and dv), score gradients, and o, which enters them through do . o (eps is half the distance of
    neighbours at 1: 2^-8 in bfloat16, which keeps 8 bits).  slop: float32 arithmetic,
    as a share of the sums of all terms' sizes.  (Against a tensor's rms, as elsewhere, no bound holds where segments of
    few and of many keys make elements of quite different size.)"""
    o, lse = Q.attention(q, k, v, qo, ko, scale, mask)
    dq, dk, dv = Q.attention_grad(do, q, k, v, qo, ko, scale, mask)
    b = [eps * np.abs(t) for t in (o, dq, dk, dv)]
    for rows, keys, h, hk in Q._segments(q, k, qo, ko, mask):
        if len(keys) == 0 or rows.stop == rows.start:
            continue
        p = np.exp(scale * (q[rows, h] @ k[keys, hk].T) - lse[rows, h, None])
        size = np.abs(do[rows, h]) @ np.abs(v[keys, hk]).T                     # of do . v
        delta = (np.abs(do[rows, h]) * np.abs(o[rows, h])).sum(1, keepdims=True)
        ds = np.abs(p * (do[rows, h] @ v[keys, hk].T - (do[rows, h] * o[rows, h]).sum(1, keepdims=True)))
        e = scale * (eps * (ds + p * delta) + slop * p * (size + delta))
        b[0][rows, h] += (eps + slop) * p @ np.abs(v[keys, hk])
        b[1][rows, h] += e @ np.abs(k[keys, hk])
        b[2][keys, hk] += e.T @ np.abs(q[rows, h])
        b[3][keys, hk] += (eps + slop) * p.T @ np.abs(do[rows, h])
    return (o, dq, dk, dv), [1.01 * x + 1e-30 for x in b]


@pytest.mark.parametrize("dtype,S,keys", [("bf16", 200, 1500), ("f32", 130, 3000)])
def test_attention_many_streams_split(wm, dtype, S, keys):  # noqa: F811
    """One row in each of more segments than a launch holds, up to `keys` keys in several splits."""
    r = np.random.default_rng(85)
    q, k, v, qo, ko, mask, do = make_attn(dtype, [1] * S, [int(x) for x in r.integers(0, keys, S)], 2, 1, 64, hidden=0.1, seed=86)
    f = wm.cross_attention(q, k, v, qo, ko, kv_mask=mask, need_lse=True)
    assert f["ws"] is not None                           # split
    b = wm.cross_attention_grad(do, q, k, v, f["o"], f["lse"], qo, ko, kv_mask=mask)
    want, most = attn_bounds(*(_np(t) for t in (do, q, k, v)), qo, ko, 0.125, mask.cpu().numpy(),
                             2.0 ** -8 if dtype == "bf16" else 2.0 ** -24, 1e-5 if dtype == "bf16" else 5e-5)
    for n, t, w, m in zip(("o", "dq", "dk", "dv"), (f["o"], b["dq"], b["dk"], b["dv"]), want, most):
        share = (np.abs(_np(t) - w) / m).max()
        print(f"[attn] {n}: {share:.2f} of its bound", flush=True)
        assert share <= 1.0, n
        assert np.linalg.norm(_np(t) - w) <= (TOL["f32"] if dtype == "f32" else TOL["bf16_attn"]) * np.linalg.norm(w), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_attention_one_row_beside_many(wm, dtype, dh):  # noqa: F811
    """Single rows in the form that takes 128 rows at a time, because one segment has more."""
    check_attn(wm, dtype, *make_attn(dtype, [1, 1, 130, 0, 1, 33], [64, 700, 90, 5, 1, 2100], 4, 2, dh, seed=87))


def test_attention_one_key_gives_zero_score_gradients(wm):  # noqa: F811
    """float32, one visible key: do . v and do . o are the same products in the same order, so dq and dk are 0."""
    for dh in (32, 64, 128):
        q, k, v, qo, ko, _, do = make_attn("f32", [3, 40, 1], [1, 1, 300], 4, 2, dh, seed=88)
        mask = torch.zeros(302, dtype=torch.uint8, device="cuda")
        mask[[0, 1, 200]] = 1
        f = wm.cross_attention(q, k, v, qo, ko, kv_mask=mask, need_lse=True)
        seg = torch.tensor([0] * 3 + [1] * 40 + [200], device="cuda")
        assert torch.equal(f["o"], v[seg].repeat_interleave(2, 1))
        b = wm.cross_attention_grad(do, q, k, v, f["o"], f["lse"], qo, ko, kv_mask=mask)
        assert (b["dq"] == 0).all() and (b["dk"] == 0).all()


# ---- single steps ----------------------------------------------------------------------
def test_conv_steps_equal_whole_f32(wm):  # noqa: F811
    x, off, w, b, st, _, _ = make_conv("f32", [7, 7], 37, 3, 89)
    whole = wm.causal_conv(x, off, w, b, T_max=7, state=st, need_state=True)
    state = st.clone()
    one = torch.arange(3, dtype=torch.int32, device="cuda")
    for t in range(7):
        f = wm.causal_conv(x.view(2, 7, 37)[:, t].contiguous(), one, w, b, T_max=1, state=state, state_out=state)
        assert torch.equal(f["y"], whole["y"].view(2, 7, 37)[:, t])
    assert torch.equal(state, whole["state"])


@pytest.mark.parametrize("N", [8, 16, 32])
def test_scan_steps_bf16(wm, N):  # noqa: F811
    """Eleven single steps in bfloat16 with the states updated in place, against the definition of the whole sequence."""
    a, opt, off, _, _ = make_scan("bf16", [11, 11, 11], 50, N, 90)
    y, hT = Q.scan(off=offsets([11] * 3), **{n: _np(t) for n, t in {**a, **opt}.items()})
    h = opt["h0"].clone()
    one = torch.arange(4, dtype=torch.int32, device="cuda")
    at = lambda x, t: x.reshape(3, 11, -1)[:, t].contiguous()  # noqa: E731
    for t in range(11):
        f = wm.selective_scan(at(a["u"], t), at(a["delta"], t), a["A"], at(a["Bm"], t), at(a["Cm"], t), one, T_max=1, D=opt["D"],
                              z=at(opt["z"], t), delta_bias=opt["delta_bias"], h0=h, hT=h)
        close(f"y {t}", f["y"], y.reshape(3, 11, -1)[:, t], TOL["bf16"])
    close("hT", h, hT, TOL["f32"])


# ---- the same bits again -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeated_calls(wm, dtype):  # noqa: F811
    """Forward and gradient calls give the same bits again, whatever memory held in between."""
    q, k, v, qo, ko, mask, do = make_attn(dtype, [1, 140, 30], [900, 300, 77], 6, 2, 64, hidden=0.2, seed=91)
    a, opt, off, dy, dhT = make_scan(dtype, [400, 3, 150], 70, 16, 92)
    s = (a["u"], a["delta"], a["A"], a["Bm"], a["Cm"], off)
    x, xo, w, b, st, cdy, ds = make_conv(dtype, [90, 0, 33], 37, 4, 93)

    def calls():
        f = wm.cross_attention(q, k, v, qo, ko, kv_mask=mask, need_lse=True)
        g = wm.cross_attention_grad(do, q, k, v, f["o"], f["lse"], qo, ko, kv_mask=mask)
        h = wm.selective_scan(*s, T_max=400, need_state=True, need_checkpoints=True, **opt)
        i = wm.selective_scan_grad(dy, *s, h["checkpoints"], T_max=400, dhT=dhT, **opt)
        c = wm.causal_conv(x, xo, w, b, T_max=90, state=st, need_state=True)
        e = wm.causal_conv_grad(cdy, x, xo, w, b, T_max=90, state=st, d_state_out=ds, need_dstate=True)
        return [(n, t) for r in (f, g, h, i, c, e) for n, t in r.items() if t is not None and n not in ("ws", "checkpoints")]
    want = [(n, t.clone()) for n, t in calls()]
    for _ in range(3):
        junk = [torch.full((1 << m,), 255, dtype=torch.uint8, device="cuda") for m in range(9, 27)]
        del junk
        for (n, t), (_, u) in zip(calls(), want):
            assert torch.equal(t, u), n
