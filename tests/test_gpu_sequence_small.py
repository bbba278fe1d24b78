"""The sequence operators' smallest gradient calls (workspaces of a few bytes, no rows at all) against the float64
oracle, with the tolerances of test_gpu_sequence.py."""
import pytest

from oracle import sequence as Q
from test_gpu_sequence import TOL, _np, check_attn, check_scan, close, make_attn, make_conv, make_scan, offsets, torch, wm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,keys,dh", [(1, 12, 77, 64), (2, 4, 9, 32), (8, 4, 60, 64), (1, 32, 100, 128), (3, 8, 0, 32)])
def test_attention(wm, dtype, rows, heads, keys, dh):  # noqa: F811
    print(f"[attn] {dtype} rows={rows} heads={heads} keys={keys} dh={dh}", flush=True)
    check_attn(wm, dtype, *make_attn(dtype, [rows], [keys], heads, heads, dh, seed=50))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,C,W", [([16], 16, 3), ([9], 21, 2), ([8, 8], 8, 3), ([1], 1, 2), ([0, 0], 4, 4)])
def test_conv(wm, dtype, lens, C, W):  # noqa: F811
    print(f"[conv] {dtype} lens={lens} C={C} W={W}", flush=True)
    x, off, w, b, st, dy, ds = make_conv(dtype, lens, C, W, 51)
    r = wm.causal_conv_grad(dy, x, off, w, b, T_max=max(lens), state=st, d_state_out=ds, need_dstate=True)
    want = Q.conv_grad(_np(dy), _np(x), offsets(lens), _np(w), _np(b), True, _np(st), _np(ds))
    for n, g, t in zip(("dx", "dweight", "dbias", "dstate"), want, (TOL[dtype], TOL["f32"], TOL["f32"], TOL[dtype])):
        close(n, r[n], g, t)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,C,N", [([1], 1, 8), ([0, 0, 0], 6, 8), ([2], 3, 16)])
def test_scan(wm, dtype, lens, C, N):  # noqa: F811
    print(f"[scan] {dtype} lens={lens} C={C} N={N}", flush=True)
    check_scan(wm, dtype, lens, C, N, 52)


def test_scan_without_sequences(wm):  # noqa: F811
    """No sequences, no rows: the weights' gradients are 0."""
    a, _, _, dy, _ = make_scan("f32", [], 3, 8, 53, full=False)
    off = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (a["u"], a["delta"], a["A"], a["Bm"], a["Cm"], off)
    f = wm.selective_scan(*args, T_max=0, need_checkpoints=True)
    r = wm.selective_scan_grad(dy, *args, f["checkpoints"], T_max=0)
    assert (r["dA"] == 0).all() and (r["dD"] == 0).all() and (r["ddelta_bias"] == 0).all()
