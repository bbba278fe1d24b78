"""What the sequence operators refuse, before anything reaches a device (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B

FAKE = 4096            # an aligned address that is never read


def _host(a):
    if a is None:
        return None, None
    a = np.asarray(a, np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p).value


def attention(q_off=(0, 4), k_off=(0, 9), **kw):
    qa, qp = _host(q_off)
    ka, kp = _host(k_off)
    a = B.Attention(dtype=B.WM_BF16, heads=4, kv_heads=2, head_dim=64, S=len(ka) - 1, q_off=qp, k_off=kp, q=FAKE, k=FAKE, v=FAKE,
                    ld_q=256, ld_k=128, ld_v=128, scale=0.125)
    for n, x in kw.items():
        setattr(a, n, x)
    a.keep = (qa, ka)
    return a


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=7), B.WM_ERR_INVALID_ARGUMENT),
    (dict(heads=3), B.WM_ERR_INVALID_ARGUMENT),           # not a multiple of kv_heads
    (dict(kv_heads=0), B.WM_ERR_INVALID_ARGUMENT),
    (dict(head_dim=48), B.WM_ERR_UNSUPPORTED),
    (dict(scale=0.0), B.WM_ERR_INVALID_ARGUMENT),
    (dict(scale=float("nan")), B.WM_ERR_INVALID_ARGUMENT),
    (dict(scale=float("inf")), B.WM_ERR_INVALID_ARGUMENT),
    (dict(q_off=None), B.WM_ERR_INVALID_ARGUMENT),
    (dict(S=0), B.WM_ERR_INVALID_ARGUMENT),
    (dict(S=513), B.WM_ERR_INVALID_ARGUMENT),
    (dict(q=None), B.WM_ERR_INVALID_ARGUMENT),
    (dict(k=FAKE + 8), B.WM_ERR_INVALID_ARGUMENT),        # not 16-byte aligned
    (dict(ld_v=120), B.WM_ERR_INVALID_ARGUMENT),          # rows overlap
    (dict(ld_k=132), B.WM_ERR_INVALID_ARGUMENT),          # rows not 16-byte aligned
    (dict(ld_q=1 << 23), B.WM_ERR_INVALID_ARGUMENT),
])
def test_attention_refuses(kw, want):
    lib = wm.load_library()
    a = attention(**kw)
    ws = ctypes.c_void_p(FAKE)
    assert lib.wm_cross_attention(a, FAKE, 256, None, ws, 1 << 30, None) == want
    assert lib.wm_last_error().decode() != ""
    assert lib.wm_cross_attention_grad(a, FAKE, 256, FAKE, FAKE, 256, FAKE, 256, FAKE, 128, FAKE, 128, ws, 1 << 30, None) == want
    assert lib.wm_cross_attention_workspace_bytes(a, 0) == 0 and lib.wm_cross_attention_workspace_bytes(a, 1) == 0


@pytest.mark.parametrize("q_off,k_off", [((1, 4), (0, 9)), ((0, 4), (2, 9)), ((0, 5, 4), (0, 3, 9)), ((0, 2, 4), (0, 9, 3))])
def test_attention_refuses_bad_tables(q_off, k_off):
    assert wm.load_library().wm_cross_attention(attention(q_off, k_off), FAKE, 256, None, None, 0, None) == B.WM_ERR_INVALID_ARGUMENT


def test_attention_refuses_outputs_and_workspace():
    lib = wm.load_library()
    bad = B.WM_ERR_INVALID_ARGUMENT
    a = attention()
    assert lib.wm_cross_attention(a, None, 256, None, None, 0, None) == bad
    assert lib.wm_cross_attention(a, FAKE, 128, None, None, 0, None) == bad
    n = lib.wm_cross_attention_workspace_bytes(a, 1)
    assert n > 0
    for args in ((None, n), (FAKE, n - 1), (FAKE + 16, n)):
        assert lib.wm_cross_attention_grad(a, FAKE, 256, FAKE, FAKE, 256, FAKE, 256, FAKE, 128, FAKE, 128, *args, None) == bad
    assert lib.wm_cross_attention_grad(a, FAKE, 256, None, FAKE, 256, FAKE, 256, FAKE, 128, FAKE, 128, FAKE, n, None) == bad
    assert lib.wm_cross_attention(None, FAKE, 256, None, None, 0, None) == bad
    long = attention((0, 1), (0, 100000))                 # split keys need a workspace
    assert lib.wm_cross_attention(long, FAKE, 256, None, None, 0, None) == bad


def conv(**kw):
    a = B.Conv(dtype=B.WM_BF16, B=2, T_max=5, channels=16, width=4, silu=1, rows=8, off=FAKE, x=FAKE, ld_x=16, weight=FAKE)
    for n, x in kw.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=-1), B.WM_ERR_INVALID_ARGUMENT), (dict(B=-1), B.WM_ERR_INVALID_ARGUMENT),
    (dict(T_max=-1), B.WM_ERR_INVALID_ARGUMENT), (dict(rows=-1), B.WM_ERR_INVALID_ARGUMENT),
    (dict(rows=1 << 31), B.WM_ERR_INVALID_ARGUMENT), (dict(channels=0), B.WM_ERR_INVALID_ARGUMENT),
    (dict(width=1), B.WM_ERR_UNSUPPORTED), (dict(width=5), B.WM_ERR_UNSUPPORTED),
    (dict(off=None), B.WM_ERR_INVALID_ARGUMENT), (dict(x=None), B.WM_ERR_INVALID_ARGUMENT),
    (dict(ld_x=15), B.WM_ERR_INVALID_ARGUMENT), (dict(weight=None), B.WM_ERR_INVALID_ARGUMENT),
])
def test_conv_refuses(kw, want):
    lib = wm.load_library()
    assert lib.wm_causal_conv(conv(**kw), FAKE, 16, None, None) == want
    assert lib.wm_causal_conv_grad(conv(**kw), FAKE, 16, None, FAKE, 16, FAKE, None, None, FAKE, 1 << 30, None) == want
    assert lib.wm_causal_conv_workspace_bytes(conv(**kw)) == 0


def test_conv_refuses_outputs_and_workspace():
    lib = wm.load_library()
    bad = B.WM_ERR_INVALID_ARGUMENT
    assert lib.wm_causal_conv(conv(), None, 16, None, None) == bad
    assert lib.wm_causal_conv(conv(), FAKE, 8, None, None) == bad
    n = lib.wm_causal_conv_workspace_bytes(conv())
    assert lib.wm_causal_conv_grad(conv(), FAKE, 16, None, FAKE, 16, None, None, None, FAKE, n, None) == bad
    assert lib.wm_causal_conv_grad(conv(), FAKE, 16, None, FAKE, 16, FAKE, None, None, FAKE, n - 1, None) == bad
    assert lib.wm_causal_conv_grad(conv(), FAKE, 16, None, FAKE, 16, FAKE, None, None, None, n, None) == bad


def scan(**kw):
    a = B.ScanArgs(dtype=B.WM_BF16, B=2, T_max=5, channels=16, states=16, rows=8, off=FAKE, u=FAKE, delta=FAKE, Bm=FAKE, Cm=FAKE,
                   ld_u=16, ld_delta=16, ld_B=16, ld_C=16, A=FAKE)
    for n, x in kw.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), B.WM_ERR_INVALID_ARGUMENT), (dict(states=12), B.WM_ERR_UNSUPPORTED), (dict(states=64), B.WM_ERR_UNSUPPORTED),
    (dict(A=None), B.WM_ERR_INVALID_ARGUMENT), (dict(u=None), B.WM_ERR_INVALID_ARGUMENT),
    (dict(delta=None), B.WM_ERR_INVALID_ARGUMENT), (dict(Bm=None), B.WM_ERR_INVALID_ARGUMENT),
    (dict(Cm=FAKE + 2), B.WM_ERR_INVALID_ARGUMENT), (dict(ld_B=20), B.WM_ERR_INVALID_ARGUMENT),
    (dict(ld_C=8), B.WM_ERR_INVALID_ARGUMENT), (dict(z=FAKE, ld_z=4), B.WM_ERR_INVALID_ARGUMENT),
    (dict(h0=FAKE + 4), B.WM_ERR_INVALID_ARGUMENT), (dict(channels=(1 << 20) + 1), B.WM_ERR_INVALID_ARGUMENT),
    (dict(B=-2), B.WM_ERR_INVALID_ARGUMENT), (dict(off=None), B.WM_ERR_INVALID_ARGUMENT),
])
def test_scan_refuses(kw, want):
    lib = wm.load_library()
    g = B.ScanGrads(du=FAKE, ddelta=FAKE, dz=FAKE, dB=FAKE, dC=FAKE, ld_du=16, ld_ddelta=16, ld_dz=16, ld_dB=16, ld_dC=16, dA=FAKE)
    assert lib.wm_scan(scan(**kw), FAKE, 16, None, None, FAKE, 1 << 30, None) == want
    assert lib.wm_scan_grad(scan(**kw), FAKE, FAKE, 16, None, g, FAKE, 1 << 30, None) == want
    assert lib.wm_scan_workspace_bytes(scan(**kw), 0) == 0 and lib.wm_scan_checkpoint_bytes(scan(**kw)) == 0


def test_scan_refuses_outputs_and_workspace():
    lib = wm.load_library()
    bad = B.WM_ERR_INVALID_ARGUMENT
    assert lib.wm_scan(scan(), None, 16, None, None, None, 0, None) == bad
    assert lib.wm_scan(scan(), FAKE, 16, FAKE + 4, None, None, 0, None) == bad
    n = lib.wm_scan_workspace_bytes(scan(), 1)
    full = dict(du=FAKE, ddelta=FAKE, dz=FAKE, dB=FAKE, dC=FAKE, ld_du=16, ld_ddelta=16, ld_dz=16, ld_dB=16, ld_dC=16, dA=FAKE)
    for missing in ("du", "ddelta", "dB", "dC", "dA"):
        g = B.ScanGrads(**{k: v for k, v in full.items() if k != missing})
        assert lib.wm_scan_grad(scan(), FAKE, FAKE, 16, None, g, FAKE, n, None) == bad
    g = B.ScanGrads(**full)
    assert lib.wm_scan_grad(scan(), None, FAKE, 16, None, g, FAKE, n, None) == bad
    assert lib.wm_scan_grad(scan(), FAKE, FAKE, 16, None, None, FAKE, n, None) == bad
    assert lib.wm_scan_grad(scan(), FAKE, FAKE, 16, None, g, FAKE, n - 1, None) == bad


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    q = torch.zeros(4, 2, 64)
    k = torch.zeros(9, 1, 64)
    with pytest.raises(ValueError, match="v must be"):
        wm.cross_attention(q, k, k.to(torch.bfloat16), [0, 4], [0, 9])         # types differ
    with pytest.raises(ValueError, match="must end at"):
        wm.cross_attention(q, k, k, [0, 5], [0, 9])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        wm.cross_attention(q.half(), k.half(), k.half(), [0, 4], [0, 9])
    with pytest.raises(ValueError, match="kv_mask"):
        wm.cross_attention(q, k, k, [0, 4], [0, 9], kv_mask=torch.ones(8, dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU"):
        wm.cross_attention(q, k, k, [0, 4], [0, 9])                            # host memory
    off = torch.tensor([0, 4], dtype=torch.int32)
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="off must be"):
        wm.causal_conv(x, off.long(), torch.zeros(8, 4), T_max=4)
    with pytest.raises(ValueError, match="weight"):
        wm.causal_conv(x, off, torch.zeros(7, 4), T_max=4)
    with pytest.raises(ValueError, match="state"):
        wm.causal_conv(x, off, torch.zeros(8, 4), T_max=4, state=torch.zeros(1, 2, 8))
    with pytest.raises(ValueError, match="GPU"):
        wm.causal_conv(x, off, torch.zeros(8, 4), T_max=4)
    A, b = torch.zeros(8, 16), torch.zeros(4, 16)
    with pytest.raises(ValueError, match="delta must be"):
        wm.selective_scan(x, x[:3], A, b, b, off, T_max=4)
    with pytest.raises(ValueError, match="Bm must be"):
        wm.selective_scan(x, x, A, b[:, :8], b, off, T_max=4)
    with pytest.raises(ValueError, match="h0 must be"):
        wm.selective_scan(x, x, A, b, b, off, T_max=4, h0=torch.zeros(2, 8, 16))
    with pytest.raises(ValueError, match="row stride"):
        wm.selective_scan(torch.zeros(8, 4).t(), x, A, b, b, off, T_max=4)
    with pytest.raises(ValueError, match="GPU"):
        wm.selective_scan(x, x, A, b, b, off, T_max=4)
