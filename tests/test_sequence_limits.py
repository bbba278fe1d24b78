"""Sizes past what a launch can hold and scales past float32 are refused before anything is enqueued (no GPU needed)."""
import ctypes

import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B
from test_sequence_refusals import FAKE, attention, conv, scan

MANY = 2 ** 26            # wavefronts: 2^32 threads, one more than a launch may have


@pytest.mark.parametrize("kw", [
    dict(B=MANY // 64, T_max=64 * 16, channels=512, ld_x=512),                 # eight channels a lane, 64 lanes a run
    dict(B=MANY // 16, T_max=16, channels=1003, ld_x=1003),                    # one channel a lane
    dict(dtype=B.WM_FP32, B=MANY // 64, T_max=128 * 16, channels=128, ld_x=128),   # two runs a wavefront
])
def test_conv(kw):
    lib = wm.load_library()
    a = conv(rows=1, **kw)
    assert lib.wm_causal_conv(a, FAKE, kw["ld_x"], None, None) == B.WM_ERR_UNSUPPORTED
    assert "too large" in lib.wm_last_error().decode()


def test_scan():
    lib = wm.load_library()
    for T in (1, 64):
        a = scan(B=MANY, T_max=T, rows=1)
        assert lib.wm_scan(a, FAKE, 16, None, None, FAKE, 1 << 40, None) == B.WM_ERR_UNSUPPORTED
        assert "too large" in lib.wm_last_error().decode()
        assert lib.wm_scan_workspace_bytes(a, 0) == 0
        assert lib.wm_scan_workspace_bytes(scan(B=MANY - 4, T_max=T, rows=1), 0) > 0
    g = B.ScanGrads(du=FAKE, ddelta=FAKE, dz=FAKE, dB=FAKE, dC=FAKE, ld_du=16, ld_ddelta=16, ld_dz=16, ld_dB=16, ld_dC=16, dA=FAKE)
    a = scan(rows=2 ** 27)                               # 2^32 values of dB and dC
    assert lib.wm_scan_grad(a, FAKE, FAKE, 16, None, g, FAKE, 1 << 40, None) == B.WM_ERR_UNSUPPORTED
    assert lib.wm_scan_workspace_bytes(a, 1) == 0 and lib.wm_scan_workspace_bytes(a, 0) > 0
    assert lib.wm_scan_workspace_bytes(scan(rows=2 ** 27 - 8), 1) > 0


def test_attention_scale():
    """scale log2(e), which the kernels work with, has to be finite too."""
    lib = wm.load_library()
    for scale in (3e38, 2.4e38):
        a = attention(scale=scale)
        assert lib.wm_cross_attention(a, FAKE, 256, None, ctypes.c_void_p(FAKE), 1 << 30, None) == B.WM_ERR_INVALID_ARGUMENT
        assert lib.wm_cross_attention_workspace_bytes(a, 1) == 0
    assert lib.wm_cross_attention_workspace_bytes(attention(scale=2.3e38), 1) > 0
