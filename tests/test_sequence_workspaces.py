"""Workspaces of the sequence operators' smallest calls: the answer of the size queries says whether NULL will do
(256) or not (more), and the binding goes by it (no GPU needed: every call here is refused for its NULL)."""
import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B
from test_sequence_refusals import FAKE, attention, conv, scan

BAD = B.WM_ERR_INVALID_ARGUMENT


def allocated(n):
    ws, size = B._workspace(n, None, "cpu")
    return ws is not None and ws.numel() == size == n


@pytest.mark.parametrize("rows,heads,keys", [(1, 12, 77), (2, 4, 9), (8, 4, 60), (1, 32, 100), (1, 1, 1), (3, 8, 0)])
def test_attention_gradient(rows, heads, keys):
    a = attention((0, rows), (0, keys), heads=heads, kv_heads=heads, ld_q=heads * 64, ld_k=heads * 64, ld_v=heads * 64)
    lib, ld = wm.load_library(), heads * 64
    n = lib.wm_cross_attention_workspace_bytes(a, 1)
    assert lib.wm_cross_attention_grad(a, FAKE, ld, FAKE, FAKE, ld, FAKE, ld, FAKE, ld, FAKE, ld, None, 0, None) == BAD
    assert n > 256 and allocated(n)
    assert lib.wm_cross_attention_grad(a, FAKE, ld, FAKE, FAKE, ld, FAKE, ld, FAKE, ld, FAKE, ld, FAKE, n - 1, None) == BAD


@pytest.mark.parametrize("channels,width,seqs,rows", [(16, 3, 1, 16), (21, 2, 1, 16), (8, 3, 2, 16), (1, 2, 1, 1), (4, 4, 0, 0)])
def test_conv_gradient(channels, width, seqs, rows):
    a = conv(channels=channels, width=width, B=seqs, rows=rows, T_max=rows, ld_x=channels)
    lib = wm.load_library()
    n = lib.wm_causal_conv_workspace_bytes(a)
    assert lib.wm_causal_conv_grad(a, FAKE, channels, None, FAKE, channels, FAKE, None, None, None, 0, None) == BAD
    assert n > 256 and allocated(n)
    assert lib.wm_causal_conv_grad(a, FAKE, channels, None, FAKE, channels, FAKE, None, None, FAKE, n - 1, None) == BAD


@pytest.mark.parametrize("channels,states,seqs,rows", [(2, 8, 1, 1), (1, 8, 0, 0), (6, 8, 3, 0), (3, 16, 2, 0), (1, 32, 1, 1)])
def test_scan_gradient(channels, states, seqs, rows):
    a = scan(channels=channels, states=states, B=seqs, rows=rows, T_max=rows, ld_u=channels, ld_delta=channels, ld_B=states, ld_C=states)
    lib = wm.load_library()
    g = B.ScanGrads(du=FAKE, ddelta=FAKE, dz=FAKE, dB=FAKE, dC=FAKE, ld_du=channels, ld_ddelta=channels, ld_dz=channels, ld_dB=states,
                    ld_dC=states, dA=FAKE)
    n = lib.wm_scan_workspace_bytes(a, 1)
    assert lib.wm_scan_grad(a, FAKE, FAKE, channels, None, g, None, 0, None) == BAD
    assert n > 256 and allocated(n)
    assert lib.wm_scan_grad(a, FAKE, FAKE, channels, None, g, FAKE, n - 1, None) == BAD


def test_none_needed():
    """Forward calls that are not split: 256, and the binding allocates nothing."""
    lib = wm.load_library()
    assert lib.wm_cross_attention_workspace_bytes(attention(), 0) == 256 == lib.wm_scan_workspace_bytes(scan(), 0)
    assert B._workspace(256, None, "cpu") == (None, 0)


def test_rows_without_a_sequence_are_refused():
    lib = wm.load_library()
    assert lib.wm_causal_conv_workspace_bytes(conv(B=0, rows=8)) == 0 == lib.wm_scan_workspace_bytes(scan(B=0, rows=8), 1)
    assert lib.wm_scan(scan(B=0, rows=8), FAKE, 16, None, None, None, 0, None) == BAD
    assert lib.wm_causal_conv(conv(B=0, rows=8), FAKE, 16, None, None) == BAD
    assert lib.wm_causal_conv_workspace_bytes(conv(B=0, rows=0)) > 0 and lib.wm_scan_workspace_bytes(scan(B=0, rows=0), 1) > 0
