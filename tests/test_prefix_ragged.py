"""Calls of cached attention whose sequences differ widely are taken by the work that they have, not by that of the longest for every
one (no GPU needed)."""
import numpy as np
import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B

FAKE = 4096            # an aligned address that is never read


def cached(seqs, rows, T_max, programs=1):
    seg = np.linspace(0, seqs, programs + 1).astype(np.int32)
    c = B.Cache(dtype=B.WM_BF16, kv_heads=8, head_dim=64, page=16, n_pages=9, B=seqs, max_pages=3, k=FAKE, v=FAKE, pages=FAKE, lens=FAKE)
    a = B.Cached(cache=c, T_max=T_max, len_max=48, heads=32, S=programs, seg_off=seg.ctypes.data, prefix_pages=FAKE, prefix_lens=FAKE,
                 prefix_max_pages=4, prefix_max=64, rows=rows, off=FAKE, q=FAKE, ld_q=2048, scale=0.125)
    a.keep = seg
    return a


@pytest.mark.parametrize("programs", [1, 3, 512])
@pytest.mark.parametrize("seqs,T_max", [(20000, 4096), (100000, 1 << 20), (400000, 3)])
def test_one_long_chunk_among_many_steps(seqs, T_max, programs):
    lib = wm.load_library()
    assert lib.wm_cached_attention_workspace_bytes(cached(seqs, seqs + min(T_max, 4096) - 1, T_max, programs)) > 0, lib.wm_last_error()


def test_rows_that_are_too_many_are_refused():
    lib = wm.load_library()
    assert lib.wm_cached_attention_workspace_bytes(cached(4, 1 << 25, 1 << 24)) == 0
    assert b"too many" in lib.wm_last_error()
    assert lib.wm_cached_attention_workspace_bytes(cached(1 << 20, 1 << 20, 1)) == 0
