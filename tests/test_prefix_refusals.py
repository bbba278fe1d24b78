"""What the operators over a shared prefix refuse, before anything reaches a device (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import paper_2606_09312_amd as wm
from paper_2606_09312_amd import binding as B

torch = pytest.importorskip("torch")

FAKE = 4096            # an aligned address that is never read
INVALID, UNSUPPORTED = B.WM_ERR_INVALID_ARGUMENT, B.WM_ERR_UNSUPPORTED


def put(a, kw):
    for n, x in kw.items():
        setattr(a.cache if n.startswith("c_") else a, n.removeprefix("c_"), x)
    return a


def host(a):
    a = np.asarray(a, np.int32)
    return a, a.ctypes.data


# ---- rotation ----------------------------------------------------------------------
def rotation(**kw):
    return put(B.Rotation(dtype=B.WM_BF16, B=2, T_max=5, heads=4, head_dim=64, rot=64, rows=8, off=FAKE, freq=FAKE, x=FAKE, ld_x=256), kw)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), INVALID), (dict(heads=0), INVALID), (dict(heads=1025), INVALID), (dict(head_dim=60), UNSUPPORTED),
    (dict(head_dim=520, ld_x=4096), UNSUPPORTED), (dict(rot=0), INVALID), (dict(rot=3), INVALID), (dict(rot=66), INVALID),
    (dict(freq=None), INVALID), (dict(off=None), INVALID), (dict(B=0), INVALID), (dict(T_max=0), INVALID), (dict(B=-1), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID), (dict(rows=(1 << 26) - 3), UNSUPPORTED), (dict(x=None), INVALID),
    (dict(x=FAKE + 8), INVALID),
    (dict(ld_x=248), INVALID), (dict(ld_x=260), INVALID), (dict(ld_x=1 << 23), INVALID),
])
def test_rotate_refuses(kw, want):
    lib = wm.load_library()
    assert lib.wm_rotate(rotation(**kw), FAKE * 2, 256, None) == want
    assert lib.wm_last_error().decode() != ""


def test_rotate_refuses_outputs():
    lib = wm.load_library()
    assert lib.wm_rotate(None, FAKE, 256, None) == INVALID
    for y, ld in ((None, 256), (FAKE * 2 + 4, 256), (FAKE * 2, 128), (FAKE, 512)):      # (in place with another stride)
        assert lib.wm_rotate(rotation(), y, ld, None) == INVALID
    assert lib.wm_rotate(rotation(rows=0, x=None, B=0, off=None), None, 0, None) == B.WM_OK


# ---- cache -------------------------------------------------------------------------
def cache():
    return B.Cache(dtype=B.WM_BF16, kv_heads=2, head_dim=64, page=16, n_pages=9, B=2, max_pages=3, k=FAKE, v=FAKE, pages=FAKE, lens=FAKE)


def append(**kw):
    return put(B.Append(cache=cache(), T_max=5, heads=4, rot=64, rows=8, off=FAKE, freq=FAKE, k=FAKE, v=FAKE, q=FAKE, ld_k=128, ld_v=128,
                        ld_q=256), kw)


def cached(seg_off=(0, 2), **kw):
    keep, p = host((0, 2) if seg_off is None else seg_off)
    a = B.Cached(cache=cache(), T_max=5, len_max=48, heads=4, S=len(keep) - 1, prefix_max_pages=4, prefix_max=64, rows=8, off=FAKE,
                 seg_off=None if seg_off is None else p, prefix_pages=FAKE, prefix_lens=FAKE, q=FAKE, ld_q=256, scale=0.125)
    a.keep = keep
    return put(a, kw)


CACHE = [
    (dict(c_dtype=3), INVALID), (dict(c_kv_heads=0), INVALID), (dict(c_head_dim=96), UNSUPPORTED), (dict(c_page=8), UNSUPPORTED),
    (dict(c_page=48), UNSUPPORTED), (dict(c_page=512), UNSUPPORTED), (dict(c_n_pages=-1), INVALID), (dict(c_B=-1), INVALID),
    (dict(c_max_pages=-1), INVALID), (dict(c_max_pages=1 << 28), UNSUPPORTED), (dict(c_k=None), INVALID), (dict(c_v=FAKE + 8), INVALID),
    (dict(c_pages=None), INVALID), (dict(c_lens=None), INVALID), (dict(off=None), INVALID), (dict(rows=-1), INVALID),
    (dict(rows=1 << 31), INVALID), (dict(T_max=0), INVALID), (dict(T_max=-1), INVALID), (dict(c_B=0), INVALID), (dict(q=FAKE + 2), INVALID),
    (dict(ld_q=192), INVALID), (dict(ld_q=260), INVALID),
]


@pytest.mark.parametrize("kw,want", CACHE + [
    (dict(rot=0), INVALID), (dict(rot=65), INVALID), (dict(rot=128), INVALID), (dict(heads=0), INVALID), (dict(q=None), INVALID),
    (dict(rows=1 << 27), UNSUPPORTED), (dict(heads=-1), INVALID), (dict(k=None), INVALID),
    (dict(v=FAKE + 4), INVALID), (dict(ld_k=120), INVALID), (dict(ld_v=132), INVALID),
])
def test_append_refuses(kw, want):
    lib = wm.load_library()
    assert lib.wm_cache_append(append(**kw), FAKE, 256, None) == want
    assert lib.wm_last_error().decode() != ""


def test_append_refuses_outputs():
    lib = wm.load_library()
    assert lib.wm_cache_append(None, FAKE, 256, None) == INVALID
    for q_out, ld in ((None, 256), (FAKE * 3 + 8, 256), (FAKE * 3, 248), (FAKE, 512)):
        assert lib.wm_cache_append(append(), q_out, ld, None) == INVALID
    assert lib.wm_cache_append(append(rows=0), FAKE, 256, None) == B.WM_OK


@pytest.mark.parametrize("kw,want", CACHE + [
    (dict(heads=3), INVALID), (dict(heads=2050), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=3e38), INVALID), (dict(len_max=49), INVALID), (dict(len_max=-1), INVALID), (dict(prefix_max=65), INVALID),
    (dict(prefix_max=-1), INVALID), (dict(prefix_lens=None), INVALID), (dict(prefix_pages=None), INVALID), (dict(seg_off=None), INVALID),
    (dict(S=513), INVALID), (dict(S=-1), INVALID), (dict(q=None), INVALID), (dict(T_max=1 << 30, rows=1 << 30), UNSUPPORTED),
])
def test_cached_refuses(kw, want):
    lib = wm.load_library()
    a = cached(**kw)
    assert lib.wm_cached_attention(a, FAKE, 256, None, FAKE, 1 << 40, None) == want
    assert lib.wm_last_error().decode() != ""
    assert lib.wm_cached_attention_workspace_bytes(a) == 0


@pytest.mark.parametrize("seg_off", [(1, 2), (0, 1), (0, 3), (0, 2, 1, 2), (0, 3, 2)])
def test_cached_refuses_bad_programs(seg_off):
    assert wm.load_library().wm_cached_attention(cached(seg_off), FAKE, 256, None, FAKE, 1 << 40, None) == INVALID


def test_cached_refuses_outputs_and_workspace():
    lib = wm.load_library()
    a = cached()
    n = lib.wm_cached_attention_workspace_bytes(a)
    assert n > 256
    for args in ((None, 256, None, FAKE, n), (FAKE, 248, None, FAKE, n), (FAKE, 256, None, None, n), (FAKE, 256, None, FAKE, n - 1),
                 (FAKE, 256, None, FAKE + 64, n)):
        assert lib.wm_cached_attention(a, *args, None) == INVALID
    assert lib.wm_cached_attention(None, FAKE, 256, None, FAKE, n, None) == INVALID
    assert lib.wm_cached_attention(cached(rows=0, q=None), None, 0, None, None, 0, None) == B.WM_OK


# ---- prefix attention --------------------------------------------------------------
def prefix(q_off=(0, 8), p_off=(0, 9), shared=None, **kw):
    (qa, qp), (pa, pp) = host(q_off), host(p_off)
    s = dict(dtype=B.WM_BF16, heads=4, kv_heads=2, head_dim=64, S=len(pa) - 1, q_off=qp, k_off=pp, q=FAKE, k=FAKE, v=FAKE, ld_q=256, ld_k=128,
             ld_v=128, scale=0.125)
    s.update(shared or {})
    a = B.Prefix(shared=B.Attention(**s), k=FAKE, v=FAKE, ld_k=128, ld_v=128, B=2, T_max=5, off=FAKE)
    for n, x in kw.items():
        setattr(a, n, x)
    a.keep = (qa, pa)
    return a


def grads(**kw):
    g = B.PrefixGrads(dq=FAKE, dk=FAKE, dv=FAKE, dpk=FAKE, dpv=FAKE, ld_dq=256, ld_dk=128, ld_dv=128, ld_dpk=128, ld_dpv=128)
    for n, x in kw.items():
        setattr(g, n, x)
    return g


@pytest.mark.parametrize("kw,want", [
    (dict(shared=dict(dtype=7)), INVALID), (dict(shared=dict(heads=3)), INVALID), (dict(shared=dict(head_dim=48)), UNSUPPORTED),
    (dict(shared=dict(scale=-1.0)), INVALID), (dict(shared=dict(q=None)), INVALID), (dict(shared=dict(ld_k=120)), INVALID),
    (dict(shared=dict(k_off=None)), INVALID), (dict(k=None), INVALID), (dict(v=FAKE + 8), INVALID), (dict(ld_k=136 + 4), INVALID),
    (dict(ld_v=64), INVALID), (dict(B=0), INVALID), (dict(B=-1), INVALID), (dict(T_max=0), INVALID), (dict(off=None), INVALID),
    (dict(q_off=(0, 9, 8), p_off=(0, 3, 9)), INVALID), (dict(q_off=(1, 8)), INVALID),
])
def test_prefix_refuses(kw, want):
    lib = wm.load_library()
    a = prefix(**kw)
    assert lib.wm_prefix_attention(a, FAKE, 256, None, FAKE, 1 << 40, None) == want
    assert lib.wm_last_error().decode() != ""
    assert lib.wm_prefix_attention_grad(a, FAKE, 256, FAKE, FAKE, 256, grads(), FAKE, 1 << 40, None) == want
    assert lib.wm_prefix_attention_workspace_bytes(a, 0) == 0 and lib.wm_prefix_attention_workspace_bytes(a, 1) == 0


def test_prefix_refuses_outputs_and_workspace():
    lib = wm.load_library()
    assert lib.wm_prefix_attention_workspace_bytes(prefix(), 0) == 256              # a loop in one part needs none
    a = prefix(p_off=(0, 60000))
    n, m = (lib.wm_prefix_attention_workspace_bytes(a, g) for g in (0, 1))
    assert n > 256 and m > 256
    for args in ((None, 256, None, FAKE, n), (FAKE, 200, None, FAKE, n), (FAKE, 256, None, None, n), (FAKE, 256, None, FAKE, n - 1)):
        assert lib.wm_prefix_attention(a, *args, None) == INVALID
    good = dict(o=FAKE, ld_o=256, lse=FAKE, d_o=FAKE, ld_do=256, g=grads(), ws=FAKE, n=m)
    for kw in (dict(o=None), dict(ld_o=8), dict(lse=None), dict(d_o=FAKE + 8), dict(g=None), dict(g=grads(dq=None)), dict(g=grads(ld_dpv=64)),
               dict(g=grads(dpk=None)), dict(g=grads(dk=FAKE + 4)), dict(ws=None), dict(n=m - 1), dict(ws=FAKE + 128)):
        assert lib.wm_prefix_attention_grad(a, *{**good, **kw}.values(), None) == INVALID, kw
    assert lib.wm_prefix_attention(None, FAKE, 256, None, FAKE, n, None) == INVALID


# ---- the binding -------------------------------------------------------------------
@pytest.fixture
def gpu(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_binding_refuses_rotations(gpu):
    x, off, f = torch.zeros(4, 2, 64), i32(0, 4), torch.zeros(32)
    for args, kw in (((x[0], off, f), {}), ((x.double(), off, f), {}), ((x, off.long(), f), {}), ((x, off, f.double()), {}), ((x, off, f[None]), {}),
                     ((x, off, f), dict(first=torch.zeros(1))), ((x, off, f), dict(first=i32(0, 0))), ((x, off, f), dict(y=x[:2])),
                     ((x, off, f), dict(status=i32(0))), ((x.transpose(1, 2), off, f), {})):
        with pytest.raises(ValueError):
            wm.rotate(*args, T_max=4, **kw)


def test_binding_refuses_caches(gpu):
    kc, pages, lens, off = torch.zeros(3, 2, 16, 64), i32(0, 1).view(1, 2), i32(4), i32(0, 4)
    k, q = torch.zeros(4, 2, 64), torch.zeros(4, 4, 64)
    good = dict(k=k, v=k, k_cache=kc, v_cache=kc, pages=pages, lens=lens, off=off)
    for kw in (dict(k=k[0]), dict(v=k[:3]), dict(k=k.bfloat16()), dict(v_cache=kc[:2]), dict(k_cache=kc.transpose(0, 1), v_cache=kc.transpose(0, 1)),
               dict(k_cache=kc[0]), dict(pages=pages.long()), dict(pages=pages[0]), dict(lens=i32(4, 4)), dict(off=i32(0, 2, 4)),
               dict(freq=torch.zeros(2, 2)), dict(q=q[..., :32]), dict(q=q[:2]), dict(q_out=q), dict(first=i32(1, 2))):
        with pytest.raises(ValueError):
            wm.cache_append(**{**good, **kw}, T_max=4)
    good = dict(q=q, k_cache=kc, v_cache=kc, pages=pages, lens=lens, off=off)
    more = dict(seg_off=[0, 1], prefix_pages=pages, prefix_lens=lens)
    for kw in (dict(q=q[0]), dict(q=q[..., :32]), dict(q=q.bfloat16()), dict(off=i32(0)), dict(o=q[:2]), dict(lse=torch.zeros(4, 2)),
               dict(prefix_pages=pages), dict(prefix_lens=lens), dict(seg_off=[0, 1]), {**more, "seg_off": [0, 2]}, {**more, "seg_off": [1]},
               {**more, "prefix_lens": i32(1, 2)}, {**more, "prefix_pages": pages[0]}, {**more, "prefix_pages": pages.long()}):
        with pytest.raises(ValueError):
            wm.cached_attention(**{**good, **kw}, T_max=4)


def test_binding_refuses_prefixes(gpu):
    q, k, pk, off = torch.zeros(4, 4, 64), torch.zeros(4, 2, 64), torch.zeros(9, 2, 64), i32(0, 4)
    good = dict(q=q, k=k, v=k, pk=pk, pv=pk, off=off, q_off=[0, 4], p_off=[0, 9])
    for kw in (dict(k=k[:3]), dict(v=k[0]), dict(k=k.bfloat16()), dict(pv=pk[:8]), dict(pk=pk[:, :1]), dict(off=off.long()), dict(q_off=[0, 3]),
               dict(p_off=[0, 8]), dict(p_off=[0, 4, 9]), dict(kv_mask=torch.ones(4, dtype=torch.uint8)), dict(o=q[:1]), dict(lse=torch.zeros(4, 2))):
        with pytest.raises(ValueError):
            wm.prefix_attention(**{**good, **kw}, T_max=4)
    lse = torch.zeros(4, 4)
    for kw in (dict(do=q[:2]), dict(o=q.double()), dict(lse=lse[:2]), dict(v=k[0])):
        with pytest.raises(ValueError):
            wm.prefix_attention_grad(**{**dict(good, do=q, o=q, lse=lse), **kw}, T_max=4)
