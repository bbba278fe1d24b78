"""ctypes binding of libwm.so (the C ABI in include/wm.h).

Argument marshalling only: every step of the evaluator runs in the library's
HIP kernels.  Device buffers are torch CUDA (HIP) tensors; the stream is
torch's current stream unless one is given.  A missing library raises.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libwm.so")

WM_OK, WM_ERR_INVALID_ARGUMENT, WM_ERR_UNSUPPORTED = 0, 1, 2
WM_ERR_OUT_OF_MEMORY, WM_ERR_DEVICE, WM_ERR_INPUT_RANGE = 3, 4, 5
WM_FP32, WM_BF16 = 0, 1
WM_NORM_NONE, WM_NORM_L2 = 0, 1
PRECISIONS = {"fp32": WM_FP32, "bf16": WM_BF16}
NORMS = {"none": WM_NORM_NONE, "l2": WM_NORM_L2}
KERNELS = {"rollout": 0, "score": 1, "topk": 2, "bucket": 3, "phi": 4, "encode": 5,
           "phi_struct": 6, "trees": 7, "loss_fwd": 8, "loss_steps": 9, "loss_bwd": 10,
           "loss_grads": 11, "text_gemm": 12, "text_attn": 13, "text_other": 14,
           "cross_attention": 15, "causal_conv": 16, "scan": 17, "rotate": 18, "cache_append": 19,
           "cached_attention": 20, "prefix_attention": 21}

# Exported symbols (kept in step with include/wm.h).
SYMBOLS = (
    "wm_model_create", "wm_model_destroy", "wm_workspace_bytes", "wm_encode_init",
    "wm_rollout", "wm_score", "wm_topk", "wm_evaluate", "wm_device_status",
    "wm_last_error", "wm_timing_enable", "wm_timing_read", "wm_forest_create",
    "wm_forest_destroy", "wm_phi_struct", "wm_score_trees", "wm_evaluate_trees",
    "wm_loss_workspace_bytes", "wm_rollout_loss", "wm_text_model_create", "wm_text_model_destroy",
    "wm_text_chunks", "wm_text_workspace_bytes", "wm_encode_text", "wm_evaluate_noalloc",
    "wm_cross_attention_workspace_bytes", "wm_cross_attention", "wm_cross_attention_grad",
    "wm_causal_conv", "wm_causal_conv_workspace_bytes", "wm_causal_conv_grad",
    "wm_scan_workspace_bytes", "wm_scan_checkpoint_bytes", "wm_scan", "wm_scan_grad",
    "wm_rotate", "wm_cache_append", "wm_cached_attention_workspace_bytes", "wm_cached_attention",
    "wm_prefix_attention_workspace_bytes", "wm_prefix_attention", "wm_prefix_attention_grad",
)


class WMError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"wm status {status}: {msg}")
        self.status = status
        self.msg = msg


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "d", "embed_dim", "n_kinds", "n_params", "trans_hidden", "cost_hidden", "hw_dim",
        "feat_dim", "enc_hidden", "precision", "norm")]


_FP = ctypes.POINTER(ctypes.c_float)


class Weights(ctypes.Structure):
    _fields_ = [
        ("type_emb", _FP), ("param_w", _FP), ("param_b", _FP),
        ("w1", _FP), ("b1", _FP), ("w2", _FP), ("b2", _FP),
        ("wc1", _FP), ("bc1", _FP), ("wc2", _FP), ("bc2", ctypes.c_float),
        ("we1", _FP), ("be1", _FP), ("we2", _FP), ("be2", _FP),
        ("wh", _FP),
    ]


class Grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "w1", "b1", "w2", "b2", "type_emb", "param_w", "param_b", "z0", "wh")]


GRAD_KEYS = ("w1", "b1", "w2", "b2", "type_emb", "param_w", "param_b")


class TextDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "vocab", "hidden", "heads", "ffn", "layers", "window", "stride", "d", "precision")]


TEXT_WEIGHT_KEYS = ("tok_emb", "pos_emb", "ln0_g", "ln0_b", "wqkv", "bqkv", "wo", "bo", "ln1_g",
                    "ln1_b", "w1", "b1", "w2", "b2", "ln2_g", "ln2_b", "wp", "bp")


class TextWeights(ctypes.Structure):
    _fields_ = [(n, _FP) for n in TEXT_WEIGHT_KEYS]

class Attention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "heads", "kv_heads", "head_dim", "S")]
                + [(n, ctypes.c_void_p) for n in ("q_off", "k_off", "q", "k", "v")]
                + [(n, ctypes.c_int64) for n in ("ld_q", "ld_k", "ld_v")]
                + [("kv_mask", ctypes.c_void_p), ("scale", ctypes.c_float)])


class Conv(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "B", "T_max", "channels", "width", "silu")]
                + [("rows", ctypes.c_int64), ("off", ctypes.c_void_p), ("x", ctypes.c_void_p), ("ld_x", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("weight", "bias", "state", "status")])


class ScanArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "B", "T_max", "channels", "states")]
                + [("rows", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("off", "u", "delta", "z", "Bm", "Cm")]
                + [(n, ctypes.c_int64) for n in ("ld_u", "ld_delta", "ld_z", "ld_B", "ld_C")]
                + [(n, ctypes.c_void_p) for n in ("A", "D", "delta_bias", "h0", "status")])


class ScanGrads(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("du", "ddelta", "dz", "dB", "dC")]
                + [(n, ctypes.c_int64) for n in ("ld_du", "ld_ddelta", "ld_dz", "ld_dB", "ld_dC")]
                + [(n, ctypes.c_void_p) for n in ("dA", "dD", "ddelta_bias", "dh0")])


class Rotation(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "B", "T_max", "heads", "head_dim", "rot", "interleaved", "inverse")]
                + [("rows", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("off", "first", "freq", "x")]
                + [("ld_x", ctypes.c_int64), ("status", ctypes.c_void_p)])


class Cache(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "kv_heads", "head_dim", "page", "n_pages", "B", "max_pages")]
                + [(n, ctypes.c_void_p) for n in ("k", "v", "pages", "lens")])


class Append(ctypes.Structure):
    _fields_ = ([("cache", Cache)] + [(n, ctypes.c_int32) for n in ("T_max", "heads", "rot", "interleaved")]
                + [("rows", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("off", "first", "freq", "k", "v", "q")]
                + [(n, ctypes.c_int64) for n in ("ld_k", "ld_v", "ld_q")] + [("status", ctypes.c_void_p)])


class Cached(ctypes.Structure):
    _fields_ = ([("cache", Cache)] + [(n, ctypes.c_int32) for n in ("T_max", "len_max", "heads", "S", "prefix_max_pages", "prefix_max")]
                + [("rows", ctypes.c_int64)] + [(n, ctypes.c_void_p) for n in ("off", "seg_off", "prefix_pages", "prefix_lens", "q")]
                + [("ld_q", ctypes.c_int64), ("scale", ctypes.c_float), ("status", ctypes.c_void_p)])


class Prefix(ctypes.Structure):
    _fields_ = ([("shared", Attention)] + [(n, ctypes.c_void_p) for n in ("k", "v")] + [(n, ctypes.c_int64) for n in ("ld_k", "ld_v")]
                + [(n, ctypes.c_int32) for n in ("B", "T_max")] + [(n, ctypes.c_void_p) for n in ("off", "status")])


class PrefixGrads(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("dq", "dk", "dv", "dpk", "dpv")]
                + [(n, ctypes.c_int64) for n in ("ld_dq", "ld_dk", "ld_dv", "ld_dpk", "ld_dpv")])


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libwm.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2606_09312_amd.build.build()")
    # Load torch first so the library binds to the HIP runtime torch uses
    # (one runtime per process; device buffers and streams come from torch).
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.wm_model_create.argtypes = [ctypes.POINTER(Dims), ctypes.POINTER(Weights), ctypes.POINTER(vp)]
    lib.wm_model_create.restype = i32
    lib.wm_model_destroy.argtypes = [vp]
    lib.wm_model_destroy.restype = None
    lib.wm_workspace_bytes.argtypes = [vp, i32, i32, i32, i32]
    lib.wm_workspace_bytes.restype = sz
    lib.wm_encode_init.argtypes = [vp, vp, i32, vp, vp]
    lib.wm_encode_init.restype = i32
    lib.wm_rollout.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
    lib.wm_rollout.restype = i32
    lib.wm_score.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp]
    lib.wm_score.restype = i32
    lib.wm_topk.argtypes = [vp, i32, i32, vp, i32, i32, vp, vp, vp]
    lib.wm_topk.restype = i32
    lib.wm_evaluate.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, vp, i32, i32,
                                vp, vp, vp, vp, vp, sz, vp]
    lib.wm_evaluate.restype = i32
    lib.wm_evaluate_noalloc.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, vp, i32, i32,
                                        vp, vp, vp, vp, vp, vp, vp]
    lib.wm_evaluate_noalloc.restype = i32
    lib.wm_device_status.argtypes = [vp, sz, vp]
    lib.wm_device_status.restype = i32
    lib.wm_last_error.argtypes = []
    lib.wm_last_error.restype = ctypes.c_char_p
    lib.wm_timing_enable.argtypes = [i32]
    lib.wm_timing_enable.restype = i32
    lib.wm_timing_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.wm_timing_read.restype = i32
    lib.wm_forest_create.argtypes = [i32, i32, i32, vp, vp, vp, ctypes.c_float, ctypes.POINTER(vp)]
    lib.wm_forest_create.restype = i32
    lib.wm_forest_destroy.argtypes = [vp]
    lib.wm_forest_destroy.restype = None
    lib.wm_phi_struct.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp]
    lib.wm_phi_struct.restype = i32
    lib.wm_score_trees.argtypes = [vp, vp, i32, vp, i32, i32, vp, i32, i32, vp, vp]
    lib.wm_score_trees.restype = i32
    lib.wm_evaluate_trees.argtypes = [vp, vp, vp, i32, vp, i32, vp, vp, vp, i32, i32, vp, i32, i32,
                                      vp, vp, vp, vp, vp, sz, vp]
    lib.wm_evaluate_trees.restype = i32
    lib.wm_loss_workspace_bytes.argtypes = [vp, i32, i32]
    lib.wm_loss_workspace_bytes.restype = sz
    lib.wm_rollout_loss.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, i32,
                                    ctypes.c_float, ctypes.c_float, vp, vp, ctypes.POINTER(Grads),
                                    vp, sz, vp]
    lib.wm_rollout_loss.restype = i32
    lib.wm_text_model_create.argtypes = [ctypes.POINTER(TextDims), ctypes.POINTER(TextWeights),
                                         ctypes.POINTER(vp)]
    lib.wm_text_model_create.restype = i32
    lib.wm_text_model_destroy.argtypes = [vp]
    lib.wm_text_model_destroy.restype = None
    lib.wm_text_chunks.argtypes = [vp, vp, i32]
    lib.wm_text_chunks.restype = i32
    lib.wm_text_workspace_bytes.argtypes = [vp, i32]
    lib.wm_text_workspace_bytes.restype = sz
    lib.wm_encode_text.argtypes = [vp, vp, vp, i32, vp, vp, sz, vp]
    lib.wm_encode_text.restype = i32
    i64 = ctypes.c_int64
    at, cv, sc = ctypes.POINTER(Attention), ctypes.POINTER(Conv), ctypes.POINTER(ScanArgs)
    lib.wm_cross_attention_workspace_bytes.argtypes = [at, i32]
    lib.wm_cross_attention_workspace_bytes.restype = sz
    lib.wm_cross_attention.argtypes = [at, vp, i64, vp, vp, sz, vp]
    lib.wm_cross_attention.restype = i32
    lib.wm_cross_attention_grad.argtypes = [at, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, sz, vp]
    lib.wm_cross_attention_grad.restype = i32
    lib.wm_causal_conv.argtypes = [cv, vp, i64, vp, vp]
    lib.wm_causal_conv.restype = i32
    lib.wm_causal_conv_workspace_bytes.argtypes = [cv]
    lib.wm_causal_conv_workspace_bytes.restype = sz
    lib.wm_causal_conv_grad.argtypes = [cv, vp, i64, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    lib.wm_causal_conv_grad.restype = i32
    lib.wm_scan_workspace_bytes.argtypes = [sc, i32]
    lib.wm_scan_workspace_bytes.restype = sz
    lib.wm_scan_checkpoint_bytes.argtypes = [sc]
    lib.wm_scan_checkpoint_bytes.restype = sz
    lib.wm_scan.argtypes = [sc, vp, i64, vp, vp, vp, sz, vp]
    lib.wm_scan.restype = i32
    lib.wm_scan_grad.argtypes = [sc, vp, vp, i64, vp, ctypes.POINTER(ScanGrads), vp, sz, vp]
    lib.wm_scan_grad.restype = i32
    ro, ap, ca, pr = (ctypes.POINTER(c) for c in (Rotation, Append, Cached, Prefix))
    lib.wm_rotate.argtypes = [ro, vp, i64, vp]
    lib.wm_rotate.restype = i32
    lib.wm_cache_append.argtypes = [ap, vp, i64, vp]
    lib.wm_cache_append.restype = i32
    lib.wm_cached_attention_workspace_bytes.argtypes = [ca]
    lib.wm_cached_attention_workspace_bytes.restype = sz
    lib.wm_cached_attention.argtypes = [ca, vp, i64, vp, vp, sz, vp]
    lib.wm_cached_attention.restype = i32
    lib.wm_prefix_attention_workspace_bytes.argtypes = [pr, i32]
    lib.wm_prefix_attention_workspace_bytes.restype = sz
    lib.wm_prefix_attention.argtypes = [pr, vp, i64, vp, vp, sz, vp]
    lib.wm_prefix_attention.restype = i32
    lib.wm_prefix_attention_grad.argtypes = [pr, vp, i64, vp, vp, i64, ctypes.POINTER(PrefixGrads), vp, sz, vp]
    lib.wm_prefix_attention_grad.restype = i32
    _lib = lib
    return lib


def _check(status: int):
    if status != WM_OK:
        raise WMError(status, load_library().wm_last_error().decode())


def _ptr(t):
    """Device pointer of a torch tensor (or None)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the library must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _host_i32(a):
    a = np.ascontiguousarray(np.asarray(a), dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _on_stream(fn):
    """Gives fn, which allocates and launches on the current stream, the keyword `stream`.

    The call then runs with that stream current, so that what it allocates (workspaces that are
    dropped on return above all) belongs to the stream's pool and is reused in the stream's order only.
    Results are kept from that reuse while the caller's stream uses them, and the caller's tensors
    from their own pool's while `stream` does.
    """
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        import torch
        here = torch.cuda.current_stream(stream.device)
        given = [t for v in (*args, *kw.values()) for t in (v.values() if isinstance(v, dict) else (v,))
                 if isinstance(t, torch.Tensor) and t.is_cuda]
        if any(t.device != stream.device for t in given):
            raise ValueError(f"stream is on {stream.device}, tensors are not")
        if stream == here:
            return fn(*args, **kw)
        with torch.cuda.stream(stream):
            r = fn(*args, **kw)
        for t in given:
            t.record_stream(stream)
        for t in r.values():
            if t is not None:
                t.record_stream(here)
        return r
    sig = inspect.signature(fn)
    call.__signature__ = sig.replace(parameters=[*sig.parameters.values(),
                                                 inspect.Parameter("stream", inspect.Parameter.KEYWORD_ONLY, default=None)])
    return call


class Model:
    """Device copy of the evaluator's weights (wm_model_create)."""

    def __init__(self, dims: Dict[str, int], weights: Dict[str, np.ndarray], precision: str = "bf16",
                 norm: str = "none"):
        """norm="l2" selects the paper-form transition (hyperplane projection
        and unit length; needs weights["wh"])."""
        lib = load_library()
        self.dims = dict(dims)
        self.precision = precision
        self.norm = norm
        d = Dims(d=dims["d"], embed_dim=dims["e"], n_kinds=dims["n_kinds"],
                 n_params=dims["n_params"], trans_hidden=dims["H"], cost_hidden=dims["C"],
                 hw_dim=dims["hw_dim"], feat_dim=dims.get("feat_dim", 0),
                 enc_hidden=dims.get("enc_hidden", 0), precision=PRECISIONS[precision],
                 norm=NORMS[norm])
        self._keep = {k: np.ascontiguousarray(v, dtype=np.float32) for k, v in weights.items()}
        w = Weights()
        for name, _ in Weights._fields_:
            if name == "bc2":
                w.bc2 = float(np.asarray(self._keep["bc2"]).reshape(-1)[0])
            elif name in self._keep:
                setattr(w, name, self._keep[name].ctypes.data_as(_FP))
        h = ctypes.c_void_p()
        _check(lib.wm_model_create(ctypes.byref(d), ctypes.byref(w), ctypes.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load_library().wm_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, B: int, T_max: int, S: int, n_hw: int) -> int:
        return int(load_library().wm_workspace_bytes(self.handle, B, T_max, S, n_hw))

    def workspace(self, B: int, T_max: int, S: int, n_hw: int, device="cuda"):
        """Zero-filled workspace tensor (uint8) of the required size."""
        import torch
        return torch.zeros(self.workspace_bytes(B, T_max, S, n_hw), dtype=torch.uint8, device=device)


def encode_init(model: Model, feats, z0, stream=None):
    S = feats.shape[0]
    _check(load_library().wm_encode_init(model.handle, _ptr(feats), S, _ptr(z0), _stream(stream)))


def rollout(model: Model, z0, seg_off, types, params, lens, zT, phi, ws, stream=None):
    seg, segp = _host_i32(seg_off)
    B, T_max = types.shape[0], types.shape[1]
    _check(load_library().wm_rollout(
        model.handle, _ptr(z0), segp, len(seg) - 1, _ptr(types), _ptr(params), _ptr(lens),
        B, T_max, _ptr(zT), _ptr(phi), _ptr(ws), ws.numel(), _stream(stream)))


def score(model: Model, zT, phi, hw, scores, stream=None):
    _check(load_library().wm_score(model.handle, _ptr(zT), _ptr(phi), zT.shape[0], _ptr(hw),
                                   hw.shape[0], _ptr(scores), _stream(stream)))


def topk(scores, seg_off, k, idx, val=None, stream=None):
    seg, segp = _host_i32(seg_off)
    _check(load_library().wm_topk(_ptr(scores), scores.shape[0], scores.shape[1], segp,
                                  len(seg) - 1, k, _ptr(idx), _ptr(val), _stream(stream)))


class Forest:
    """Device copy of a tree-ensemble ranker (wm_forest_create)."""

    def __init__(self, feat, thr, leaf, base: float, n_features: int):
        lib = load_library()
        feat = np.ascontiguousarray(feat, dtype=np.int32)
        self._keep = (feat, np.ascontiguousarray(thr, dtype=np.float32),
                      np.ascontiguousarray(leaf, dtype=np.float32))
        n_trees, n_int = feat.shape
        depth = int(round(np.log2(n_int + 1)))
        self.n_trees, self.depth, self.n_features = n_trees, depth, n_features
        h = ctypes.c_void_p()
        _check(lib.wm_forest_create(n_trees, depth, n_features,
                                    *[a.ctypes.data_as(ctypes.c_void_p) for a in self._keep],
                                    float(base), ctypes.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load_library().wm_forest_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def phi_struct(types, params, lens, n_kinds: int, phi_s, stream=None):
    B, T_max = types.shape[0], types.shape[1]
    _check(load_library().wm_phi_struct(_ptr(types), _ptr(params), _ptr(lens), B, T_max, n_kinds,
                                        params.shape[2], _ptr(phi_s), _stream(stream)))


def score_trees(forest: Forest, zT, phi_s, hw, scores, stream=None):
    _check(load_library().wm_score_trees(forest.handle, _ptr(zT), zT.shape[1], _ptr(phi_s),
                                         phi_s.shape[1], zT.shape[0], _ptr(hw), hw.shape[0],
                                         hw.shape[1], _ptr(scores), _stream(stream)))


@_on_stream
def evaluate(model: Model, init, seg_off, types, params, lens, hw, k, *, init_is_feats=False,
             scores=None, zT=None, idx=None, val=None, ws=None, forest=None):
    """Fused [encode,] rollout, score and top-k (wm_evaluate) on device tensors;
    with a Forest, the tree-ensemble ranker on structured action features
    (wm_evaluate_trees).

    Returns a dict with idx [n_hw][S][k], val, and scores / zT when given.
    """
    import torch
    seg, segp = _host_i32(seg_off)
    S = len(seg) - 1
    B, T_max = types.shape[0], types.shape[1]
    n_hw = hw.shape[0]
    dev = types.device
    if idx is None:
        idx = torch.empty((n_hw, S, k), dtype=torch.int32, device=dev)
    if val is None:
        val = torch.empty((n_hw, S, k), dtype=torch.float32, device=dev)
    if ws is None:
        ws = model.workspace(B, T_max, S, n_hw, device=dev)
    args = (_ptr(init), 1 if init_is_feats else 0, segp, S, _ptr(types), _ptr(params),
            _ptr(lens), B, T_max, _ptr(hw), n_hw, k, _ptr(scores), _ptr(zT), _ptr(idx), _ptr(val),
            _ptr(ws), ws.numel(), _stream(None))
    if forest is None:
        _check(load_library().wm_evaluate(model.handle, *args))
    else:
        _check(load_library().wm_evaluate_trees(model.handle, forest.handle, *args))
    return {"idx": idx, "val": val, "scores": scores, "zT": zT, "ws": ws}


def evaluate_noalloc(model: Model, init, seg_off, types, params, lens, hw, k, *, scores, zT, phi,
                     idx, status, val=None, init_is_feats=False, stream=None):
    """wm_evaluate_noalloc: the fused path with every output supplied by the
    caller (scores [n_hw][B], zT [B][d], phi [B][e], idx [n_hw][S][k], val or
    None, status int32 [64]) and no workspace; nothing is allocated.  Check
    the device error word with device_status(status)."""
    seg, segp = _host_i32(seg_off)
    S = len(seg) - 1
    B, T_max = types.shape[0], types.shape[1]
    n_hw = hw.shape[0]
    _check(load_library().wm_evaluate_noalloc(
        model.handle, _ptr(init), 1 if init_is_feats else 0, segp, S, _ptr(types), _ptr(params),
        _ptr(lens), B, T_max, _ptr(hw), n_hw, k, _ptr(scores), _ptr(zT), _ptr(phi), _ptr(idx),
        _ptr(val), _ptr(status), _stream(stream)))
    return {"idx": idx, "val": val, "scores": scores, "zT": zT, "phi": phi, "status": status}


def grad_shapes(model: Model) -> Dict[str, tuple]:
    """Shapes of the weight gradients of a model (PyTorch Linear layout)."""
    d = model.dims
    shapes = {"w1": (d["H"], d["d"] + d["e"]), "b1": (d["H"],), "w2": (d["d"], d["H"]),
              "b2": (d["d"],), "type_emb": (d["n_kinds"], d["e"]),
              "param_w": (d["e"], d["n_params"]), "param_b": (d["e"],)}
    if model.norm == "l2":
        shapes["wh"] = (d["d"], d["e"])
    return shapes


def loss_workspace(model: Model, B: int, T_max: int, device="cuda"):
    """Zero-filled workspace tensor (uint8) for rollout_loss."""
    import torch
    n = int(load_library().wm_loss_workspace_bytes(model.handle, B, T_max))
    return torch.zeros(n, dtype=torch.uint8, device=device)


@_on_stream
def rollout_loss(model: Model, z0, seg_off, types, params, lens, targets, negatives, lam: float,
                 gamma: float, *, grads=True, dz0=True, loss=None, total=None, out=None, ws=None):
    """Rollout loss and its gradients (wm_rollout_loss) on device tensors.

    targets [B][T_max][d], negatives [B][T_max][n_neg][d].  Returns a dict
    with loss [B], total [1] and, when grads is true, the weight gradients
    (keys of grad_shapes) and z0 [B][d] (when dz0 is true).  `out` may hold
    preallocated gradient tensors under the same keys.
    """
    import torch
    seg, segp = _host_i32(seg_off)
    S = len(seg) - 1
    B, T_max = types.shape[0], types.shape[1]
    dev = types.device
    if loss is None:
        loss = torch.empty(B, dtype=torch.float32, device=dev)
    if total is None:
        total = torch.empty(1, dtype=torch.float32, device=dev)
    if ws is None:
        ws = loss_workspace(model, B, T_max, device=dev)
    res = {"loss": loss, "total": total, "ws": ws}
    gp = None
    if grads:
        out = dict(out or {})
        for k, shp in grad_shapes(model).items():
            if k not in out:
                out[k] = torch.empty(shp, dtype=torch.float32, device=dev)
        if dz0 and "z0" not in out:
            out["z0"] = torch.empty((B, model.dims["d"]), dtype=torch.float32, device=dev)
        g = Grads(**{k: _ptr(v).value for k, v in out.items() if k in dict(Grads._fields_)})
        gp = ctypes.byref(g)
        res.update(out)
    _check(load_library().wm_rollout_loss(
        model.handle, _ptr(z0), segp, S, _ptr(types), _ptr(params), _ptr(lens), B, T_max,
        _ptr(targets), _ptr(negatives), negatives.shape[2] if negatives.dim() == 4 else 0,
        float(lam), float(gamma), _ptr(loss), _ptr(total), gp, _ptr(ws), ws.numel(),
        _stream(None)))
    return res


class TextModel:
    """Device copy of the chunked transformer state encoder (wm_text_model_create)."""

    def __init__(self, w, weights: Dict[str, np.ndarray], precision: str = "bf16"):
        """w: object with vocab, hidden, heads, ffn, layers, window, stride, d."""
        lib = load_library()
        self.w = w
        self.precision = precision
        d = TextDims(vocab=w.vocab, hidden=w.hidden, heads=w.heads, ffn=w.ffn, layers=w.layers,
                     window=w.window, stride=w.stride, d=w.d, precision=PRECISIONS[precision])
        self._keep = {k: np.ascontiguousarray(weights[k], dtype=np.float32) for k in TEXT_WEIGHT_KEYS}
        tw = TextWeights(**{k: self._keep[k].ctypes.data_as(_FP) for k in TEXT_WEIGHT_KEYS})
        h = ctypes.c_void_p()
        _check(lib.wm_text_model_create(ctypes.byref(d), ctypes.byref(tw), ctypes.byref(h)))
        self.handle = h
        self._keep = None           # copied to the device

    def close(self):
        if getattr(self, "handle", None):
            load_library().wm_text_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def chunks(self, tok_off) -> int:
        off, offp = _host_i32(tok_off)
        n = int(load_library().wm_text_chunks(self.handle, offp, len(off) - 1))
        if n < 0:
            raise WMError(WM_ERR_INVALID_ARGUMENT, "bad tok_off")
        return n

    def workspace(self, tok_off, device="cuda"):
        import torch
        n = int(load_library().wm_text_workspace_bytes(self.handle, self.chunks(tok_off)))
        return torch.zeros(n, dtype=torch.uint8, device=device)


def encode_text(model: TextModel, tokens, tok_off, z0=None, ws=None, stream=None):
    """z0 [S][d] from concatenated token ids (device int32) and HOST tok_off [S+1]."""
    return _encode_text(model, tokens, tok_off, z0, ws, stream=stream)


@_on_stream
def _encode_text(model, tokens, tok_off, z0, ws):
    import torch
    off, offp = _host_i32(tok_off)
    S = len(off) - 1
    dev = tokens.device
    if z0 is None:
        z0 = torch.empty((S, model.w.d), dtype=torch.float32, device=dev)
    if ws is None:
        ws = model.workspace(off, device=dev)
    _check(load_library().wm_encode_text(model.handle, _ptr(tokens), offp, S, _ptr(z0), _ptr(ws),
                                         ws.numel(), _stream(None)))
    return {"z0": z0, "ws": ws}


# ---- sequence operators ----------------------------------------------------------
# The checks run on every call of a step-by-step rollout, whose kernels take some 10 us: they
# compare shapes, types and devices directly and build the argument blocks positionally.
_DTYPES = {}


def _dtype(t):
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: WM_BF16, torch.float32: WM_FP32})
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"tensors must be float32 or bfloat16, not {t.dtype}")
    return d


def _on_gpu(t):
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")


def _same(like, shape, **tensors):
    """Checks that tensors (None allowed) are on like's device with its dtype and `shape`."""
    dtype, dev = like.dtype, like.device
    for name, t in tensors.items():
        if t is not None and (t.shape != shape or t.dtype != dtype or t.device != dev):
            raise ValueError(f"{name} must be {tuple(shape)} {dtype} on {dev}, not {tuple(t.shape)} {t.dtype} on {t.device}")


def _f32(dev, shape, **tensors):
    """Checks that tensors (None allowed) are dense float32 of `shape` on `dev`."""
    for name, t in tensors.items():
        if t is not None and (t.shape != shape or _DTYPES.get(t.dtype) != WM_FP32 or t.device != dev or not t.is_contiguous()):
            raise ValueError(f"{name} must be dense {tuple(shape)} float32 on {dev}")


def _rows(name, t):
    """Row stride of a matrix [rows][width] or [rows][heads][width] whose rows are dense."""
    shape, stride = t.shape, t.stride()
    width = 1
    for i in range(len(shape) - 1, 0, -1):
        n = shape[i]
        if n > 1 and stride[i] != width:
            raise ValueError(f"{name}: only the row stride may differ from a dense tensor's")
        width *= n
    return stride[0] if shape[0] > 1 else width


def _addr(t):
    return None if t is None else t.data_ptr()


def _given(name, t, dev):
    """Bytes of a caller's workspace or kept states."""
    if t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be dense on {dev}")
    return t.numel() * t.element_size()


def _workspace(n, given, dev):
    """The workspace and its bytes; the library answers 256 where it needs none, more where it does."""
    import torch
    if given is not None:
        return given, _given("ws", given, dev)
    return (torch.empty(n, dtype=torch.uint8, device=dev), n) if n > 256 else (None, 0)


def _launch(fn, dev, *args):
    """A library call on the current stream of dev, which is the current device meanwhile."""
    import torch
    stream = torch.cuda.current_stream(dev.index).cuda_stream
    if torch.cuda.current_device() == dev.index:
        _check(fn(*args, stream))
    else:
        with torch.cuda.device(dev):
            _check(fn(*args, stream))


def _attention(q, k, v, q_off, k_off, kv_mask, scale):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k and v are [rows][heads][head_dim]")
    if k.shape[2] != q.shape[2]:
        raise ValueError("q and k differ in head_dim")
    dtype = _dtype(q)
    _same(q, k.shape, k=k, v=v)
    qo, ko = np.ascontiguousarray(q_off, dtype=np.int32), np.ascontiguousarray(k_off, dtype=np.int32)
    qp, kp = qo.ctypes.data, ko.ctypes.data
    if qo.ndim != 1 or len(qo) != len(ko) or len(qo) < 2:
        raise ValueError("q_off and k_off need S + 1 entries each")
    if qo[-1] != q.shape[0] or ko[-1] != k.shape[0]:
        raise ValueError("q_off and k_off must end at the number of rows")
    if kv_mask is not None:
        import torch
        if kv_mask.dtype not in (torch.uint8, torch.bool) or tuple(kv_mask.shape) != (k.shape[0],) or \
                kv_mask.device != q.device or not kv_mask.is_contiguous():
            raise ValueError("kv_mask must be dense uint8 or bool [key rows] on the tensors' device")
    # in the order of Attention's fields
    a = Attention(dtype, q.shape[1], k.shape[1], q.shape[2], len(qo) - 1, qp, kp, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                  _rows("q", q), _rows("k", k), _rows("v", v), _addr(kv_mask), q.shape[2] ** -0.5 if scale is None else scale)
    a.keep = (qo, ko)
    _on_gpu(q)
    return a


@_on_stream
def cross_attention(q, k, v, q_off, k_off, *, kv_mask=None, scale=None, o=None, lse=None, need_lse=False, ws=None):
    """Cross attention of query rows to the key rows of their segment (wm_cross_attention).

    q [rows][heads][head_dim], k and v [rows][kv_heads][head_dim], float32 or bfloat16; row strides may
    be larger than dense.  q_off, k_off: HOST [S + 1].  kv_mask: uint8 or bool per key row (0 =
    hidden).  scale defaults to head_dim ** -0.5.  Returns o, lse [rows][heads] (with need_lse or
    when given; the gradient needs it) and ws.
    """
    import torch
    a = _attention(q, k, v, q_off, k_off, kv_mask, scale)
    if o is None:
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _same(q, q.shape, o=o)
    if lse is None and need_lse:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    _f32(q.device, q.shape[:2], lse=lse)
    lib = load_library()
    ws, n = _workspace(lib.wm_cross_attention_workspace_bytes(a, 0), ws, q.device)
    _launch(lib.wm_cross_attention, q.device, a, o.data_ptr(), _rows("o", o), _addr(lse), _addr(ws), n)
    return {"o": o, "lse": lse, "ws": ws}


@_on_stream
def cross_attention_grad(do, q, k, v, o, lse, q_off, k_off, *, kv_mask=None, scale=None, dq=None, dk=None, dv=None, ws=None):
    """Gradients dq, dk, dv of cross_attention given do = dL/do (wm_cross_attention_grad)."""
    import torch
    a = _attention(q, k, v, q_off, k_off, kv_mask, scale)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
    _same(q, q.shape, o=o, do=do, dq=dq)
    _same(q, k.shape, dk=dk, dv=dv)
    _f32(q.device, q.shape[:2], lse=lse)
    lib = load_library()
    ws, n = _workspace(lib.wm_cross_attention_workspace_bytes(a, 1), ws, q.device)
    _launch(lib.wm_cross_attention_grad, q.device, a, o.data_ptr(), _rows("o", o), _addr(lse), do.data_ptr(), _rows("do", do),
            dq.data_ptr(), _rows("dq", dq), dk.data_ptr(), _rows("dk", dk), dv.data_ptr(), _rows("dv", dv), _addr(ws), n)
    return {"dq": dq, "dk": dk, "dv": dv, "ws": ws}


def _offsets_ok(off, dev):
    import torch
    if off.dtype != torch.int32 or off.dim() != 1 or off.numel() < 1 or off.device != dev or not off.is_contiguous():
        raise ValueError("off must be dense int32 [B + 1] on the tensors' device")
    return off.numel() - 1


def _status_ok(status, dev):
    import torch
    if status.dtype != torch.int32 or status.numel() < 64 or status.device != dev or not status.is_contiguous():
        raise ValueError("status must be dense int32 [64] on the tensors' device")


def _conv(x, off, weight, bias, T_max, silu, state, status):
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x is [rows][channels], weight [channels][width]")
    C, W = x.shape[1], weight.shape[1]
    B = _offsets_ok(off, x.device)
    dtype = _dtype(x)
    _f32(x.device, (C, W), weight=weight)
    _f32(x.device, (C,), bias=bias)
    _same(x, (B, W - 1, C), state=state)
    if state is not None and not state.is_contiguous():
        raise ValueError("state must be dense")
    _on_gpu(x)
    if status is not None:
        _status_ok(status, x.device)
    # in the order of Conv's fields
    return Conv(dtype, B, T_max, C, W, 1 if silu else 0, x.shape[0], off.data_ptr(), x.data_ptr(), _rows("x", x),
                weight.data_ptr(), _addr(bias), _addr(state), _addr(status))


@_on_stream
def causal_conv(x, off, weight, bias=None, *, T_max, silu=True, state=None, state_out=None, need_state=False, y=None,
                status=None):
    """Causal convolution along packed ragged sequences (wm_causal_conv).

    x [rows][channels] float32 or bfloat16, off device int32 [B + 1], T_max: the longest sequence's
    rows, weight [channels][width] and bias [channels] float32; state [B][width - 1][channels]:
    the inputs before every sequence.  Returns y and state (the last width - 1 inputs, with
    need_state or state_out, which may be `state`).  status: zeroed int32 [64] for device_status.
    """
    import torch
    a = _conv(x, off, weight, bias, T_max, silu, state, status)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if y is None else y
    if state_out is None and need_state:
        state_out = torch.empty((a.B, a.width - 1, a.channels), dtype=x.dtype, device=x.device)
    _same(x, x.shape, y=y)
    _same(x, (a.B, a.width - 1, a.channels), state_out=state_out)
    _launch(load_library().wm_causal_conv, x.device, a, y.data_ptr(), _rows("y", y), _ptr(state_out))
    return {"y": y, "state": state_out}


@_on_stream
def causal_conv_grad(dy, x, off, weight, bias=None, *, T_max, silu=True, state=None, d_state_out=None, need_dstate=False,
                     status=None, ws=None):
    """Gradients dx, dweight, dbias and (with need_dstate) dstate of causal_conv (wm_causal_conv_grad)."""
    import torch
    a = _conv(x, off, weight, bias, T_max, silu, state, status)
    dev = x.device
    _same(x, x.shape, dy=dy)
    shape = (a.B, a.width - 1, a.channels)
    _same(x, shape, d_state_out=d_state_out)
    dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
    dw = torch.empty(weight.shape, dtype=torch.float32, device=dev)
    db = torch.empty(a.channels, dtype=torch.float32, device=dev)
    ds = torch.empty(shape, dtype=x.dtype, device=dev) if need_dstate else None
    lib = load_library()
    ws, n = _workspace(lib.wm_causal_conv_workspace_bytes(a), ws, dev)
    _launch(lib.wm_causal_conv_grad, dev, a, dy.data_ptr(), _rows("dy", dy), _ptr(d_state_out), dx.data_ptr(), _rows("dx", dx),
            dw.data_ptr(), db.data_ptr(), _addr(ds), _addr(ws), n)
    return {"dx": dx, "dweight": dw, "dbias": db, "dstate": ds, "ws": ws}


def _scan(u, delta, A, Bm, Cm, off, T_max, D, z, delta_bias, h0, status):
    if u.dim() != 2 or A.dim() != 2 or Bm.dim() != 2:
        raise ValueError("u is [rows][channels], A [channels][states], Bm and Cm [rows][states]")
    C, N = A.shape
    B = _offsets_ok(off, u.device)
    dtype = _dtype(u)
    _same(u, (u.shape[0], C), u=u, delta=delta, z=z)
    _same(u, (u.shape[0], N), Bm=Bm, Cm=Cm)
    _f32(u.device, (C, N), A=A)
    _f32(u.device, (C,), D=D, delta_bias=delta_bias)
    _f32(u.device, (B, C, N), h0=h0)
    lds = [_rows(n, t) if t is not None else 0 for n, t in (("u", u), ("delta", delta), ("z", z), ("Bm", Bm), ("Cm", Cm))]
    _on_gpu(u)
    if status is not None:
        _status_ok(status, u.device)
    # in the order of ScanArgs' fields
    return ScanArgs(dtype, B, T_max, C, N, u.shape[0], off.data_ptr(), u.data_ptr(), delta.data_ptr(), _addr(z), Bm.data_ptr(),
                    Cm.data_ptr(), *lds, A.data_ptr(), _addr(D), _addr(delta_bias), _addr(h0), _addr(status))


@_on_stream
def selective_scan(u, delta, A, Bm, Cm, off, *, T_max, D=None, z=None, delta_bias=None, h0=None, hT=None, need_state=False,
                   need_checkpoints=False, checkpoints=None, y=None, status=None, ws=None):
    """Selective state-space scan along packed ragged sequences (wm_scan); T_max = 1 is one step.

    u, delta, z [rows][channels], Bm, Cm [rows][states], float32 or bfloat16; A [channels][states], D and
    delta_bias [channels], h0 [B][channels][states] float32; off device int32 [B + 1].  Returns y, hT
    (with need_state, or given: may be h0) and checkpoints (with need_checkpoints, or given: what
    selective_scan_grad needs).  status: zeroed int32 [64] for device_status.
    """
    import torch
    a = _scan(u, delta, A, Bm, Cm, off, T_max, D, z, delta_bias, h0, status)
    dev = u.device
    lib = load_library()
    y = torch.empty(u.shape, dtype=u.dtype, device=dev) if y is None else y
    if hT is None and need_state:
        hT = torch.empty((a.B, a.channels, a.states), dtype=torch.float32, device=dev)
    if checkpoints is None and need_checkpoints:
        checkpoints = torch.empty(lib.wm_scan_checkpoint_bytes(a), dtype=torch.uint8, device=dev)
    _same(u, u.shape, y=y)
    _f32(dev, (a.B, a.channels, a.states), hT=hT)
    if checkpoints is not None and _given("checkpoints", checkpoints, dev) < lib.wm_scan_checkpoint_bytes(a):
        raise ValueError("checkpoints is too small")
    ws, n = (None, 0) if T_max <= 1 and ws is None else _workspace(lib.wm_scan_workspace_bytes(a, 0), ws, dev)
    _launch(lib.wm_scan, dev, a, y.data_ptr(), _rows("y", y), _addr(hT), _addr(checkpoints), _addr(ws), n)
    return {"y": y, "hT": hT, "checkpoints": checkpoints, "ws": ws}


@_on_stream
def selective_scan_grad(dy, u, delta, A, Bm, Cm, off, checkpoints, *, T_max, D=None, z=None, delta_bias=None, h0=None, dhT=None,
                        need_dh0=None, status=None, ws=None):
    """Gradients of selective_scan (wm_scan_grad): du, ddelta, dA, dB, dC, dD, ddelta_bias, dz (with z) and dh0
    (with h0, or need_dh0), given dy, the forward call's checkpoints and dhT (None = 0)."""
    import torch
    a = _scan(u, delta, A, Bm, Cm, off, T_max, D, z, delta_bias, h0, status)
    dev = u.device
    _same(u, u.shape, dy=dy)
    shape = (a.B, a.channels, a.states)
    _f32(dev, shape, dhT=dhT)
    need_dh0 = h0 is not None if need_dh0 is None else need_dh0
    lib = load_library()
    if checkpoints is None or _given("checkpoints", checkpoints, dev) < lib.wm_scan_checkpoint_bytes(a):
        raise ValueError("checkpoints is missing or too small")
    like = dict(dtype=u.dtype, device=dev)
    f32 = dict(dtype=torch.float32, device=dev)
    C, N = A.shape
    r = {"du": torch.empty(u.shape, **like), "ddelta": torch.empty(u.shape, **like),
         "dz": torch.empty(u.shape, **like) if z is not None else None, "dB": torch.empty(Bm.shape, **like),
         "dC": torch.empty(Cm.shape, **like), "dA": torch.empty((C, N), **f32), "dD": torch.empty(C, **f32),
         "ddelta_bias": torch.empty(C, **f32), "dh0": torch.empty(shape, **f32) if need_dh0 else None}
    g = ScanGrads(ld_du=C, ld_ddelta=C, ld_dz=C, ld_dB=N, ld_dC=N, **{k: _addr(t) for k, t in r.items()})
    ws, n = _workspace(lib.wm_scan_workspace_bytes(a, 1), ws, dev)
    _launch(lib.wm_scan_grad, dev, a, _addr(checkpoints), dy.data_ptr(), _rows("dy", dy), _addr(dhT), g, _addr(ws), n)
    return {**r, "ws": ws}


# ---- attention over a shared prefix ------------------------------------------------
# A step of a program is a few microseconds of kernels: the checks look at each tensor once (on the host, 9 us for an append, 14 before).
def _dense(name, t, dtype, gpu, shape):
    """Address of a dense tensor (None allowed) of `shape` on device `gpu`."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or t.get_device() != gpu or not t.is_contiguous():
        raise ValueError(f"{name} must be dense {tuple(shape)} {dtype} on the GPU of the other tensors")
    return t.data_ptr()


def _rows3(name, t, dtype, gpu, shape):
    """Address and row stride of [rows][heads][head_dim] whose rows are dense."""
    if t.dtype != dtype or t.shape != shape or t.get_device() != gpu:
        raise ValueError(f"{name} must be {tuple(shape)} {dtype} on the GPU of the other tensors, not {tuple(t.shape)} {t.dtype} on {t.device}")
    rows, heads, dim = shape
    s = t.stride()
    if (s[2] != 1 and dim > 1) or (s[1] != dim and heads > 1):
        raise ValueError(f"{name}: only the row stride may differ from a dense tensor's")
    return t.data_ptr(), s[0] if rows > 1 else heads * dim


def _status(name, t, gpu):
    if t is None:
        return None
    if t.numel() < 64:
        raise ValueError(f"{name} must be dense int32 [64] on the tensors' device")
    import torch
    return _dense(name, t, torch.int32, gpu, t.shape)


def _shape3(name, t):
    shape = t.shape
    if len(shape) != 3:
        raise ValueError(f"{name} is [rows][heads][head_dim]")
    return shape


def _length1(name, t):
    shape = t.shape
    if len(shape) != 1 or shape[0] < 1:
        raise ValueError(f"{name} has one axis, not empty")
    return shape[0]


@_on_stream
def rotate(x, off, freq, *, T_max, first=None, interleaved=False, inverse=False, y=None, status=None):
    """Rotation of packed rows by position (wm_rotate): pair i of a head by position * freq[i].

    x [rows][heads][head_dim] float32 or bfloat16, off device int32 [B + 1], T_max: the longest sequence's
    rows; freq [rot / 2] float32 turns the first rot features of a head: features i and i + rot / 2, or 2 i and
    2 i + 1 (interleaved).  Row i of sequence s is at position first[s] + i (first: device int32 [B], None = 0).
    inverse turns back: the gradient of a rotation is the rotation of its gradient with the other sign.  Returns
    y (given: may be x; rows behind the last sequence stay).  status: zeroed int32 [64] for device_status.
    """
    import torch
    shape, dtype, gpu = _shape3("x", x), x.dtype, x.get_device()
    kind, B, pairs = _dtype(x), _length1("off", off) - 1, _length1("freq", freq)
    _on_gpu(x)
    xp, ld_x = _rows3("x", x, dtype, gpu, shape)
    y = torch.empty(shape, dtype=dtype, device=x.device) if y is None else y
    yp, ld_y = _rows3("y", y, dtype, gpu, shape)
    # in the order of Rotation's fields
    a = Rotation(kind, B, T_max, shape[1], shape[2], 2 * pairs, 1 if interleaved else 0, 1 if inverse else 0, shape[0],
                 _dense("off", off, torch.int32, gpu, (B + 1,)), _dense("first", first, torch.int32, gpu, (B,)),
                 _dense("freq", freq, torch.float32, gpu, (pairs,)), xp, ld_x, _status("status", status, gpu))
    _launch(load_library().wm_rotate, x.device, a, yp, ld_y)
    return {"y": y}


def _cache(k_cache, v_cache, pages, lens):
    shape, table, kind = k_cache.shape, pages.shape, _dtype(k_cache)
    if len(shape) != 4 or len(table) != 2:
        raise ValueError("caches are [n_pages][kv_heads][page][head_dim], pages [B][max_pages]")
    _on_gpu(k_cache)
    import torch
    dtype, gpu = k_cache.dtype, k_cache.get_device()
    n, heads, page, dim = shape
    B, width = table
    # in the order of Cache's fields
    return Cache(kind, heads, dim, page, n, B, width, _dense("k_cache", k_cache, dtype, gpu, shape),
                 _dense("v_cache", v_cache, dtype, gpu, shape), _dense("pages", pages, torch.int32, gpu, table),
                 _dense("lens", lens, torch.int32, gpu, (B,)))


@_on_stream
def cache_append(k, v, k_cache, v_cache, pages, lens, off, *, T_max, first=None, freq=None, interleaved=False, q=None, q_out=None,
                 status=None):
    """Appends keys and values to a paged cache, the keys rotated on the way (wm_cache_append).

    k, v [rows][kv_heads][head_dim] (q [rows][heads][head_dim]) of the caches' type; k_cache, v_cache
    [n_pages][kv_heads][page][head_dim], changed in place; pages int32 [B][max_pages], lens int32 [B], off int32 [B + 1]
    on the device.  lens counts the new rows: row i of the n of sequence s goes to slot lens[s] - n + i, at position
    first[s] + slot.  freq and interleaved as in rotate; without freq nothing is rotated.  Returns q (rotated alike;
    q_out may be q), k_cache and v_cache.  status: zeroed int32 [64] for device_status.
    """
    import torch
    c = _cache(k_cache, v_cache, pages, lens)
    dtype, dev, gpu, int32, B = k_cache.dtype, k_cache.device, k_cache.get_device(), torch.int32, c.B
    rows = _shape3("k", k)[0]
    (kp, ld_k), (vp, ld_v) = (_rows3(n, t, dtype, gpu, (rows, c.kv_heads, c.head_dim)) for n, t in (("k", k), ("v", v)))
    pairs = 0 if freq is None else _length1("freq", freq)
    heads = ld_q = ld_out = 0
    qp = out = None
    if q is not None:
        heads = _shape3("q", q)[1]
        shape = (rows, heads, c.head_dim)
        qp, ld_q = _rows3("q", q, dtype, gpu, shape)
        q_out = torch.empty(shape, dtype=dtype, device=dev) if q_out is None else q_out
        out, ld_out = _rows3("q_out", q_out, dtype, gpu, shape)
    elif q_out is not None:
        raise ValueError("q_out without q")
    # in the order of Append's fields
    a = Append(c, T_max, heads, 2 * pairs, 1 if interleaved else 0, rows, _dense("off", off, int32, gpu, (B + 1,)),
               _dense("first", first, int32, gpu, (B,)), _dense("freq", freq, torch.float32, gpu, (pairs,)), kp, vp, qp, ld_k, ld_v, ld_q,
               _status("status", status, gpu))
    _launch(load_library().wm_cache_append, dev, a, out, ld_out)
    return {"q": q_out, "k_cache": k_cache, "v_cache": v_cache}


@_on_stream
def cached_attention(q, k_cache, v_cache, pages, lens, off, *, T_max, len_max=None, seg_off=None, prefix_pages=None, prefix_lens=None,
                     prefix_max=None, scale=None, o=None, lse=None, need_lse=False, status=None, ws=None):
    """Attention of new rows to their sequence's cached keys and to those that its program's sequences share
    (wm_cached_attention).

    q [rows][heads][head_dim]; caches, pages, lens and off as in cache_append: row i of the n of sequence s sees the
    sequence's keys 0 .. lens[s] - n + i.  With seg_off (HOST [S + 1], from 0 to B), the sequences of program p also see
    its prefix_lens[p] keys (device int32 [S]) in the pages prefix_pages[p] (device int32 [S][...]) of the same pool.  len_max and
    prefix_max: no length is greater (default: what the tables hold; closer bounds divide the work better).  scale
    defaults to head_dim ** -0.5.  Returns o, lse [rows][heads] (with need_lse or when given; rows behind the last sequence
    stay) and ws.  status: zeroed int32 [64] for device_status.
    """
    import torch
    c = _cache(k_cache, v_cache, pages, lens)
    dtype, dev, gpu, int32, B = k_cache.dtype, k_cache.device, k_cache.get_device(), torch.int32, c.B
    rows, heads, dim = shape = _shape3("q", q)
    if dim != c.head_dim:
        raise ValueError("q and the caches differ in head_dim")
    qp, ld_q = _rows3("q", q, dtype, gpu, shape)
    len_max = c.max_pages * c.page if len_max is None else len_max
    S = shared_pages = 0
    seg = segp = table = shared_lens = None
    if seg_off is None:
        if prefix_pages is not None or prefix_lens is not None:
            raise ValueError("prefix_pages and prefix_lens need seg_off")
    else:
        if prefix_pages is None or prefix_lens is None or prefix_pages.dim() != 2:
            raise ValueError("seg_off needs prefix_pages [S][...] and prefix_lens [S]")
        seg = np.ascontiguousarray(seg_off, dtype=np.int32)
        S = len(seg) - 1
        if seg.ndim != 1 or S < 1 or seg[-1] != B:
            raise ValueError("seg_off must end at the number of sequences")
        segp, shared_pages = seg.ctypes.data, prefix_pages.shape[1]
        table = _dense("prefix_pages", prefix_pages, int32, gpu, (S, shared_pages))
        shared_lens = _dense("prefix_lens", prefix_lens, int32, gpu, (S,))
    prefix_max = shared_pages * c.page if prefix_max is None else prefix_max
    o = torch.empty(shape, dtype=dtype, device=dev) if o is None else o
    op, ld_o = _rows3("o", o, dtype, gpu, shape)
    if lse is None and need_lse:
        lse = torch.empty((rows, heads), dtype=torch.float32, device=dev)
    # in the order of Cached's fields
    a = Cached(c, T_max, len_max, heads, S, shared_pages, prefix_max, rows, _dense("off", off, int32, gpu, (B + 1,)), segp, table, shared_lens,
               qp, ld_q, dim ** -0.5 if scale is None else scale, _status("status", status, gpu))
    lib = load_library()
    ws, n = _workspace(lib.wm_cached_attention_workspace_bytes(a), ws, dev)
    _launch(lib.wm_cached_attention, dev, a, op, ld_o, _dense("lse", lse, torch.float32, gpu, (rows, heads)), _addr(ws), n)
    return {"o": o, "lse": lse, "ws": ws}


def _prefix(q, k, v, pk, pv, off, q_off, p_off, T_max, kv_mask, scale, status):
    _shape3("k", k)
    _shape3("pk", pk)
    a = _attention(q, pk, pv, q_off, p_off, kv_mask, scale)
    _same(q, (q.shape[0],) + tuple(pk.shape[1:]), k=k, v=v)
    B = _offsets_ok(off, q.device)
    if status is not None:
        _status_ok(status, q.device)
    # in the order of Prefix's fields
    p = Prefix(a, k.data_ptr(), v.data_ptr(), _rows("k", k), _rows("v", v), B, T_max, off.data_ptr(), _addr(status))
    p.keep = a.keep
    return p


@_on_stream
def prefix_attention(q, k, v, pk, pv, off, q_off, p_off, *, T_max, kv_mask=None, scale=None, o=None, lse=None, need_lse=False,
                     status=None, ws=None):
    """Causal attention of packed sequences whose programs' keys come first (wm_prefix_attention).

    q [rows][heads][head_dim], own keys k, v [rows][kv_heads][head_dim], the programs' keys pk, pv
    [program rows][kv_heads][head_dim], float32 or bfloat16; row strides may be larger than dense.  off: device int32
    [B + 1], the sequences' rows (at most T_max each); q_off, p_off: HOST [S + 1], the programs' query rows and keys.  A
    row sees its program's keys (those with kv_mask != 0) and own keys from its sequence's first row to itself.  Returns o, lse
    [rows][heads] (with need_lse or when given; the gradient needs it) and ws.  Rows behind the last sequence stay.  status: zeroed
    int32 [64] for device_status.
    """
    import torch
    a = _prefix(q, k, v, pk, pv, off, q_off, p_off, T_max, kv_mask, scale, status)
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if o is None else o
    _same(q, q.shape, o=o)
    if lse is None and need_lse:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    _f32(q.device, q.shape[:2], lse=lse)
    lib = load_library()
    ws, n = _workspace(lib.wm_prefix_attention_workspace_bytes(a, 0), ws, q.device)
    _launch(lib.wm_prefix_attention, q.device, a, o.data_ptr(), _rows("o", o), _addr(lse), _addr(ws), n)
    return {"o": o, "lse": lse, "ws": ws}


@_on_stream
def prefix_attention_grad(do, q, k, v, pk, pv, o, lse, off, q_off, p_off, *, T_max, kv_mask=None, scale=None, dq=None, dk=None, dv=None,
                          dpk=None, dpv=None, status=None, ws=None):
    """Gradients dq, dk, dv, dpk and dpv of prefix_attention given do = dL/do (wm_prefix_attention_grad).

    Each may be given, with a row stride larger than dense.  Rows behind the last sequence stay: in a gradient that is not
    given they hold what its memory held.
    """
    import torch
    a = _prefix(q, k, v, pk, pv, off, q_off, p_off, T_max, kv_mask, scale, status)
    dev = q.device
    _same(q, q.shape, o=o, do=do, dq=dq)
    _same(q, k.shape, dk=dk, dv=dv)
    _same(q, pk.shape, dpk=dpk, dpv=dpv)
    _f32(dev, q.shape[:2], lse=lse)
    r = {n: torch.empty(t.shape, dtype=t.dtype, device=dev) if g is None else g
         for n, t, g in (("dq", q, dq), ("dk", k, dk), ("dv", v, dv), ("dpk", pk, dpk), ("dpv", pv, dpv))}
    g = PrefixGrads(*[_addr(t) for t in r.values()], *[_rows(n, t) for n, t in r.items()])
    lib = load_library()
    ws, n = _workspace(lib.wm_prefix_attention_workspace_bytes(a, 1), ws, dev)
    _launch(lib.wm_prefix_attention_grad, dev, a, o.data_ptr(), _rows("o", o), _addr(lse), do.data_ptr(), _rows("do", do), g, _addr(ws), n)
    return {**r, "ws": ws}


def device_status(ws, stream=None) -> int:
    """Synchronise and read/clear the workspace error word; raises on an error."""
    _check(load_library().wm_device_status(_ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    return WM_OK


def timing_enable(on: bool):
    _check(load_library().wm_timing_enable(1 if on else 0))


def timing_read(kernel: str):
    """(total milliseconds, launches) recorded for a kernel family since enabling."""
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(load_library().wm_timing_read(KERNELS[kernel], ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value
