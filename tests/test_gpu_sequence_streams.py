"""The sequence operators with `stream=`: results on a busy side stream are those of the current stream, and memory that a
call drops on return is not handed to the current stream's work while the side stream still uses it."""
import pytest

from test_gpu_sequence import make_attn, make_conv, make_scan, torch, wm  # noqa: F401

pytestmark = pytest.mark.gpu


def operators(wm):  # noqa: F811
    """(operator, workspace bytes to look out for, call) of loops that are split or cut, so that workspaces are used."""
    q, k, v, qo, ko, _, do = make_attn("bf16", [40], [3000], 4, 1, 64, seed=70)
    f = wm.cross_attention(q, k, v, qo, ko, need_lse=True)
    a, opt, off, dy, dhT = make_scan("f32", [300, 129], 48, 16, 71)
    s = (a["u"], a["delta"], a["A"], a["Bm"], a["Cm"], off)
    g = wm.selective_scan(*s, T_max=300, need_state=True, need_checkpoints=True, **opt)
    x, xo, w, b, st, cdy, ds = make_conv("bf16", [30, 9], 48, 4, 72)
    return {
        "cross_attention": lambda **kw: wm.cross_attention(q, k, v, qo, ko, need_lse=True, **kw),
        "cross_attention_grad": lambda **kw: wm.cross_attention_grad(do, q, k, v, f["o"], f["lse"], qo, ko, **kw),
        "selective_scan": lambda **kw: wm.selective_scan(*s, T_max=300, need_state=True, need_checkpoints=True, **opt, **kw),
        "selective_scan_grad": lambda **kw: wm.selective_scan_grad(dy, *s, g["checkpoints"], T_max=300, dhT=dhT, **opt, **kw),
        "causal_conv": lambda **kw: wm.causal_conv(x, xo, w, b, T_max=30, state=st, need_state=True, **kw),
        "causal_conv_grad": lambda **kw: wm.causal_conv_grad(cdy, x, xo, w, b, T_max=30, state=st, d_state_out=ds, need_dstate=True, **kw),
    }


def test_given_stream(wm):  # noqa: F811
    m = torch.randn(8192, 8192, device="cuda").to(torch.bfloat16)
    busy = torch.empty_like(m)
    side = torch.cuda.Stream()
    for name, call in operators(wm).items():
        print(f"[stream] {name}", flush=True)
        r = call()
        keys = [n for n, t in r.items() if t is not None and n not in ("ws", "checkpoints")]
        sizes = [t.numel() * t.element_size() for t in r.values() if t is not None]
        want = {n: r[n].clone() for n in keys}
        del r
        for n in keys:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                for _ in range(5):
                    torch.mm(m, m, out=busy)
            got = call(stream=side)[n]                   # the other results and the workspace are dropped
            junk = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(2)]
            torch.cuda.current_stream().wait_stream(side)
            kept = got.clone()
            del got                                      # .. and so is this one while the current stream still reads it
            with torch.cuda.stream(side):
                over = [torch.full((size,), 9, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(2)]
            torch.cuda.synchronize()
            assert torch.equal(kept, want[n]), n
            assert all((j == 7).all() for j in junk) and all((j == 9).all() for j in over), n
