"""A sequence model of schedules built from the library's sequence operators.

Every candidate schedule is a sequence of actions.  One layer mixes each sequence along its steps (short
causal convolution, then a selective state-space scan whose step sizes and input/output rows are
projections of the convolution's output), then every step looks at the encoded tokens of its
program (cross attention; all candidates of a program share its keys and values), and a linear
head predicts the latent state after the step.

The example trains the layer on synthetic targets, all sequences at once, and then rolls the same
candidates out one action at a time (convolution and scan states updated in place, one query per
candidate), which has to give the same predictions.

    python examples/schedule_sequence_model.py
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_09312_amd as wm  # noqa: E402


class Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, off, T):
        ctx.save_for_backward(x, w, b, off)
        ctx.T = T
        return wm.causal_conv(x, off, w, b, T_max=T)["y"]

    @staticmethod
    def backward(ctx, dy):
        x, w, b, off = ctx.saved_tensors
        g = wm.causal_conv_grad(dy.contiguous(), x, off, w, b, T_max=ctx.T)
        return g["dx"], g["dweight"], g["dbias"], None, None


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, Bm, Cm, D, z, bias, off, T):
        f = wm.selective_scan(u, delta, A, Bm, Cm, off, T_max=T, D=D, z=z, delta_bias=bias, need_checkpoints=True)
        ctx.save_for_backward(u, delta, A, Bm, Cm, D, z, bias, off, f["checkpoints"])
        ctx.T = T
        return f["y"]

    @staticmethod
    def backward(ctx, dy):
        u, delta, A, Bm, Cm, D, z, bias, off, kept = ctx.saved_tensors
        g = wm.selective_scan_grad(dy.contiguous(), u, delta, A, Bm, Cm, off, kept, T_max=ctx.T, D=D, z=z, delta_bias=bias)
        return g["du"], g["ddelta"], g["dA"], g["dB"], g["dC"], g["dD"], g["dz"], g["ddelta_bias"], None, None


class CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_off, k_off):
        f = wm.cross_attention(q, k, v, q_off, k_off, need_lse=True)
        ctx.save_for_backward(q, k, v, f["o"], f["lse"])
        ctx.off = q_off, k_off
        return f["o"]

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        g = wm.cross_attention_grad(do.contiguous(), q, k, v, o, lse, *ctx.off)
        return g["dq"], g["dk"], g["dv"], None, None


class Layer(torch.nn.Module):
    """Conv, scan and cross attention over packed rows (width d, inner width 2 d)."""

    def __init__(self, d, tokens_d, heads=4, kv_heads=2, head_dim=32, states=16, taps=4, dtype=torch.float32):
        super().__init__()
        self.inner, self.states, self.heads, self.kv_heads, self.head_dim = 2 * d, states, heads, kv_heads, head_dim
        lin = lambda i, o: torch.nn.Parameter((torch.randn(i, o) * i ** -0.5).to(dtype))  # noqa: E731
        f32 = lambda t: torch.nn.Parameter(t.float())  # noqa: E731
        c = self.inner
        self.w_in, self.w_out = lin(d, 2 * c), lin(c, d)
        self.w_sel = lin(c, c + 2 * states)                       # delta, B and C from the convolution's output
        self.conv_w, self.conv_b = f32(torch.randn(c, taps) * taps ** -0.5), f32(torch.zeros(c))
        self.log_a = f32(torch.log(torch.arange(1, states + 1).float()).repeat(c, 1))
        self.D, self.delta_bias = f32(torch.ones(c)), f32(torch.full((c,), -3.0))
        self.w_q, self.w_kv = lin(d, heads * head_dim), lin(tokens_d, 2 * kv_heads * head_dim)
        self.w_o, self.w_head = lin(heads * head_dim, d), lin(d, d)

    def keys(self, tokens):
        kv = (tokens @ self.w_kv).view(-1, 2, self.kv_heads, self.head_dim)
        return kv[:, 0], kv[:, 1]

    def selection(self, u):
        s = u @ self.w_sel
        c, n = self.inner, self.states
        return s[:, :c], s[:, c:c + n], s[:, c + n:]

    def forward(self, x, off, T, tokens, q_off, k_off):
        """All steps at once: x [rows][d] packed by candidate, candidates grouped by program."""
        h = x @ self.w_in
        u = Conv.apply(h[:, :self.inner], self.conv_w, self.conv_b, off, T)
        delta, Bm, Cm = self.selection(u)
        y = Scan.apply(u, delta, -torch.exp(self.log_a), Bm, Cm, self.D, h[:, self.inner:], self.delta_bias, off, T)
        x = x + y @ self.w_out
        k, v = self.keys(tokens)
        o = CrossAttention.apply((x @ self.w_q).view(-1, self.heads, self.head_dim), k, v, q_off, k_off)
        return (x + o.flatten(1) @ self.w_o) @ self.w_head

    @torch.no_grad()
    def start(self, B, tokens, k_off, dev, dtype):
        """State of a rollout of B candidates: convolution inputs, scan states, the programs' keys."""
        return {"conv": torch.zeros((B, self.conv_w.shape[1] - 1, self.inner), dtype=dtype, device=dev),
                "h": torch.zeros((B, self.inner, self.states), device=dev), "kv": self.keys(tokens), "k_off": k_off,
                "A": -torch.exp(self.log_a), "off": torch.arange(B + 1, dtype=torch.int32, device=dev)}

    @torch.no_grad()
    def step(self, x, s, q_off):
        """One action of every candidate: x [B][d]."""
        h = x @ self.w_in
        u = wm.causal_conv(h[:, :self.inner], s["off"], self.conv_w, self.conv_b, T_max=1, state=s["conv"], state_out=s["conv"])["y"]
        delta, Bm, Cm = self.selection(u)
        y = wm.selective_scan(u, delta, s["A"], Bm, Cm, s["off"], T_max=1, D=self.D, z=h[:, self.inner:],
                              delta_bias=self.delta_bias, h0=s["h"], hT=s["h"])["y"]
        x = x + y @ self.w_out
        o = wm.cross_attention((x @ self.w_q).view(-1, self.heads, self.head_dim), *s["kv"], q_off, s["k_off"])["o"]
        return (x + o.flatten(1) @ self.w_o) @ self.w_head


def run(programs=4, per_program=64, T=24, d=64, train_steps=20, dtype=torch.float32, seed=0, log=print):
    """Trains and rolls out; returns the losses and the largest difference of the two ways of running."""
    torch.manual_seed(seed)
    dev = torch.device("cuda")
    r = np.random.default_rng(seed)
    B = programs * per_program
    tok = [int(n) for n in r.integers(40, 200, programs)]
    k_off = np.concatenate([[0], np.cumsum(tok)])
    tokens = torch.randn(int(k_off[-1]), d, device=dev).to(dtype)                # in place of an encoder's token states
    off = torch.arange(0, B * T + 1, T, dtype=torch.int32, device=dev)
    q_off = np.arange(programs + 1) * per_program * T
    x = torch.randn(B * T, d, device=dev).to(dtype)                              # action embeddings
    target = torch.randn(B * T, d, device=dev) * 0.1 + 0.5 * x.float().roll(1, 0)
    layer = Layer(d, d, dtype=dtype).to(dev)
    opt = torch.optim.Adam(layer.parameters(), lr=3e-3)
    losses = []
    for i in range(train_steps):
        p = layer(x, off, T, tokens, q_off, k_off)
        loss = (p.float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
        log(f"step {i}: loss {losses[-1]:.4f}")
    with torch.no_grad():
        whole = layer(x, off, T, tokens, q_off, k_off).view(B, T, d)
    state = layer.start(B, tokens, k_off, dev, dtype)
    rows = np.arange(programs + 1) * per_program
    stepped = torch.stack([layer.step(x.view(B, T, d)[:, t].contiguous(), state, rows) for t in range(T)], 1)
    diff = ((stepped - whole).float().abs().max() / whole.float().abs().max()).item()
    log(f"{B} candidates, {T} actions: one action at a time against all at once, largest difference {diff:.1e}")
    return losses, diff


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--bf16", action="store_true")
    a = ap.parse_args()
    run(train_steps=a.steps, dtype=torch.bfloat16 if a.bf16 else torch.float32)
