"""Helpers of the tests of the operators over a shared prefix: inputs, and comparison with the float64 oracle.

Comparison: ||g - o||_2 / ||o||_2 over a tensor, and the largest |g - o| against max(|o|, rms(o)).  Tolerances, from
the formats.  A stored bfloat16 value is off by at most half a step, 2^-8 of itself: a rotated or copied row 2^-8.
Attention also rounds the probabilities, and in its gradient the score gradients, to bfloat16 as product
operands, 2^-8 of each at most, in sums whose terms do not cancel them on the whole: 2^-7.  float32 attention: sums of at most a
few thousand products of 2^-24 each, of either sign, and an exponential whose argument (below 40 here) is
rounded to 2^-24 of itself, 40 x 6e-8 = 2.4e-6 at the worst and a tenth of that over a tensor: 2e-6.  float32
rotation: sine and cosine are off by at most 2e-7 (a Horner step at 1 rounds to 2^-24, the angle to 2^-25 of pi / 4, the angle
in 64 bits to 2^-52 of up to 2^24 turns: 4e-9), two products and a sum by 2^-24 each: 4e-7.  Largest elements: 16 times
the 2-norm's (a result can be smaller than what is summed for it), in float32 attention 5e-5.  Results that are 0 by
definition are compared absolutely."""
import numpy as np

ATTN = {"f32": 2e-6, "bf16": 2.0 ** -7}
TURN = {"f32": 4e-7, "bf16": 2.0 ** -8}
LSE = 2e-6


def dt(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def host(t):
    return t.detach().double().cpu().numpy()


def close(name, got, want, tol, spread=None):
    """spread: what a result may be off besides, element by element."""
    g, o = host(got), np.asarray(want, np.float64)
    assert g.shape == o.shape, name
    fin = np.isfinite(o)
    assert np.array_equal(np.isnan(g), np.isnan(o)), f"{name}: NaN in other places"
    inf = np.isinf(o)
    assert (g[inf] == o[inf]).all() and np.isfinite(g[fin]).all(), f"{name}: values that are not finite"
    d = np.abs(g[fin] - o[fin])
    if spread is not None:
        d = np.maximum(d - spread[fin], 0.0)
    norm = np.linalg.norm(o[fin])
    if norm == 0.0:
        assert d.max(initial=0.0) <= tol, f"{name}: {d.max()} for 0"
        return
    rel = np.linalg.norm(d) / norm
    most = (d / np.maximum(norm / np.sqrt(fin.sum()), np.abs(o[fin]))).max()
    assert rel <= tol, f"{name}: relative 2-norm {rel:.2e} > {tol:.2e}"
    assert most <= (5e-5 if ATTN["f32"] <= tol < 2e-5 else 16 * tol), f"{name}: largest {most:.2e}"


def offsets(lens):
    return [0] + [int(x) for x in np.cumsum(lens)]


def frequencies(rot, theta=10000.0):
    import torch
    return (theta ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)).float().cuda()


def i32(a):
    import torch
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


def same_bits(a, b):
    import torch
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


class Pool:
    """A pool of pages in random order with tables for ragged lengths; what no key has is NaN, unused entries -1."""

    def __init__(self, dtype, page, Hk, dh, own, shared=(), seed=0, spare=3, wide=0):
        import torch
        r = np.random.default_rng(seed)
        counts = [-(-n // page) for n in list(own) + list(shared)]
        total = sum(counts) + spare
        order = r.permutation(total).astype(np.int32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((total, Hk, page, dh), generator=g, device="cuda").to(dt(dtype)) for _ in range(2))
        used = np.zeros((total, page), bool)

        def table(lens, cnt, at):
            t = np.full((len(lens), max(cnt, default=0) + wide), -1, np.int32)
            for i, (n, c) in enumerate(zip(lens, cnt)):
                t[i, :c] = order[at:at + c]
                for j in range(n):
                    used[t[i, j // page], j % page] = True
                at += c
            return t, at
        self.pages, at = table(own, counts[:len(own)], 0)
        self.prefix_pages, _ = table(shared, counts[len(own):], at)
        dead = torch.tensor(~used, device="cuda")[:, None, :, None]
        for t in (self.k, self.v):
            t.masked_fill_(dead, float("nan"))
        self.page, self.own, self.shared = page, list(own), list(shared)
