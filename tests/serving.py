"""Shared by the tests of norms with the rotary append, of attention with sinks
and over shared prefixes: references in 64 bits with their error bounds."""
import math

import torch

from tests.paged import U

U32 = 2.0 ** -24


def masked_reference(b, seen, scale=None):
    """(out, lse, bound of out, bound of lse) of softmax attention in 64 bits over the keys that
    seen(s, positions [rows, 1], keys [tokens]) lets a row see.

    Bounds as those of tests/paged.py: a score is off by (hd + 2) steps of 2^-24 of the sum of its products'
    magnitudes and 4 of its own size (the factor to log2 units); a weight by that twice and 2 steps; sums of n
    terms add n steps, a join of parts 2 more each (at most 64 of them: 128); then the weights' rounding before the
    second product and the output's own, in bf16 2^-8 each."""
    scale = scale or b.hd ** -0.5
    g, u = b.nq // b.nkv, U[b.dtype]
    out = torch.zeros(b.n_rows, b.nq, b.hd, dtype=torch.float64, device="cuda")
    lse = torch.full((b.n_rows, b.nq), -math.inf, dtype=torch.float64, device="cuda")
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    for s, (n, t) in enumerate(zip(b.new, b.total)):
        if n == 0:
            continue
        kk, vv = b.cached(s)
        kk, vv = kk.double().permute(1, 2, 0).contiguous(), vv.double().permute(1, 0, 2).contiguous()
        key = torch.arange(t, device="cuda")
        for r0 in range(0, n, 1024):
            r1 = min(n, r0 + 1024)
            pos = torch.arange(t - n + r0, t - n + r1, device="cuda")[:, None]
            sees = seen(s, pos, key)
            some = sees.any(1)
            rows = slice(b.starts[s] + r0, b.starts[s] + r1)
            for h in range(b.nq):
                q = b.q[rows, h].double()
                sc = torch.where(sees, scale * (q @ kk[h // g]), -math.inf)
                mag = scale * (q.abs() @ kk[h // g].abs())
                delta = ((b.hd + 2) * U32 * torch.where(sees, mag, 0.0)).amax(1) + \
                    4 * U32 * torch.where(sees, sc.abs(), 0.0).amax(1)
                m = torch.where(some, sc.amax(1), 0.0)
                p = (sc - m[:, None]).exp()
                z = p.sum(1)
                w = p / torch.where(some, z, 1.0)[:, None]
                out[rows, h] = w @ vv[h // g]
                rel = 2 * delta + (t + 132) * U32 + u * (1 if b.dtype == torch.bfloat16 else 0)
                bo[rows, h] = (w @ vv[h // g].abs()) * (rel[:, None] + u) * (1 + 2.0 ** -6)
                lse[rows, h] = torch.where(some, m + z.log(), -math.inf)
                bl[rows, h] = delta + (t + 132) * U32 + 4 * U32 * torch.where(some, lse[rows, h].abs(), 0.0)
    return out, lse, bo, bl


def sink_mask(window, sinks):
    """Which keys a row sees in a window besides the first keys."""
    def seen(s, pos, key):
        near = key > pos - window if window else key >= 0
        return (key <= pos) & (near | (key < sinks))
    return seen


def normed(x, gain, eps):
    """(x g / sqrt(mean x^2 + eps) in 64 bits, bound of its error in fp32): a sum of hd squares in any order is off by
    hd + 2 steps of 2^-24 at most, of which the root keeps half; the reciprocal root, mean and products add 8."""
    d = x.double()
    y = d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps) * gain.double()
    return y, y.abs() * (x.shape[-1] / 2 + 9) * U32


def rotated(y, slack, freq, pos, layout, dtype):
    """(normed values y rotated by pos * freq, bound): the angle in half turns is rounded to 24 bits, cosine and sine
    are within 2 steps, products and their sum within one each: 2^-21 of the pair's magnitudes; then the storage type."""
    r = 2 * len(freq)
    out, bound = y.clone(), slack.clone()
    if r:
        a = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
        i0 = torch.arange(r // 2, device="cuda") * (2 if layout == "interleaved" else 1)
        i1 = i0 + (1 if layout == "interleaved" else r // 2)
        p, q = y[..., i0], y[..., i1]
        out[..., i0], out[..., i1] = p * a.cos() - q * a.sin(), q * a.cos() + p * a.sin()
        bound[..., i0] = bound[..., i1] = slack[..., i0] + slack[..., i1] + 2.0 ** -21 * (p.abs() + q.abs())
    return out, bound + U[dtype] * (out.abs() + bound)
