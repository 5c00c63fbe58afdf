"""Plain implementations of the operators of include/pat_operators.h in 64 bits, on the CPU, and the tolerances of their tests.

Tolerances count roundings: half a step is HALF[type] relative to the rounded value; a sum of n products in fp32 is off by at most
n times a step of 2^-23 of the sum of its products' magnitudes (the matrix cores round towards zero at worst, a step instead of half of one)."""
from __future__ import annotations

import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def angles(n_pos, d, base=10000.0):
    j = torch.arange(d // 2, dtype=torch.float64)
    return torch.arange(n_pos, dtype=torch.float64)[:, None] * base ** (-2.0 * j / d)


def rotate(x, pos, base=10000.0):
    """x [rows, heads, d] at positions pos [rows], in 64 bits; and the magnitudes |a| + |b| of each pair."""
    d = x.shape[-1]
    ang = pos.double()[:, None] * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    mag = (a.abs() + b.abs()).repeat(1, 1, 2)
    return torch.cat([a * c - b * s, a * s + b * c], -1), mag


def rms(x, g, eps):
    return x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * g


def attend(q, keys, values):
    """One query [hq, d] over keys, values [n, hkv, d] in 64 bits -> (result [hq, d], allowance [hq, d] of the computation before the last rounding)."""
    hq, d = q.shape
    if keys.shape[0] == 0:
        return torch.zeros(hq, d, dtype=torch.float64), torch.zeros(hq, d, dtype=torch.float64)
    G = hq // keys.shape[1]
    k, v = keys.double().repeat_interleave(G, 1), values.double().repeat_interleave(G, 1)
    prod = k * q.double()
    s = prod.sum(-1) / math.sqrt(d)                                        # [n, hq]
    p = torch.softmax(s, 0)
    out, mag = (p[..., None] * v).sum(0), (p[..., None] * v.abs()).sum(0)
    score = (d + 4) * 2.0 ** -23 * (prod.abs().sum(-1).amax(0) / math.sqrt(d)) + 2.0 ** -20      # of a score: its sum, its scale, the exponent's function
    n = keys.shape[0]
    rel = 2 * score[:, None] + 2.0 ** -15 + 2 * (n + 64) * 2.0 ** -23      # p twice (above and below), its bf16 terms, the sums over keys
    return out, rel * mag


def eight_bit(x, rows):
    """The 8-bit form of x [m, k]: the values, block by block, element by element by definition."""
    x = x.double()
    out = torch.empty_like(x)
    for r in range(0, x.shape[0], rows):
        for c in range(0, x.shape[1], 128):
            b = x[r:r + rows, c:c + 128]
            fin = torch.isfinite(b)
            top = float(b[fin].abs().max()) if bool(fin.any()) else 0.0
            e = 0
            if top > 0:
                e = math.frexp(top / 448.0)[1] - 1
                while 448.0 * 2.0 ** e < top:
                    e += 1
                while 448.0 * 2.0 ** (e - 1) >= top:
                    e -= 1
                e = max(e, -127)
            u = b / 2.0 ** e
            step = 2.0 ** (torch.frexp(u.abs().clamp(min=2.0 ** -6, max=448.0).nan_to_num(1.0))[1] - 1 - 3).double()
            v = torch.round(u / step) * step * 2.0 ** e
            out[r:r + rows, c:c + 128] = torch.where(fin, v, torch.nan)
    return out


def project(xq, wq):
    """(product of the 8-bit forms, allowance of its fp32 sum)."""
    return xq @ wq.t(), xq.shape[1] * 2.0 ** -23 * (xq.abs() @ wq.abs().t())


def check(got, ref, allowance, dtype=None):
    """|got - ref| within the allowance and one rounding to the type."""
    half = HALF[dtype or got.dtype]
    got = got.double().cpu()
    ref, allowance = ref.double().cpu(), allowance.double().cpu()
    assert got.shape == ref.shape
    bad = ~((got - ref).abs() <= allowance + half * (ref.abs() + allowance) + 1e-37)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ref).abs().nan_to_num(1e30).max()):.3g}, first at {bad.nonzero()[0].tolist()}"
