"""Inputs of the operators of include/pat_operators.h on which every order of fp32 sums gives the same number, so that long results can be held to their last bits: a block
of columns, a tile of keys or one page that a kernel leaves out, takes twice or takes from elsewhere shows however long the sum is."""
from __future__ import annotations

import numpy as np
import torch

BF16_HALF = 2.0 ** -8                                          # half a step of bf16, relative

# ---- projections: x and W hold integers of up to 15, which 4 significant bits hold, whatever the block's largest; products are integers of up to 225 and sums of
# 28672 of them stay below 2^24


def integers(m, k, seed, device="cpu"):
    """fp32 [m, k] of -15 .. 15 without zero."""
    g = torch.Generator(device=device).manual_seed(seed)
    x = torch.randint(1, 16, (m, k), generator=g, device=device, dtype=torch.int32)
    return (x * (1 - 2 * torch.randint(0, 2, (m, k), generator=g, device=device, dtype=torch.int32))).float()


def project(x, w):
    """x W^T in 64 bits; a sum of magnitudes below 2^24 is checked first."""
    assert x.shape[1] * float(x.abs().max()) * float(w.abs().max()) < 2 ** 24
    return x.double() @ w.double().t()


def project_ok(got, ref):
    """fp32: equal.  bf16: within half a step and 5e-5 of a row's norm, which the 8-bit matrix instruction may drop."""
    if got.dtype == torch.float32:
        return bool(torch.equal(got.double(), ref))
    lost = 5e-5 * ref.pow(2).mean(1, keepdim=True).sqrt()
    return bool(((got.double() - ref).abs() <= lost + BF16_HALF * (ref.abs() + lost)).all())


# ---- attention: keys of +-1 and values that are integers of up to 64


class Cache:
    """groups: [(shared tokens, [cached tokens of each sequence, none shorter than that])].  Pages in random order, a prefix's whole ones shared; NaN where nothing lies."""

    def __init__(self, groups, hkv, d, P, seed):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.shared = [n for _, seqs in groups for n in seqs], [s for s, _ in groups]
        self.start = np.concatenate([[0], np.cumsum([len(seqs) for _, seqs in groups])])
        total = sum(s // P for s in self.shared) + sum(-(-n // P) - s // P for s, seqs in groups for n in seqs)
        order, at = np.random.default_rng(seed).permutation(total), 0
        self.table = np.full((len(self.lens), max(-(-n // P) for n in self.lens)), -1, np.int64)
        self.k, self.v = (torch.full((total, hkv, P, d), float("nan"), dtype=torch.bfloat16) for _ in range(2))
        self.kv, s = [], 0
        for shared, seqs in groups:
            whole = order[at:at + shared // P]
            at += len(whole)
            prefix = self._some(g, shared, hkv, d)
            for n in seqs:
                k, v = (torch.cat([a, b]) for a, b in zip(prefix, self._some(g, n - shared, hkv, d)))
                pages = -(-n // P)
                own = order[at:at + pages - len(whole)]
                at += len(own)
                self.table[s, :pages] = np.concatenate([whole, own])
                for pool, t in ((self.k, k), (self.v, v)):
                    full = torch.full((pages * P, hkv, d), float("nan"), dtype=torch.bfloat16)
                    full[:n] = t
                    pool[torch.as_tensor(self.table[s, :pages])] = full.view(pages, P, hkv, d).transpose(1, 2)
                self.kv.append((k, v))
                s += 1

    @staticmethod
    def _some(g, n, hkv, d):
        k = 1 - 2 * torch.randint(0, 2, (n, hkv, d), generator=g)
        v = torch.randint(1, 65, (n, hkv, d), generator=g) * (1 - 2 * torch.randint(0, 2, (n, hkv, d), generator=g))
        return k.to(torch.bfloat16), v.to(torch.bfloat16)


def mean(values, hq):
    """The result for q = 0, where all keys weigh the same: [hq, d] in 64 bits."""
    return values.double().mean(0).repeat_interleave(hq // values.shape[1], 0)


def mean_ok(got, ref):
    """Sums and counts are exact; a reciprocal and a product are rounded, and a bf16 result once more."""
    half = 3 * 2.0 ** -24 + (BF16_HALF * (1 + 2.0 ** -22) if got.dtype == torch.bfloat16 else 0.0)
    return bool(((got.double() - ref).abs() <= half * ref.abs()).all())


PEAK = 16.0


def peaked(keys, at, hq):
    """q [hq, d] of one sequence, head h 16 times its key at[h]: that key's score is 16 sqrt(d).  Another's is 12 sqrt(d) at the most where alone() holds: 30000 of them
    and 64 features weigh 30000 e^-32 = 4e-10 together."""
    G = hq // keys.shape[1]
    return torch.stack([PEAK * keys[at[h], h // G].float() for h in range(hq)])


def alone(keys, at, hq):
    """No other key's product with it is above three quarters of its own."""
    G, d = hq // keys.shape[1], keys.shape[2]
    for h in range(hq):
        same = keys[:, h // G].float() @ keys[at[h], h // G].float()
        same[at[h]] = 0
        if float(same.max()) > d / 2 + d / 4:
            return False
    return True


def peak_ok(got, values, at):
    """The value at the head's key: integers of 7 bits in bf16.  In fp32 the matrix cores may cut off a step of 2^-23 with each of three terms of every tile of 32 keys, whose weights
    are far below a step, 940 tiles at the most: 2^-11.  Values are a 64th of each other apart or more."""
    G = got.shape[0] // values.shape[1]
    ref = torch.stack([values[at[h], h // G] for h in range(got.shape[0])]).double()
    if got.dtype == torch.bfloat16:
        return bool(torch.equal(got.double(), ref))
    return bool(((got.double() - ref).abs() <= 2.0 ** -11 * ref.abs()).all())


# ---- attention's fp32 terms: one feature makes the score, so that nothing is summed


def queries(hq, d, seed):
    """q [hq, d] fp32 whose first feature has all 24 bits and lies between sqrt(d) and 5 sqrt(d): against a key that is 1 there the score is between 1 and 5."""
    q = torch.zeros(hq, d)
    q[:, 0] = (1 + 4 * torch.rand(hq, generator=torch.Generator().manual_seed(seed))) * d ** 0.5
    return q


def weights_ok(got, n, score):
    """One key of that score and value 0, n of score 0 and value 1: n p / (1 + n p) with p = exp(-score).  p is the same above and below, so its own error,
    (score + 3) 2^-22, counts 1 / (1 + n p).  Roundings of half a step, 2^-24, in sums of 500 keys as chunks of 32 a wave: below 8 of a lane, 2 between lanes, 4 between waves,
    8 between parts; above 24 of three products' sums (cut off, four each), 4 between waves, 16 between parts; a reciprocal, a product: 72 at the most."""
    p = torch.exp(-score.double())
    ref = n * p / (1 + n * p)
    return bool(((got.double() - ref).abs() <= ref * (72 * 2.0 ** -24 + (score.double() + 3) * 2.0 ** -22 / (1 + n * p))).all())


def queries_ok(got, score):
    """The same of two keys: p / (1 + p).  The argument of the exponent, of the size of the score, is rounded three times (scale, product, sum), its function to a step;
    16 roundings of half a step in three products' sums, joins and the division."""
    ref = torch.sigmoid(-score.double())
    return bool(((got.double() - ref).abs() <= ref * (16 * 2.0 ** -24 + (score.double() + 3) * 2.0 ** -22)).all())
