"""Decode attention over shared prefixes: what the softmax weights' terms on the matrix cores leave of a bf16 result."""
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def test_bf16_results_are_not_biased(pat):
    """The mean error of 2^22 results of values in [1, 2), whose rounding is the only one that counts: each is off by at most half a step,
    2^-8, to either side alike, so their mean has a standard deviation of 2^-8 / sqrt(3 * 2^22) = 1.1e-6.  Five of them, and 2^-19 for the fp32
    arithmetic of some 40 keys, are 7.4e-6; weights that are cut off after 16 bits beside a sum of whole ones leave the results 0.9e-5 short."""
    n, hq, d, P, shared, own, members = 2048, 16, 128, 16, 24, 17, 8
    g = torch.Generator().manual_seed(1)
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)      # noqa: E731
    length, groups, per = shared + own, n // members, -(-(shared + own) // P)
    n_pages = groups + n * (per - 1)                           # the prefix fills one page whole, and a part of each sequence's second
    k = torch.randn(n_pages, hq, P, d, generator=g).to(torch.bfloat16).to(DEV)
    v = (1 + torch.rand(n_pages, hq, P, d, generator=g)).to(torch.bfloat16).clamp(max=2 - 2.0 ** -7).to(DEV)
    table = torch.empty(n, per, dtype=torch.int64)
    table[:, 0] = torch.arange(n) // members
    table[:, 1:] = groups + torch.arange(n * (per - 1)).view(n, per - 1)
    rest = shared - P
    first = table[::members, 1].repeat_interleave(members).to(DEV)
    for t in (k, v):
        t[table[:, 1].to(DEV), :, :rest] = t[first, :, :rest]
    q = torch.randn(n, hq, d, generator=g).to(torch.bfloat16).to(DEV)
    plan = pat.pat_op_attn_plan(i32([length] * n), i32(range(0, n + 1, members)), i32([shared] * groups), length, hq, hq, d)
    got = pat.pat_op_attn_shared(q, k, v, i32(table), plan)
    total = 0.0
    for s in range(0, n, 64):                                  # keys and values of 64 sequences at a time, in 64 bits
        ks, vs = (t[table[s:s + 64].to(DEV)].transpose(2, 3).reshape(64, per * P, hq, d)[:, :length].double() for t in (k, v))
        p = torch.softmax((ks * q[s:s + 64, None].double()).sum(-1) / math.sqrt(d), 1)
        total += float((got[s:s + 64].double() - (p[..., None] * vs).sum(1)).sum())
    mean = total / got.numel()
    assert got.numel() == 1 << 22 and abs(mean) <= 5 * 2.0 ** -8 / math.sqrt(3 * got.numel()) + 2.0 ** -19, mean
