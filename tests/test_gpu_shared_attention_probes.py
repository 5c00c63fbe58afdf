"""Decode attention over shared prefixes on keys and values by which a single key, tile or page that is left out, taken twice or read from elsewhere shows, however long the sequences."""
import numpy as np
import pytest
import torch

import operator_probes as probes
from gpu_util import DEV

pytestmark = pytest.mark.gpu

# groups, query heads, KV heads, features, tokens of a page
CASES = [
    ([(41, [50, 43, 60]), (0, [7]), (33, [33, 34])], 4, 4, 64, 16),
    ([(0, [30000])] + [(0, [1])] * 2000 + [(12000, [12000, 12001])], 1, 1, 64, 16),      # a wave walks more than 32 tiles, and looks its pages up anew
    ([(20000, [27000, 20001, 23500]), (0, [7000])], 2, 2, 128, 64),
    ([(9000, [11500, 9001, 10250])], 8, 1, 128, 64),
    ([(5000, [5900, 5001, 5450]), (0, [900])], 8, 8, 128, 128),
    ([(700, [720 + i for i in range(9)])], 40, 1, 64, 32),
    ([(3000, [16384, 3100]), (0, [9001])], 4, 4, 128, 64),
]


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


@pytest.fixture(scope="module", params=range(len(CASES)))
def case(pat, request):
    groups, hq, hkv, d, P = CASES[request.param]
    c = probes.Cache(groups, hkv, d, P, request.param)
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)      # noqa: E731
    plan = pat.pat_op_attn_plan(i32(c.lens), i32(c.start), i32(c.shared), max(c.lens), hq, hkv, d)
    c.k, c.v, table = c.k.to(DEV), c.v.to(DEV), i32(c.table)
    return c, hq, d, lambda q: pat.pat_op_attn_shared(q.to(DEV), c.k, c.v, table, plan).cpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_all_keys_weigh_the_same(case, dtype):
    c, hq, d, run = case
    got = run(torch.zeros(len(c.lens), hq, d, dtype=dtype))
    for s in sorted({*range(min(40, len(c.lens))), *range(max(0, len(c.lens) - 3), len(c.lens))}):
        assert probes.mean_ok(got[s], probes.mean(c.kv[s][1], hq)), s


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_key_weighs_all(case, dtype):
    """A position of each sequence and head, spread over the sequence's whole length by twelve calls."""
    c, hq, d, run = case
    calls, rng = 12, np.random.default_rng(1)
    seqs = sorted({*range(min(10, len(c.lens))), *range(max(0, len(c.lens) - 2), len(c.lens))})
    order = {s: rng.permutation(calls * hq) for s in seqs}
    for i in range(calls):
        q, at = torch.zeros(len(c.lens), hq, d), {}
        for s in seqs:
            n = c.lens[s]
            at[s] = [min(n - 1, int((int(order[s][i * hq + h]) + rng.random()) * n / (calls * hq))) for h in range(hq)]
            assert probes.alone(c.kv[s][0], at[s], hq)
            q[s] = probes.peaked(c.kv[s][0], at[s], hq)
        got = run(q.to(dtype))
        for s in seqs:
            assert probes.peak_ok(got[s], c.kv[s][1], at[s]), (i, s, at[s])


@pytest.mark.parametrize("shared", [0, 300])
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 64), (16, 1, 64), (4, 4, 64), (3, 3, 64)])
def test_fp32_weights_and_queries_keep_all_their_bits(pat, hq, hkv, d, shared):
    """fp32 results are of weights and queries in three bf16 terms, which are all of them."""
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device=DEV)      # noqa: E731
    P, seqs, groups = 64, 6, [0, 3, 6]
    q = torch.stack([probes.queries(hq, d, s) for s in range(seqs)])
    score = q[..., 0].double() / d ** 0.5
    for n in (500, 1):
        per = -(-(n + 1) // P)
        k = torch.zeros(2 * per, hkv, P, d, dtype=torch.bfloat16)
        v = torch.ones_like(k)
        at = min(n, 2)                                         # the key that has a score
        k[::per, :, at, 0], v[::per, :, at] = 1, 0
        table = i32([[g * per + p for p in range(per)] for g in range(2) for _ in range(3)])
        plan = pat.pat_op_attn_plan(i32([n + 1] * seqs), i32(groups), i32([min(shared, n)] * 2), n + 1, hq, hkv, d)
        got = pat.pat_op_attn_shared(q.to(DEV), k.to(DEV), v.to(DEV), table, plan).cpu()
        for s in range(seqs):
            for f in (0, d - 1):
                assert (probes.weights_ok(got[s, :, f], n, score[s]) if n > 1 else probes.queries_ok(got[s, :, f], score[s])), (n, s, f)
