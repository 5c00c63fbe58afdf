"""Operands that lie side by side in one buffer, or in place where that is allowed, are taken as they are; ones that overlap are refused."""
import pytest
import torch

import operator_probes as probes
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_a_product_beside_its_input(pat, m):
    k, n = 256, 272
    w = probes.integers(n, k, 1, DEV)
    pw = pat.pat_op_f8_pack_weight(w)
    x = probes.integers(m, k, 2, DEV)
    for first, to in ((0, k), (n, 0)):                         # x then y in each row, and the other way round
        buf = torch.zeros(m, k + n, device=DEV)
        buf[:, first:first + k] = x
        pat.pat_op_f8_gemm(*pw, n, buf[:, first:first + k], buf[:, to:to + n])
        assert torch.equal(buf[:, to:to + n].double(), probes.project(x, w)) and torch.equal(buf[:, first:first + k], x)
    rows = torch.zeros(2 * m, k + n, device=DEV)               # y's rows behind all of x's
    rows[:m, :k] = x
    pat.pat_op_f8_gemm(*pw, n, rows[:m, :k], rows[m:, :n])
    assert torch.equal(rows[m:, :n].double(), probes.project(x, w))


@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_a_product_over_its_input_is_refused(pat, m):
    w = torch.ones(256, 256, device=DEV)
    pw = pat.pat_op_f8_pack_weight(w)
    x = torch.ones(m, 512, device=DEV)
    for y in (x[:, :256], x[:, 255:511]):
        for mode in (0, 1):
            with pytest.raises(pat.PatError):
                pat.pat_op_f8_gemm(*pw, 256, x[:, :256], y, mode)
    assert bool((x == 1).all())


@pytest.mark.parametrize("rows", [1, 3])
def test_rotated_queries_over_other_rows_are_refused_and_beside_them_are_not(pat, rows):
    hq, hkv, d = 4, 2, 64
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)      # noqa: E731
    k = torch.zeros(rows, hkv, 16, d, dtype=torch.bfloat16, device=DEV)
    v, cs = k.clone(), pat.pat_op_rope_table(16, d, device=DEV)
    seq, pos, table = i(*range(rows)), i(*range(rows)), i(*range(rows)).view(rows, 1)
    wide = torch.randn(rows, 12, d, device=DEV)
    qkv, want = wide[:, :8].reshape(rows, 8 * d).clone(), torch.empty(rows, hq, d, device=DEV)
    pat.pat_op_kv_append(qkv, seq, pos, cs, k, v, table, want)
    whole = wide.view(rows, 12 * d)
    with pytest.raises(pat.PatError):
        pat.pat_op_kv_append(whole[:, :8 * d], seq, pos, cs, k, v, table, wide[:, 7:11])
    with pytest.raises(pat.PatError):
        pat.pat_op_kv_append(whole[:, :8 * d], seq, pos, cs, k, v, table, wide[:, 1:5])
    got = pat.pat_op_kv_append(whole[:, :8 * d], seq, pos, cs, k, v, table, wide[:, 8:])
    assert torch.equal(got, want) and torch.equal(whole[:, :8 * d], qkv)
    got = pat.pat_op_kv_append(whole[:, :8 * d], seq, pos, cs, k, v, table, wide[:, :hq])
    assert torch.equal(got, want)
