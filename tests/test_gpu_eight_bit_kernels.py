"""Every kernel of the 8-bit projections on integers, whose fp32 sums are exact in any order: long products held to their last bits."""
import pytest
import torch

import operator_probes as probes
from f8_shapes import BF16, F32, STREAM, TILES_OF
from gpu_util import DEV

pytestmark = pytest.mark.gpu
TYPE = {F32: torch.float32, BF16: torch.bfloat16}


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def _check(pat, n, k, m, x_type, y_type):
    x, w = probes.integers(m, k, 1, DEV), probes.integers(n, k, 2, DEV)
    ref = probes.project(x, w)
    pw = pat.pat_op_f8_pack_weight(w.to(torch.bfloat16))
    got = pat.pat_op_f8_gemm(*pw, n, x.to(TYPE[x_type]), y_dtype=TYPE[y_type])
    assert probes.project_ok(got, ref)
    # rows of y that do not begin at a multiple of 16 bytes, added to
    y = torch.full((m, n + 3), 2.0, dtype=TYPE[y_type], device=DEV)
    pat.pat_op_f8_gemm(*pw, n, x.to(TYPE[x_type]), y[:, 1:n + 1], mode=1)
    assert probes.project_ok(y[:, 1:n + 1], ref + 2) and bool((y[:, 0] == 2).all()) and bool((y[:, n + 1:] == 2).all())


@pytest.mark.parametrize("n,k,m,x_type,y_type", sorted(STREAM))
def test_streaming_products(pat, n, k, m, x_type, y_type):
    _check(pat, n, k, m, x_type, y_type)


@pytest.mark.parametrize("n,k,m,y_type", sorted(TILES_OF))
def test_products_by_tiles(pat, n, k, m, y_type):
    _check(pat, n, k, m, BF16, y_type)


@pytest.mark.parametrize("y_type", [F32, BF16])
@pytest.mark.parametrize("m", [1, 3, 70])
def test_the_longest_sums(pat, m, y_type):
    _check(pat, 500, 28672, m, F32, y_type)


@pytest.mark.parametrize("y_type", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(5, 300, 700), (16, 300, 2500), (40, 300, 700), (64, 6000, 700), (140, 300, 700), (300, 9000, 700)])
def test_scales_of_every_size(pat, m, n, k, y_type):
    """Powers of two on both sides change nothing but the result's exponent, for results of either type."""
    x, w = probes.integers(m, k, 3, DEV), probes.integers(n, k, 4, DEV)
    ref = probes.project(x, w)
    for ex, ew in ((120, -110), (-118, 110), (-60, -45), (50, 45), (100, -20), (-30, 118)):
        y = pat.pat_op_f8_gemm(*pat.pat_op_f8_pack_weight(w * 2.0 ** ew), n, x * 2.0 ** ex, y_dtype=TYPE[y_type])
        got = y.double() * 2.0 ** -(ex + ew)
        assert probes.project_ok(got.to(y.dtype), ref), (ex, ew)
