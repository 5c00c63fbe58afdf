"""Which kernel an 8-bit projection takes: the shapes of f8_shapes.py reach every one there is.  Needs no GPU."""
import ctypes

import pytest

import paper_2605_23945_amd as pat
from f8_shapes import BF16, F32, PACKED, RAW, STREAM, TILES, TILES_OF, plan


def test_streaming_shapes_reach_every_kernel():
    lib = pat.load_library()
    for shape, want in STREAM.items():
        assert plan(lib, *shape) == want, shape
    seen = {(p[0], p[1], p[2], x if p[0] == RAW else None, y) for (_, _, _, x, y), p in STREAM.items()}
    assert seen == {(RAW, t, 1, x, y) for t in (1, 2, 3) for x in (F32, BF16) for y in (F32, BF16)} | \
        {(PACKED, t, b, None, y) for t in (1, 2, 3) for b in (1, 2, 3, 4) for y in (F32, BF16)} - {(PACKED, 3, 4, None, F32)}


def test_tile_shapes_reach_every_kernel_whole_and_cut():
    lib = pat.load_library()
    for (n, k, m, y), (tiles, waves, cuts) in TILES_OF.items():
        for x in (F32, BF16):
            assert plan(lib, n, k, m, x, y) == (TILES, tiles, 2 * waves, waves, cuts), (n, k, m, y)
    seen = {(t, w, c > 1, y) for (_, _, _, y), (t, w, c) in TILES_OF.items()}
    assert seen == {(t, w, c, BF16) for t, w in ((4, 4), (8, 4), (12, 4), (8, 8), (12, 8)) for c in (False, True)} | {(4, 4, c, F32) for c in (False, True)}


@pytest.mark.parametrize("args", [(0, 64, 4, 0, 0), (64, 0, 4, 0, 0), (64, 64, 0, 0, 0), (64, 64, -1, 0, 0), (64, 64, (1 << 19) + 1, 0, 0), (64, 64, 4, 2, 0), (64, 64, 4, 0, -1),
                                  ((1 << 22) + 1, 64, 4, 0, 0), ((1 << 17) + 1, 64, 1 << 19, 0, 0)])
def test_the_query_refuses_what_the_product_refuses(args):
    lib = pat.load_library()
    assert lib.pat_op_f8_gemm_plan(*args, (ctypes.c_int32 * 5)()) == pat.binding.PAT_EINVAL
    assert lib.pat_op_f8_gemm_plan(64, 64, 4, 0, 0, None) == pat.binding.PAT_EINVAL
