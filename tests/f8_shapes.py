"""Products that reach every kernel of the 8-bit projections, each with the kernel it is meant for.  test_eight_bit_kernels.py holds them against the rule, the GPU tests run them."""
import ctypes

F32, BF16 = 0, 1
RAW, PACKED, TILES = 0, 1, 2

# the streaming products (up to 64 rows): 1, 2 or 3 weight tiles of 16 a workgroup by n; k ends inside a block of 128 columns, and in all but one each of the
# eight waves turns its ring of blocks
_N = {1: 1000, 2: 6001, 3: 12304}
_RAW = [(1, 9900, F32), (2, 5001, F32), (5, 5001, BF16), (16, 1000, F32), (16, 2000, BF16)]      # rows, k, x's type
_PACKED = [(16, 4001, F32), (16, 4001, BF16), (27, 3333, F32), (40, 3333, BF16), (64, 3333, F32), (64, 3333, BF16)]


def _stream():
    out = {}
    for kind, cases in ((RAW, _RAW), (PACKED, _PACKED)):
        for m, k, x in cases:
            for tiles, n in _N.items():
                for y in (F32, BF16):
                    mb = (m + 15) // 16
                    out[(n, k, m, x, y)] = (kind, 2 if (tiles, mb, y) == (3, 4, F32) else tiles, mb, 8, 1)
    return out


# above 64 rows: n, k, m, type of y -> weight tiles, waves, cuts of k
TILES_OF = {
    (385, 1266, 260, F32): (4, 4, 1), (16, 8800, 66, F32): (4, 4, 6), (2700, 2604, 148, F32): (4, 4, 2),
    (385, 1328, 67, BF16): (4, 4, 1), (16, 8800, 66, BF16): (4, 4, 6),
    (8205, 1268, 130, BF16): (8, 4, 1), (2720, 5973, 134, BF16): (8, 4, 4), (800, 10485, 2765, BF16): (8, 8, 3),
    (16535, 1282, 133, BF16): (12, 4, 1), (6699, 8760, 68, BF16): (12, 4, 6),
    (25439, 1265, 130, BF16): (8, 8, 1), (6243, 9739, 130, BF16): (8, 8, 5), (4548, 9196, 425, BF16): (12, 4, 2),
    (22334, 1313, 258, BF16): (12, 8, 1), (8607, 9321, 130, BF16): (12, 8, 5), (2209, 10483, 482, BF16): (8, 4, 3),
}
STREAM = _stream()


def plan(lib, n, k, m, x, y):
    p = (ctypes.c_int32 * 5)()
    assert lib.pat_op_f8_gemm_plan(n, k, m, x, y, p) == 0
    return tuple(p)
