"""Results that would overwrite rows which other workgroups still read are refused before anything reaches a GPU: no pointer here is ever followed."""
import os
import shutil
import subprocess

import pytest

import paper_2605_23945_amd as pat
from paper_2605_23945_amd._build import CSRC
from test_operator_refusals import APPEND, EINVAL, GEMM, P
from test_operator_refusals import test_append_refuses as append_refuses
from test_operator_refusals import test_product_refuses as product_refuses

FAR = P + (1 << 24)

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "row_overlap.h"
// every placing of two operands' rows in one buffer, against its bytes
int main()
{
    const int cases[][5] = {{1, 4, 4, 4, 4}, {3, 4, 12, 4, 12}, {3, 4, 12, 8, 12}, {4, 2, 6, 2, 6}, {3, 4, 12, 3, 5}, {5, 1, 3, 2, 7}, {2, 8, 8, 8, 16}, {2, 8, 16, 8, 16}, {5, 3, 7, 2, 7}, {1, 3, 9, 5, 9}, {6, 1, 9, 1, 4}, {6, 3, 4, 1, 11}};
    long yes = 0, no = 0;
    for (auto &c : cases) {
        const int m = c[0], wa = c[1], la = c[2], wb = c[3], lb = c[4], at = 200;
        for (int off = -lb * m - 4; off <= la * m + 4; ++off) {
            std::vector<char> mine(500, 0);
            bool want = false;
            for (int i = 0; i < m; ++i) for (int o = 0; o < wa; ++o) mine[at + i * la + o] = 1;
            for (int i = 0; i < m; ++i) for (int o = 0; o < wb; ++o) want = want || mine[at + off + i * lb + o];
            if (pat::rows_overlap(&mine[at], la, wa, &mine[at + off], lb, wb, m) != want) { printf("%d %d %d %d %d at %d\n", m, wa, la, wb, lb, off); return 1; }
            ++(want ? yes : no);
        }
    }
    printf("%ld %ld\n", yes, no);
    return 0;
}
"""


@pytest.fixture(scope="module")
def lib():
    return pat.load_library()


@pytest.mark.skipif(not shutil.which("g++"), reason="no g++")
def test_overlaps_are_found_byte_for_byte(tmp_path):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + CSRC, str(src), "-o", str(exe)], check=True, timeout=120)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
    yes, no = map(int, r.stdout.split())
    assert yes > 100 and no > 100


@pytest.mark.skipif(not shutil.which("g++"), reason="no g++")
def test_rows_side_by_side_are_told_apart_at_once(tmp_path):
    """2^19 rows of x and y in one buffer, a thousand times: a walk over the rows would take seconds."""
    src, exe = tmp_path / "many.cpp", tmp_path / "many"
    src.write_text(r"""
#include "row_overlap.h"
int main()
{
    const char *p = reinterpret_cast<const char *>(0x100000);
    int found = 0;
    for (int i = 0; i < 1000; ++i) found += pat::rows_overlap(p, 4096, 1024, p + 1024 + i, 4096, 2048, 1 << 19);
    return found;
}
""")
    subprocess.run(["g++", "-std=c++17", "-O0", "-I" + CSRC, str(src), "-o", str(exe)], check=True, timeout=120)
    assert subprocess.run([str(exe)], timeout=2).returncode == 0


# x is 4 rows of 256 bf16 at P, y 4 rows of 32 fp32
@pytest.mark.parametrize("bad", [dict(), dict(y=P + 4 * 512 - 4), dict(y=P + 512, ldy=128), dict(y=P - 4 * 128 + 4), dict(n=256, k=256, ldy=256, y_type=1), dict(ldx=512, y=P + 508, ldy=256),
                                 dict(mode=1), dict(m=70), dict(m=70, y=P + 70 * 512 - 4)])
def test_product_refuses_a_result_over_its_input(lib, bad):
    assert lib.pat_op_f8_gemm(*dict(GEMM, **bad).values()) == EINVAL


# qkv is 3 rows of 12 heads of 64 fp32 features at P; in place means the same rows
@pytest.mark.parametrize("bad", [dict(ldq=4 * 64), dict(q=P + 64 * 4, ldq=12 * 64), dict(q=P + 11 * 64 * 4, ldq=12 * 64), dict(q=P - 64 * 4, ldq=12 * 64), dict(q=P + 3 * 12 * 64 * 4 - 16), dict(rows=1, q=P + 256),
                                 dict(q=P + 8 * 64 * 4, ldq=16 * 64)])
def test_append_refuses_a_result_over_other_rows(lib, bad):
    assert lib.pat_op_kv_append(*{**APPEND, "rows": 3, **bad}.values()) == EINVAL


@pytest.mark.parametrize("bad", append_refuses.pytestmark[0].args[1])
def test_append_refuses_the_same_apart(lib, bad):
    bad = {k: v + FAR - P if k == "q" and v else v for k, v in bad.items()}
    assert lib.pat_op_kv_append(*{**APPEND, "rows": 1, "q": FAR, **bad}.values()) == EINVAL


@pytest.mark.parametrize("bad", product_refuses.pytestmark[0].args[1])
def test_product_refuses_the_same_apart(lib, bad):
    bad = {k: v + FAR - P if k == "y" and v else v for k, v in bad.items()}
    assert lib.pat_op_f8_gemm(*{**GEMM, "y": FAR, **bad}.values()) == EINVAL
