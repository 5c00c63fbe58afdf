"""The largest append: a launch has fewer than 2^32 threads.  No pointer here is ever followed."""
import pytest

import paper_2605_23945_amd as pat
from test_operator_refusals import APPEND, EINVAL, P


@pytest.mark.parametrize("heads,rows", [(3, (1 << 28) // 3), (12, (1 << 28) // 12), (15, (1 << 28) // 15), (12, (1 << 28) // 12 + 1)])
def test_rows_whose_lanes_fill_32_bits_are_refused(heads, rows):
    """fp32 heads of 128 features take 16 lanes: 2^28 - 15 .. 2^28 - 1 of them round up to workgroups of 2^32 lanes."""
    assert rows * heads >= (1 << 28) - 15
    hkv = heads // 3
    a = {**APPEND, "rows": rows, "hq": hkv, "hkv": hkv, "type": 0, "d": 128, "ld": heads * 128, "ldq": hkv * 128, "q": P + (1 << 44)}
    assert pat.load_library().pat_op_kv_append(*a.values()) == EINVAL
