"""The 8-bit products of many rows (gemm_f8.hip) wait for a block's weights, which all waves of a workgroup read from LDS, by the number of loads that a wave
has issued since: a number too large by one lets a wave read what has not arrived.  Read from the assembly of the kernels compiled here: their loop is
walked with its loads in order and the waits written in the source alone, without those that the compiler adds for its own loads.  Needs no GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_23945_amd._build import CSRC, FLAGS

HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
KERNELS = {(4, 4, 4, "f"), (4, 4, 4, "t"), (8, 4, 4, "t"), (12, 4, 3, "t"), (8, 8, 4, "t"), (12, 8, 4, "t")}      # weight tiles, waves, stages, result's type


@pytest.fixture(scope="module")
def loops():
    """The loop of every tile kernel, as lines."""
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    r = subprocess.run([HIPCC, *FLAGS, "--cuda-device-only", "-S", "-o", "-", os.path.join(CSRC, "gemm_f8.hip")], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    found = {}
    for m in re.finditer(r"^_ZN\S*14f8_tile_kernelILi(\d+)ELi(\d+)ELi(\d+)E([ft])E\S*:.*?^\.Lfunc_end", r.stdout, flags=re.M | re.S):
        lines = [l.strip() for l in m.group(0).splitlines()]
        labels = {l.split(":")[0]: i for i, l in enumerate(lines) if re.match(r"\.LBB\w+:", l)}
        for i, l in enumerate(lines):
            b = re.match(r"s_cbranch_\w+ (\.LBB\w+)", l)
            if b and labels[b.group(1)] < i:
                body = lines[labels[b.group(1)]:i]
                if sum(x == "s_barrier" for x in body):
                    found[(int(m.group(1)), int(m.group(2)), int(m.group(3)), m.group(4))] = body
    return found


def first_early(body, stages, per_stage, turns=4):
    """The first step at whose barrier the next step's weights may still be under way by the written waits; None: there is none.

    A step ends its reads at a barrier and then requests the weights of `stages` steps on; all loads before the loop have arrived."""
    under_way, requested, step, written = [], 0, 0, False
    for l in body * turns:
        if "ASMSTART" in l or "ASMEND" in l:
            written = "ASMSTART" in l
        elif l.startswith("global_load_lds"):
            under_way.append(requested // per_stage + stages)      # the step that reads it
            requested += 1
        elif re.match(r"(global|buffer|flat|scratch)_(load|store|atomic)", l):
            under_way.append(None)
        elif l.startswith("s_waitcnt") and written:
            n = re.search(r"vmcnt\((\d+)\)", l)
            if n:
                under_way = under_way[max(0, len(under_way) - int(n.group(1))):]
        elif l == "s_barrier":
            if step + 1 in under_way:
                return step
            step += 1
    assert step == 4 * turns and requested == step * per_stage
    return None


def test_every_tile_kernel_is_looked_at(loops):
    assert set(loops) == KERNELS


@pytest.mark.parametrize("kernel", sorted(KERNELS))
def test_weights_have_arrived_by_the_written_waits(loops, kernel):
    tiles, waves, stages, _ = kernel
    assert first_early(loops[kernel], stages, 2 * tiles // waves) is None


def test_a_wait_that_is_one_too_lax_is_found():
    step = ["global_load_dwordx4"] * 4 + [";;#ASMSTART", "s_waitcnt vmcnt(%d)", ";;#ASMEND", "s_barrier"] + ["global_load_lds_dwordx4"] * 2
    body = step * 4                                            # newer than the next step's weights: x of three steps, weights of two
    assert first_early([l % 16 if "%d" in l else l for l in body], 4, 2) is None
    assert first_early([l % 17 if "%d" in l else l for l in body], 4, 2) is not None
