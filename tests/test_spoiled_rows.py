"""The order of stores in the attention kernels under a mask, read from their assembly.

Where a masked tile holds a value that is not finite, the rows that see it get NaN after the results are written.  In the
kernels of few rows any wave may have written a row that another one spoils: every wave's result has to have landed, and
the waves have to have met, before the first NaN is stored."""
import os
import subprocess

import pytest

from mfma_hazards import functions
from paper_2604_20289_amd import build


def blocks_of(body):
    """Basic blocks [(instructions, successors)] of one kernel's [(line, instruction or label)]."""
    blocks, at = [[]], {}
    for _, text in body:
        if text.endswith(":"):
            if blocks[-1]:
                blocks.append([])
            at[text[:-1]] = len(blocks) - 1
        else:
            blocks[-1].append(text)
            if text.startswith(("s_branch", "s_cbranch", "s_endpgm")):
                blocks.append([])
    out = []
    for i, b in enumerate(blocks):
        end = b[-1].split() if b else ["s_nop"]
        after = [at[end[1]]] if end[0] == "s_branch" or end[0].startswith("s_cbranch") else []
        if end[0] not in ("s_branch", "s_endpgm") and i + 1 < len(blocks):
            after.append(i + 1)
        out.append((b, after))
    return out


def early(body):
    """NaN stores (the kernels store them through generic pointers, results through global ones) that a way from a result's store
    reaches without the wave's wait for its stores and then a barrier."""
    blocks, found = blocks_of(body), set()
    # stores of results on the way: 0 none that another wave could still have under way, 1 landed, 2 not
    worst, todo = [-1] * len(blocks), [(0, 0)]
    while todo:
        i, state = todo.pop()
        if state <= worst[i]:
            continue
        worst[i] = state
        for n, text in enumerate(blocks[i][0]):
            op = text.split()[0]
            if op.startswith("global_store"):
                state = 2
            elif op.startswith("flat_store") and state > 0:
                found.add((i, n, text))
            elif op == "s_waitcnt" and "vmcnt(0)" in text:
                state = min(state, 1)
            elif op == "s_barrier" and state == 1:
                state = 0
        todo += [(j, state) for j in blocks[i][1]]
    return sorted(found)


def test_rows_are_spoiled_after_all_waves_have_written(tmp_path):
    out = str(tmp_path / "branch.s")
    r = subprocess.run([build._hipcc(), *build.COMMON_FLAGS, "-x", "hip", "-S", "--cuda-device-only",
                        os.path.join(build.CSRC, "xc_branch.hip"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = functions(open(out).read(), r"branch_(few|f32)_kernelILi\d+ELb1E")
    assert len(kernels) == 5  # head dims 64 and 128, in float32 32 too
    for name, body in kernels.items():
        bodies = 2 if "few" in name else 1  # of few rows, one of 32 and one of 64
        kinds = 2 if "few" in name else 1   # a row's own result, or that of a piece
        assert sum(t.startswith("flat_store") for _, t in body) == bodies * kinds
        assert early(body) == [], name


RESULT, SPOIL, WAIT, MEET = "global_store_dwordx4 v[0:1], v[2:5], off", "flat_store_dword v[0:1], v2", "s_waitcnt vmcnt(0)", "s_barrier"


@pytest.mark.parametrize("body,count", [
    ([RESULT, SPOIL], 1),
    ([RESULT, WAIT, SPOIL], 1),
    ([RESULT, MEET, SPOIL], 1),
    ([RESULT, MEET, WAIT, SPOIL], 1),
    ([RESULT, WAIT, MEET, SPOIL], 0),
    ([RESULT, WAIT, MEET, RESULT, SPOIL], 1),
    ([RESULT, "s_cbranch_scc1 .LBB0_1", WAIT, MEET, ".LBB0_1:", SPOIL], 1),
    (["s_branch .LBB0_2", ".LBB0_1:", SPOIL, "s_endpgm", ".LBB0_2:", RESULT, "s_branch .LBB0_1"], 1),
])
def test_the_reader(body, count):
    assert len(early(list(enumerate(body)))) == count
