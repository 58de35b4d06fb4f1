"""Copies from memory into LDS find their scalar operands written.

Such a copy (global_load_lds) takes its place in LDS from m0.  The hardware does
not hold it back for an m0 written by the instruction right before: one wait state
has to stand between, or the copy may land where the one before it went.  Nor does it hold
back any load for a base address that a vector instruction wrote into scalar
registers less than five wait states earlier.  The compiler puts the waits where it
writes the instructions itself; the copies here are inline assembly, in which it
puts none.  So the assembly of the kernels is checked, the base addresses along every path.
"""
import os
import re
import subprocess

import pytest

from test_matrix_waits import CSRC, HIPCC, functions

BASE_WAIT = 5


def is_copy(op):
    return op is not None and op.startswith("global_load_lds")


def scalars(operand):
    out = set()
    for lo, hi in re.findall(r"\bs\[(\d+):(\d+)\]", operand):
        out |= set(range(int(lo), int(hi) + 1))
    return out | {int(i) for i in re.findall(r"(?<![\w\[])s(\d+)\b", operand)}


def early_copies(code):
    """Copies right behind the write of their m0, and copies from a base that a vector instruction has just written."""
    label = {lab: i for i, (lab, _, _) in enumerate(code) if lab}
    found = []
    for start, (_, op, args) in enumerate(code):
        if op is None or not args:
            continue
        if op.startswith("s_") and args[0] == "m0":
            behind = next((c for c in code[start + 1:] if c[0] is None), None)
            if behind and is_copy(behind[1]):
                found.append((op, behind[1], 0))
        written = scalars(args[0]) if op.startswith("v_") else set()
        if not written:
            continue
        best, todo = {}, [(start + 1, 0, frozenset(written))]
        while todo:
            i, n, live = todo.pop()
            while i < len(code) and n < BASE_WAIT and live and best.get((i, live), 99) > n:
                best[i, live] = n
                lab, o, a = code[i]
                i += 1
                if lab:
                    continue
                if o == "s_endpgm":
                    break
                if o == "s_nop":
                    n += int(a[0])
                elif o == "s_branch":
                    i = label[a[0]]
                elif o.startswith("s_cbranch"):
                    todo.append((label[a[0]], n + 1, live))
                elif is_copy(o):
                    if set().union(*map(scalars, a)) & live:
                        found.append((op, o, n))
                        break
                elif o.startswith("s_") and a:
                    live -= scalars(a[0])
                n += 1
    return found


def test_the_check_sees_an_early_copy():
    text = """_Zf:
\tv_readfirstlane_b32 s5, v9
\ts_cbranch_scc1 .LBB0_1
\ts_nop 7
.LBB0_1:
\ts_mov_b32 m0, s8
\tglobal_load_lds_dwordx4 v0, s[4:5]
.Lfunc_end0:
"""
    (code,) = functions(text).values()
    assert sorted(early_copies(code)) == [("s_mov_b32", "global_load_lds_dwordx4", 0),
                                          ("v_readfirstlane_b32", "global_load_lds_dwordx4", 2)]
    (code,) = functions(text.replace("m0, s8", "m0, s8\n\ts_nop 2")).values()
    assert early_copies(code) == []
    (code,) = functions(text.replace("m0, s8", "m0, s8\n\ts_add_u32 s5, s6, s7")).values()
    assert early_copies(code) == []


@pytest.mark.skipif(HIPCC is None, reason="needs hipcc")
@pytest.mark.parametrize("source", ["paged_attention.hip", "gemm.hip"])
def test_no_copy_is_early(source, tmp_path):
    from paper_2606_12243_amd import build
    asm = tmp_path / "out.s"
    cmd = [HIPCC, *build.FLAGS, "-x", "hip", "--cuda-device-only", "-S", os.path.join(CSRC, source), "-o", str(asm)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = functions(asm.read_text())
    assert any(is_copy(op) for c in kernels.values() for _, op, _ in c)
    # nothing else in these kernels uses m0
    for name, c in kernels.items():
        if any(is_copy(op) for _, op, _ in c):
            used = {(op, a[0]) for _, op, a in c if op is not None and "m0" in a}
            assert used == {("s_mov_b32", "m0")}, name
    assert {name: e for name, e in ((n, early_copies(c)) for n, c in kernels.items()) if e} == {}
