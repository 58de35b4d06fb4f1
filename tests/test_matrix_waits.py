"""The paged-cache kernels read no matrix result before it is written.

The hardware does not stop a vector instruction that reads a matrix instruction's
destination too early; the compiler has to put enough instructions between.  It
has been seen to count too few where the read is in another basic block (a
branch around the masks), which gave one wrong score.  So the assembly of
the kernels is checked along every path: from each matrix instruction to the
first read of its destination by another than a chained matrix instruction.
"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_12243_amd", "csrc")
HIPCC = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")

# wait states from a matrix instruction to a read of its result (8 and 16 passes; fp64)
WAIT = {"v_mfma_f32_32x32x16_bf16": 11, "v_mfma_f32_32x32x2_f32": 18, "v_mfma_f32_16x16x4_f32": 10,
        "v_mfma_f64_16x16x4_f64": 19}
STORES = ("ds_write", "global_store", "buffer_store", "scratch_store", "flat_store")


def registers(operand):
    out = set()
    for kind, lo, hi in re.findall(r"\b([va])\[(\d+):(\d+)\]", operand):
        out |= {(kind, i) for i in range(int(lo), int(hi) + 1)}
    for kind, i in re.findall(r"(?<![\w\[])([va])(\d+)\b", operand):
        out.add((kind, int(i)))
    return out


def functions(text):
    """Instructions and labels of every function of an assembly file."""
    out, code = {}, None
    for line in text.splitlines():
        m = re.match(r"^(_Z\w+):", line)
        if m:
            code = out.setdefault(m[1], [])
        elif code is not None and line.startswith(".Lfunc_end"):
            code = None
        elif code is not None:
            m = re.match(r"^(\.LBB\w+):", line)
            ins = line.split(";")[0].strip()
            if m:
                code.append((m[1], None, []))
            elif ins and not ins.startswith("."):
                op, _, rest = ins.partition(" ")
                code.append((None, op, [a.strip() for a in rest.split(",")] if rest else []))
    return out


def early_reads(code):
    """Reads of a matrix instruction's destination before its wait states have passed."""
    label = {lab: i for i, (lab, _, _) in enumerate(code) if lab}
    found = []
    for start, (_, mfma, args) in enumerate(code):
        if mfma is None or not mfma.startswith("v_mfma"):
            continue
        assert mfma in WAIT, f"no wait states known for {mfma}"
        best, todo = {}, [(start + 1, 0, frozenset(registers(args[0])))]
        while todo:
            i, n, live = todo.pop()
            while i < len(code) and n < WAIT[mfma] and live and best.get((i, live), 99) > n:
                best[i, live] = n
                lab, op, a = code[i]
                i += 1
                if lab:
                    continue
                if op == "s_endpgm":
                    break
                if op == "s_nop":
                    n += int(a[0])
                elif op == "s_branch":
                    i = label[a[0]]
                elif op.startswith("s_cbranch"):
                    todo.append((label[a[0]], n + 1, live))
                elif op.startswith("v_mfma"):
                    if set().union(*map(registers, a[1:3])) & live:
                        found.append((mfma, op, n))
                        break
                    live -= registers(a[0])  # (a chained one takes over)
                elif op[0] in "vdgbf":
                    store = op.startswith(STORES)
                    if set().union(set(), *map(registers, a if store else a[1:])) & live:
                        found.append((mfma, op, n))
                        break
                    if not store and a:
                        live -= registers(a[0])
                n += 1
    return found


def test_the_check_sees_an_early_read():
    text = """_Zf:
\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], 0
\ts_cbranch_vccz .LBB0_1
\ts_nop 15
.LBB0_1:
\ts_nop 7
\tv_max_f32_e32 v30, v15, v15
.Lfunc_end0:
"""
    (code,) = functions(text).values()
    assert early_reads(code) == [("v_mfma_f32_32x32x16_bf16", "v_max_f32_e32", 9)]
    (code,) = functions(text.replace("s_nop 7", "s_nop 9")).values()
    assert early_reads(code) == []


@pytest.mark.skipif(HIPCC is None, reason="needs hipcc")
@pytest.mark.parametrize("source", ["paged.hip", "paged_attention.hip"])
def test_no_matrix_result_is_read_early(source, tmp_path):
    from paper_2606_12243_amd import build
    asm = tmp_path / "out.s"
    cmd = [HIPCC, *build.FLAGS, "-x", "hip", "--cuda-device-only", "-S", os.path.join(CSRC, source), "-o", str(asm)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels = functions(asm.read_text())
    assert sum(op is not None and op.startswith("v_mfma") for c in kernels.values() for _, op, _ in c) > 0
    assert {name: e for name, e in ((n, early_reads(c)) for n, c in kernels.items()) if e} == {}
