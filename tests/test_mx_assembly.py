"""The 4-bit products' LDS reads written in assembly, in the code that the compiler makes of them.

The kernels keep such reads under way over other work, and the compiler takes their registers for written at once: it may copy one, or give it to
something else, before the data is there.  Nothing at run time shows that reliably, so the compiled code itself is looked at: from every
such read along every path to the next wait for all LDS reads, no instruction may name a register that the read will write.  And
every path from a read has such a wait before the program ends."""
import os
import re
import subprocess

import pytest

from paper_2502_16927_amd import build


def registers(text):
    out = set()
    for m in re.finditer(r"\bv\[(\d+):(\d+)\]", text):
        out |= set(range(int(m.group(1)), int(m.group(2)) + 1))
    return out | {int(m.group(1)) for m in re.finditer(r"\bv(\d+)\b", text)}


def kernels(assembly):
    """{name: ([(instruction, written by hand)], {label: index})} of an assembly file."""
    out = {}
    for m in re.finditer(r"^(_Z\w+kernel\w*):", assembly, re.M):
        body = assembly[m.end():]
        code, labels, by_hand = [], {}, False
        for line in body[:body.index(".Lfunc_end")].split("\n"):
            if "ASMSTART" in line or "ASMEND" in line:
                by_hand = "ASMSTART" in line
                continue
            line = line.split(";")[0].strip()
            if line.endswith(":"):
                labels[line[:-1]] = len(code)
            elif line and not line.startswith("."):
                code.append((line, by_hand))
        out[m.group(1)] = code, labels
    return out


def faults(code, labels):
    """(how many reads by hand, what is wrong with them)."""
    reads, wrong = 0, []
    for i, (read, by_hand) in enumerate(code):
        if not (by_hand and read.startswith("ds_read")):
            continue
        reads += 1
        written = registers(read.split(",")[0])
        seen, todo = set(), [i + 1]
        while todo:
            k = todo.pop()
            if k in seen:
                continue
            seen.add(k)
            line = code[k][0]
            op, _, operands = line.partition(" ")
            if op == "s_waitcnt" and "lgkmcnt(0)" in operands:
                continue
            if op == "s_endpgm":
                wrong.append(f"{i}: {read}: no wait before the end")
                continue
            assert op not in ("s_setpc_b64", "s_swappc_b64"), "calls and returns are not followed"
            if not op.startswith("s_") and registers(operands) & written:
                wrong.append(f"{i}: {read}: touched by {k}: {line}")
                continue
            if op.startswith(("s_branch", "s_cbranch")):
                todo.append(labels[operands.strip()])
            if op != "s_branch":
                todo.append(k + 1)
    return reads, wrong


PLANTED = """
_Z1akernel:
; %bb.0:
	v_mov_b32_e32 v9, 0
.LBB0_1:
	;;#ASMSTART
	ds_read_b128 v[4:7], v9 offset:16
	;;#ASMEND
	v_add_u32_e32 v9, 1, v9
	s_cbranch_scc1 .LBB0_3
; %bb.2:
	{before}
	s_waitcnt lgkmcnt(0)
	v_mov_b32_e32 v8, v5
	s_cbranch_vccnz .LBB0_1
	s_endpgm
.LBB0_3:
	{other}
	s_endpgm
.Lfunc_end0:
"""


@pytest.mark.parametrize("before,other,wrong", [
    ("s_nop 0", "s_waitcnt vmcnt(0) lgkmcnt(0)", 0),
    ("v_mov_b32_e32 v8, v5", "s_waitcnt lgkmcnt(0)", 1),             # read too early
    ("v_mov_b32_e32 v6, 0", "s_waitcnt lgkmcnt(0)", 1),              # given to something else
    ("s_nop 0", "s_waitcnt vmcnt(0)", 1),                            # another wait, on the branch
    ("s_nop 0", "global_store_dwordx4 v[0:1], v[4:7], off", 1),
])
def test_planted_mistakes_are_found(before, other, wrong):
    (code, labels), = kernels(PLANTED.format(before=before, other=other)).values()
    reads, found = faults(code, labels)
    assert reads == 1 and len(found) == wrong, found


def test_registers_of_reads_under_way_are_left_alone(tmp_path):
    out = str(tmp_path / "mx_product.s")
    subprocess.run(["hipcc", *build.FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, "mx_product.hip"), "-o", out], check=True, capture_output=True, timeout=600)
    every = kernels(open(out).read())
    with_reads = 0
    for name, (code, labels) in every.items():
        reads, wrong = faults(code, labels)
        with_reads += reads > 0
        assert not wrong, f"{name}: {wrong[:5]}"
    assert len(every) == 12 and with_reads == 9, "the ring kernels' reads are found"
