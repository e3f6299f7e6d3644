"""The vocabulary's products issue matrix instructions in inline assembly, where the
compiler does not look after the slots that the hardware wants between them and
the vector unit: two between a vector instruction and the matrix instruction that
reads what it wrote, and the passes of the matrix instruction before its sums are
read.  The source keeps them apart; this reads the gfx950 assembly to see that it
still does.  Runs on the CPU: hipcc cross-compiles."""
import os
import re
import shutil
import subprocess

import pytest

import paper_1601_04033_amd._build as lib_build

REGISTER = re.compile(r"^-?\|?([av])(?:\[(\d+):(\d+)\]|(\d+))\|?$")
SLOTS = 2       # a vector instruction's result, read by a matrix instruction
PASSES = 18     # an upper bound of a matrix instruction's, until its sums may be read


def registers(operand):
    m = REGISTER.match(operand.strip())
    if not m:
        return set()
    low, high = (int(m[2]), int(m[3])) if m[2] else (int(m[4]), int(m[4]))
    return {(m[1], i) for i in range(low, high + 1)}


def parse(text):
    """Functions as lists of ("label", name), ("asm", True / False) and ("op", mnemonic, operands)."""
    functions, body = [], None
    for line in text.splitlines():
        s = line.strip()
        if s.startswith(".type") and s.endswith("@function"):
            body = []
            functions.append(body)
        elif body is None:
            continue
        elif "#ASMSTART" in s or "#ASMEND" in s:
            body.append(("asm", "#ASMSTART" in s))
        elif re.match(r"^[.\w$]+:", s):
            body.append(("label", s.split(":")[0]))
        elif s and s[0] not in ".;":
            name, _, rest = s.split(";")[0].strip().partition(" ")
            body.append(("op", name, re.split(r",\s*(?![^\[]*\])", rest.strip()) if rest else []))
    return functions


def written(name, operands):
    """Registers that a vector instruction (not a matrix one) writes."""
    if not name.startswith("v_") or name.startswith(("v_mfma", "v_cmp", "v_readfirstlane", "v_readlane")):
        return set()
    out = set(registers(operands[0])) if operands else set()
    if "swap" in name:
        out |= registers(operands[1])
    return out


def before(body, at, slots, branches, seen=()):
    """Instructions within `slots` before body[at], along every way that leads there."""
    while slots > 0 and at > 0:
        at -= 1
        kind, *rest = body[at]
        if kind == "label":
            for source in branches.get(rest[0], []):
                if source not in seen:
                    yield from before(body, source + 1, slots, branches, (*seen, source))
        elif kind == "op":
            if rest[0] in ("s_branch", "s_endpgm") and not seen:
                return          # what stands before is not what ran before
            yield rest
            slots -= int(rest[1][0], 0) + 1 if rest[0] == "s_nop" else 1


def check(text):
    """(matrix instructions in inline assembly, faults)"""
    count, faults = 0, []
    for body in parse(text):
        branches = {}
        for at, (kind, *rest) in enumerate(body):
            if kind == "op" and rest[0].startswith(("s_branch", "s_cbranch")):
                branches.setdefault(rest[1][0], []).append(at)
        inline, open_sums, waited = False, set(), 0
        for at, (kind, *rest) in enumerate(body):
            if kind == "asm":
                inline = rest[0]
            if kind != "op":
                continue
            name, operands = rest
            if name.startswith("v_mfma") and inline:
                count += 1
                reads = set().union(*(registers(o) for o in operands[1:4]))
                for other, ops in before(body, at, SLOTS, branches):
                    if written(other, ops) & reads:
                        faults.append((other, ops, name, operands))
                open_sums |= registers(operands[0])
                waited = 0
                continue
            if open_sums:
                touched = set().union(*(registers(o) for o in operands)) if operands else set()
                if waited < PASSES and touched & open_sums and not name.startswith("v_mfma"):
                    faults.append(("sums read early", name, operands))
                waited += int(operands[0], 0) + 1 if name == "s_nop" else 1
                if waited >= PASSES:
                    open_sums = set()
    return count, faults


def test_the_reader_sees_what_it_is_for():
    head = "\t.type\tf,@function\nf:\n"
    asm = "\t;;#ASMSTART\n\tv_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]\n\t;;#ASMEND\n"
    assert check(head + asm) == (1, [])
    for write in ("v_mov_b32_e32 v5, 0", "v_accvgpr_write_b32 a2, 0", "v_permlane32_swap_b32_e32 v1, v9", "v_add_u32_e32 v4, v1, v2"):
        assert len(check(head + f"\t{write}\n" + asm)[1]) == 1
        assert len(check(head + f"\t{write}\n\ts_add_i32 s0, s0, 1\n" + asm)[1]) == 1
        assert not check(head + f"\t{write}\n\ts_nop 1\n" + asm)[1]
        # around a loop
        assert len(check(head + ".L1:\n" + asm + f"\t{write}\n\ts_cbranch_scc1 .L1\n")[1]) >= 1
    assert not check(head + "\tv_mov_b32_e32 v12, 0\n" + asm)[1]
    read = "\tv_accvgpr_read_b32 v0, a1\n"
    assert len(check(head + asm + read)[1]) == 1
    assert len(check(head + asm + "\ts_nop 15\n" + read)[1]) == 1
    assert not check(head + asm + "\ts_nop 15\n\ts_nop 15\n" + read)[1]


@pytest.mark.skipif(shutil.which(lib_build.HIPCC) is None and not os.path.exists(lib_build.HIPCC),
                    reason="hipcc is not installed")
def test_matrix_instructions_of_the_vocabulary(tmp_path):
    out = tmp_path / "vocab_product.s"
    cmd = [lib_build.HIPCC, *lib_build.FLAGS, "-Wno-unused-command-line-argument", "--cuda-device-only", "-S",
           os.path.join(lib_build.CSRC, "vocab_product.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    count, faults = check(out.read_text())
    # two types, five kernels of 256 x 256 each, rounds of five stages of 128 instructions
    assert count >= 2 * 5 * 5 * 128
    assert not faults, faults[:5]
