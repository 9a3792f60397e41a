"""The built kernels wait for their matrix products.

A matrix instruction's result is there some wait states after it, and nothing in the machine holds
an instruction that asks for it earlier: the compiler puts enough others, or s_nop, between them.
Where paths of different lengths lead from the product to its use it has counted along the longer
one alone, and the shorter one then reads a register before its last terms are in it: a result that
is off by them, now and then.  So every path of every kernel is walked here, in the machine code
that this repository's build made of its sources.

Wait states: an instruction is one, s_nop n is n + 1.  A product of p passes (of four cycles) needs
p + 4 in the 16-bit formats, p + 2 in fp32, before anything but a product's sum takes it up, as the
compiler has it where no branch lies between."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_27384_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT = {"v_mfma_f32_32x32x16_bf16": 8 + 4, "v_mfma_f32_16x16x32_bf16": 4 + 4,
        "v_mfma_f32_32x32x2_f32": 16 + 2, "v_mfma_f32_16x16x4_f32": 8 + 2}
MEMORY = ("global", "buffer", "flat", "ds", "scratch")


def registers(operand):
    """('v' or 'a', first, last), or None."""
    m = re.match(r"[-|]*([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operand)
    return m and ((m[1], int(m[2]), int(m[3])) if m[2] else (m[1], int(m[4]), int(m[4])))


def overlap(a, b):
    return a and b and a[0] == b[0] and a[1] <= b[2] and b[1] <= a[2]


def kernels(listing):
    """(name, instructions, addresses) of a listing; an instruction: (operation, operands, target)."""
    name, ins, at = None, [], []
    for line in listing:
        text, _, note = line.partition("//")
        if line.startswith("\t") and note:
            op, _, rest = text.strip().partition(" ")
            m = re.search(r"\+0x([0-9a-f]+)>", note)
            ins.append((op, [x.strip() for x in rest.split(",")], int(m[1], 16) if m else 0))
            at.append(int(note.split(":")[0], 16))
        elif line.endswith(">:\n"):
            if name:
                yield name, ins, at
            name, ins, at = line[line.index("<") + 1:-3], [], []
    if name:
        yield name, ins, at


def early(ins, at):
    """The products' results that some path takes up too early: (product, user, wait states short)."""
    where = {a - at[0]: i for i, a in enumerate(at)}
    found = []
    for i, (op, a, _) in enumerate(ins):
        if not op.startswith("v_mfma"):
            continue
        result, best, work = registers(a[0]), {}, [(i + 1, 0)]
        while work:
            j, waited = work.pop()
            if j >= len(ins) or waited >= WAIT[op] or best.get(j, 99) <= waited:
                continue
            best[j] = waited
            op2, b, target = ins[j]
            used = []
            if op2.startswith("v_mfma"):
                used = [x for x in b[1:3] if overlap(registers(x), result)]
                used += [x for x in b[3:4] if overlap(registers(x), result) and registers(x) != result]
                if registers(b[0]) == result and not used:
                    continue  # goes on with the sum, or begins another: that one's wait counts
            elif op2.startswith("v_") or op2.startswith(MEMORY):
                used = [x for x in b if overlap(registers(x), result)]
            if used:
                found.append((i, j, WAIT[op] - waited))
            if op2 == "s_endpgm":
                continue
            if op2 == "s_branch" or op2.startswith("s_cbranch"):
                work.append((where[target], waited + 1))
            if op2 != "s_branch":
                work.append((j + 1, waited + (1 + int(b[0], 0) if op2 == "s_nop" else 1)))
    return found


def listing(lines):
    """A listing of these instructions, four bytes each; '-> n' names a branch's target."""
    out = ["0000000000001000 <kernel>:\n"]
    for i, x in enumerate(lines):
        text, _, target = x.partition("->")
        out.append("\t%s // %012X: 0 %s\n" % (text, 0x1000 + 4 * i, "<kernel+0x%x>" % (4 * int(target)) if target else ""))
    return out


@pytest.mark.parametrize("between,short", [
    (["s_nop 11"], 0), (["s_nop 10"], 1), (["s_nop 3", "s_nop 6"], 1),
    (["s_cbranch_execz 3 -> 4"] + ["s_nop 0"] * 2 + ["s_nop 9"], 1),   # the taken path is the short one
    (["s_cbranch_execz 1 -> 3", "s_branch 0 -> 3", "s_nop 9"], 1),
    (["v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], v[44:47], v[0:15]", "s_nop 9"], 2),
    (["v_mfma_f32_32x32x16_bf16 v[16:31], v[0:3], v[44:47], v[16:31]", "s_nop 11"], 12)])
def test_paths_are_walked(between, short):
    lines = ["v_mfma_f32_32x32x16_bf16 v[0:15], v[40:43], v[44:47], 0", *between, "v_add_f32_e32 v50, v51, v7", "s_endpgm"]
    (name, ins, at), = kernels(listing(lines))
    assert name == "kernel" and max((x for _, _, x in early(ins, at)), default=0) == short


def code(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    if not os.path.exists(build.OUT):
        build.build()
    lib = shutil.copy(build.OUT, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, timeout=60)
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950"):
            with subprocess.Popen([OBJDUMP, "-d", os.path.join(tmp_path, f)], stdout=subprocess.PIPE, text=True) as p:
                yield from kernels(p.stdout)


def test_every_product_is_waited_for(tmp_path):
    products = 0
    for name, ins, at in code(tmp_path):
        products += sum(op.startswith("v_mfma") for op, _, _ in ins)
        assert not [(ins[i][:2], ins[j][:2], "%#x" % at[j], short) for i, j, short in early(ins, at)], name
    assert products > 10000
