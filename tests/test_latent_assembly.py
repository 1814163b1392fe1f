"""Wait states around the matrix instructions that the latent attention writes as inline assembly, in the assembly that the compiler makes of it.

The compiler keeps the wait states of its own instructions, not those of inline assembly: nothing may touch the result of a matrix instruction written so
too early, what it reads may not have been written by a vector instruction right before it, and no vector instruction written so may touch a result of the
compiler's too early.  The kernels wait behind their products (products_done); that the compiler puts no copy of a result before the wait is checked
here, for every instance."""
import os
import re
import subprocess

import pytest

from paper_2407_00023_amd import build

RESULT = 18   # wait states until a result of 16 passes may be read, more than those of the forms in use
OPERAND = 2   # between a vector instruction and a matrix instruction that reads what it wrote


def registers(text):
    out = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {(kind, i) for i in range(int(a), int(b) + 1)}
    return out | {(kind, int(a)) for kind, a in re.findall(r"\b([va])(\d+)\b", text)}


def blocks_of(lines):
    """Straight pieces of the listing: [label or None, [(line number, instruction, written as inline assembly)]]."""
    blocks, inline = [[None, []]], False
    for number, line in enumerate(lines, 1):
        if "ASMSTART" in line:
            inline = True
        elif "ASMEND" in line:
            inline = False
        s = line.split(";")[0].strip()
        if s.endswith(":"):
            blocks.append([s[:-1], []])
        elif s and not s.startswith("."):
            blocks[-1][1].append((number, s, inline))
            if s.startswith(("s_branch", "s_cbranch", "s_endpgm", "s_setpc")):
                blocks.append([None, []])
    return blocks


def faults(lines):
    """What is wrong in an assembly listing, as text.  Along every path through it: wait states since each register was written, the fewest of all paths."""
    blocks = blocks_of(lines)
    at_label = {label: i for i, (label, _) in enumerate(blocks) if label}
    entry = [({}, {}) for _ in blocks]   # register: (states, line, written as inline assembly), of results, and of what vector instructions wrote
    found, todo = set(), set(range(len(blocks)))
    while todo:
        i = min(todo)
        todo.remove(i)
        results, written = dict(entry[i][0]), dict(entry[i][1])
        goes_on, targets = True, []
        for number, s, inline in blocks[i][1]:
            op, _, rest = s.partition(" ")
            operands = [x.strip() for x in rest.split(",")]
            mfma = op.startswith("v_mfma")
            if mfma:
                read = registers(operands[1] + operands[2])
                if not inline:
                    read |= registers(operands[3])
                else:
                    found |= {f"line {number}: {s} reads what line {written[r][1]} has just written" for r in read | registers(operands[3]) if r in written}
            else:
                read = set() if op.startswith("s_") else registers(rest)
            found |= {f"line {number}: {s} touches the result of line {results[r][1]}" for r in read if r in results and (results[r][2] or inline)}
            states = int(operands[0], 0) + 1 if op == "s_nop" else 1
            results = {r: (n + states, l, by) for r, (n, l, by) in results.items() if n + states < RESULT}
            written = {r: (n + states, l) for r, (n, l) in written.items() if n + states < OPERAND}
            if mfma:
                results.update({r: (0, number, inline) for r in registers(operands[0])})
            elif op.startswith("v_") and not mfma:
                written.update({r: (0, number) for r in registers(operands[0])})
            if op.startswith(("s_branch", "s_cbranch")):
                targets.append(at_label.get(rest.strip()))
            goes_on = not op.startswith(("s_branch", "s_endpgm", "s_setpc"))
        for j in targets + ([i + 1] if goes_on else []):
            if j is None or j >= len(blocks):
                continue
            for now, there in zip((results, written), entry[j]):
                for r, x in now.items():
                    if r not in there or x < there[r]:
                        there[r] = x
                        todo.add(j)
    return sorted(found)


def test_the_check_finds_what_it_is_for():
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], v[0:3]"
    inline = [";;#ASMSTART", mfma, ";;#ASMEND"]
    wait = [";;#ASMSTART", "s_nop 15", "s_nop 3", ";;#ASMEND"]
    copy = ["v_accvgpr_write_b32 a0, v2"]
    assert not faults(inline + inline + wait + copy)
    assert faults(inline + copy)
    assert faults(inline + inline + ["s_nop 7"] + copy)
    assert faults(["v_mov_b32_e32 v9, v20"] + inline)
    assert not faults(["v_mov_b32_e32 v9, v20", "s_nop 1"] + inline)
    assert faults(inline + ["s_cbranch_scc1 .LBB0_1", "s_nop 15", "s_nop 15", ".LBB0_1:"] + copy)   # (the branch goes round the wait)
    assert not faults(inline + wait + [".LBB0_1:"] + copy + ["s_nop 1"] + inline + wait + ["s_cbranch_scc1 .LBB0_1"])
    assert faults(wait + [".LBB0_1:"] + copy + ["s_nop 1"] + inline + ["s_cbranch_scc1 .LBB0_1"])
    assert faults(inline + ["v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[8:11], a[0:3]"])
    assert not faults([mfma] + copy)   # (the compiler's own)
    assert faults([mfma, ";;#ASMSTART", "v_max3_f32 v20, |v0|, |v1|, v20", ";;#ASMEND"])
    assert not faults([mfma] + wait + [";;#ASMSTART", "v_max3_f32 v20, |v0|, |v1|, v20", ";;#ASMEND"])


@pytest.fixture(scope="module", params=["latent_bf16.hip", "latent_expand.hip"])
def listing(tmp_path_factory, request):
    out = str(tmp_path_factory.mktemp("asm") / "latent.s")
    subprocess.run([build._hipcc()] + build.FLAGS + ["-S", "--cuda-device-only", os.path.join(build.CSRC, request.param), "-o", out],
                   check=True, capture_output=True)
    return open(out).read().split("\n")


def test_results_are_waited_for(listing):
    assert sum("v_mfma" in line for line in listing) > 1000
    assert faults(listing) == []


def test_the_loop_keeps_everything_in_registers(listing):
    """The block that has the output's products beside the probabilities touches no scratch memory: a reload waits for all loads on their way."""
    block, blocks = [], []
    for line in listing:
        if re.match(r"(\.LBB|_Z)\w+:", line):
            blocks.append(block)
            block = []
        block.append(line)
    loops = [b for b in blocks + [block] if sum("v_mfma" in x for x in b) >= 8 and any("v_exp_f32" in x for x in b)]
    assert len(loops) >= 4
    for b in loops:
        assert not [x for x in b if re.match(r"\s+scratch_", x)]
