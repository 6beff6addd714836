"""CPU: no vector instruction of the built library reads what a matrix instruction computes before it is there, whichever way a branch goes.

The hardware does not wait by itself: the compiler puts other instructions, or s_nop, between the two.  Where two ways lead into a block it has been seen to count along the longer one alone, so
that a read behind a taken branch came 2 instructions after the matrix instruction, where 8 are needed.  The library's own code objects are disassembled and walked along every way."""
import os
import re
import subprocess
from concurrent.futures import ProcessPoolExecutor

import pytest

import paper_2510_18716_amd as ssd

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# passes (a matrix instruction begins when the one before it has been through them), and how many instructions have to lie between it and a vector instruction that reads its result:
# the least that the compiler itself puts between the two in one block
MATRIX = {"v_mfma_f32_16x16x32_bf16": (4, 8), "v_mfma_f32_16x16x4_f32": (8, 10), "v_mfma_f32_32x32x16_bf16": (8, 12), "v_mfma_f32_32x32x2_f32": (16, 18)}
FAR = max(need for _, need in MATRIX.values())
LINE = re.compile(r"^\t(\w+)([^/]*)// ([0-9A-F]{12}):(?:.*<(?:[^+>]*)\+0x([0-9a-f]+)>)?")
REG = re.compile(r"\b[va](?:\[(\d+):(\d+)\]|(\d+)\b)")


def registers(text):
    out = set()
    for a, b, one in REG.findall(text):
        out.update(range(int(a), int(b) + 1) if a else (int(one),))
    return out


def operands(text):
    """(what comes first, the rest)."""
    depth = 0
    for i, ch in enumerate(text):
        depth += (ch == "[") - (ch == "]")
        if ch == "," and depth == 0:
            return text[:i], text[i:]
    return text, ""


def early_reads(code):
    """code: [(opcode, operands, offset of a branch's target or None)] of one function, with `at` {offset: index}.  Yields (matrix instruction, reading instruction, instructions between)."""
    ins, at = code
    for i, (op, text, _) in enumerate(ins):
        if not op.startswith("v_mfma"):
            continue
        passes, need = MATRIX[op.replace("_e64", "")]
        if not any(x[0].startswith(("s_cbranch", "s_branch")) for x in ins[i + 1:i + 1 + need]):
            continue                                                # within a block the compiler counts right
        ways = [(i + 1, 0, passes - 1, frozenset(registers(operands(text)[0])))]
        seen = set()
        while ways:
            j, between, free, live = ways.pop()                     # free: when the matrix unit takes the next one
            while j < len(ins) and between < need and live:
                if (j, between, live) in seen:
                    break
                seen.add((j, between, live))
                name, rest, target = ins[j]
                if name == "s_endpgm":
                    break
                if name.startswith(("s_cbranch", "s_branch")):
                    if target in at:
                        ways.append((at[target], between + 1, free, live))
                    if name == "s_branch":
                        break
                elif name == "s_nop":
                    between += int(rest.strip() or "0", 0)
                elif name.startswith("v_mfma"):
                    between = max(between, free)
                    free = between + MATRIX[name.replace("_e64", "")][0]
                    live = live - registers(operands(rest)[0])
                elif name.startswith(("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")):
                    first, others = operands(rest)
                    writes = name.startswith(("ds_read", "global_load", "buffer_load", "scratch_load", "flat_load")) or name.startswith("v_") and not name.startswith("v_cmp")
                    reads = registers(others if writes and "swap" not in name and not name.startswith(("v_fmac", "v_dot2c")) else rest)
                    if reads & live:
                        yield i, j, between
                        live = live - reads
                    if writes:
                        live = live - registers(first)
                between += 1
                j += 1


def functions(text):
    """(name, code) of the functions that have matrix instructions."""
    for block in text.split("\n\n"):
        if "v_mfma" not in block or ">:" not in block:
            continue
        head, _, body = block.lstrip("\n").partition("\n")
        name, base, ins, at = head.split("<")[1][:-2], int(head.split()[0], 16), [], {}
        for line in body.split("\n"):
            m = LINE.match(line)
            if m:
                at[int(m[3], 16) - base] = len(ins)
                ins.append((m[1], m[2], int(m[4], 16) if m[4] else None))
        yield name, (ins, at)


def early_reads_of(path):
    """(matrix instructions, what of them is read too early) of a code object."""
    text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], check=True, stdout=subprocess.PIPE, text=True).stdout
    matrix, found = 0, []
    for name, code in functions(text):
        matrix += sum(op.startswith("v_mfma") for op, _, _ in code[0])
        found += [(name, " ".join(code[0][i][:2]).strip(), " ".join(code[0][j][:2]).strip(), n) for i, j, n in early_reads(code)]
    return matrix, found


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_results_of_matrix_instructions_are_waited_for(tmp_path, library=None):
    lib = tmp_path / "lib.so"
    lib.symlink_to(os.path.abspath(library or ssd.lib_path))
    subprocess.run([OBJDUMP, "--offloading", str(lib)], check=True, stdout=subprocess.DEVNULL, cwd=tmp_path)
    objects = sorted((str(p) for p in tmp_path.iterdir() if "gfx950" in p.name), key=os.path.getsize, reverse=True)
    assert objects
    with ProcessPoolExecutor(4) as pool:
        each = list(pool.map(early_reads_of, objects))
    matrix, found = sum(n for n, _ in each), [x for _, some in each for x in some]
    assert matrix > 1000                                            # the library was read
    assert not found, "%d reads, the first: %s" % (len(found), found[:3])


def test_the_walk_finds_a_read_behind_a_taken_branch():
    """A matrix instruction, a branch over eight moves to a block that reads its result; and the same with the wait."""
    head = [("v_mfma_f32_16x16x32_bf16", " v[0:3], v[4:7], v[8:11], v[0:3]", None), ("s_cbranch_scc1", " 9", 40)]
    moves = [("v_mov_b32_e32", " v20, v21", None)] * 8
    tail = [("v_max_f32_e32", " v22, v1, v1", None), ("s_endpgm", "", None)]
    at = {4 * i: i for i in range(20)}
    assert [x[1:] for x in early_reads((head + moves + tail, at))] == [(10, 1)]
    waited = head[:1] + [("s_nop", " 6", None)] + [("s_cbranch_scc1", " 9", 44)] + moves + tail
    assert list(early_reads((waited, at))) == []
