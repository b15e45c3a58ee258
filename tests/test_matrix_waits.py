"""Waits for the matrix cores in the built library (CPU).

A matrix instruction's result is there some time after it was issued, and the hardware
does not hold back a vector instruction that reads (or overwrites) it too early: the
compiler has to put as many instructions or s_nop between.  It has missed one on the way
back to a loop's head, where accumulators were copied between the register files: the copy
took one register of the last product before it was written, in some runs of a kernel and
not in others.  So the machine code of every kernel is walked from each matrix instruction
along all branches."""
from __future__ import annotations

import heapq
import os
import re
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"

# Passes of four cycles each (the CDNA instruction tables).  A vector instruction has to be
# issued at least two states after them (one for products of floats), a state being an
# instruction's issue.  A taken branch, which drops what was fetched, counts for two.
PASSES = {"32x32x16_bf16": 8, "32x32x2_f32": 16, "16x16x4_f32": 8}
REGISTER = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))")


def registers(operands):
    r = set()
    for o in operands:
        for f, lo, hi, one in REGISTER.findall(o):
            r.update((f, i) for i in range(int(lo or one), int(hi or one) + 1))
    return r


def parse(text):
    """{function: (instructions [(name, operands, target)], {address: index})}"""
    functions, name = {}, None
    for line in text.splitlines():
        m = re.match(r"^([0-9a-f]+) <(.+)>:$", line)
        if m:
            name = m.group(2)
            functions[name] = ([], {}, int(m.group(1), 16))
            continue
        m = re.match(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):[0-9A-F ]*(?:<(.+?)(?:\+0x([0-9a-f]+))?>)?$",
                     line)
        if not m or name is None:
            continue
        code, at, start = functions[name]
        target = start + int(m.group(5) or "0", 16) if m.group(4) == name else None
        at[int(m.group(3), 16)] = len(code)
        code.append((m.group(1), re.split(r",\s*(?![^\[]*\])", m.group(2)), target))
    return {n: (c, a) for n, (c, a, _) in functions.items()}


def early(code, at, i):
    """The first use of matrix instruction i's result that comes too early, or None."""
    op, operands, _ = code[i]
    shape = next((p for p in PASSES if p in op), None)
    assert shape, f"no passes known of {op}"
    result = registers(operands[:1])
    need = PASSES[shape] + (1 if shape.endswith("_f32") else 2)
    queue, seen = [(0, i + 1, PASSES[shape])], {}
    while queue:
        t, j, free = heapq.heappop(queue)
        if t >= need or j >= len(code) or seen.get(j, need) <= t:
            continue
        seen[j] = t
        op, operands, target = code[j]
        if op == "s_nop":
            heapq.heappush(queue, (t + int(operands[0], 0) + 1, j + 1, free))
        elif op == "s_branch":
            heapq.heappush(queue, (t + 2, at[target], free))
        elif op == "s_endpgm":
            continue
        elif op.startswith("s_cbranch"):
            heapq.heappush(queue, (t + 2, at[target], free))
            heapq.heappush(queue, (t + 1, j + 1, free))
        elif "mfma" in op:
            # it is issued when the matrix core is free again; results passed on as the
            # next one's sum are the hardware's business
            t = max(t, free)
            if registers(operands[1:3]) & result and t < need:
                return j, t
            if registers(operands[:1]) & result:
                continue
            heapq.heappush(queue, (t + 1, j + 1, t + PASSES[next(p for p in PASSES if p in op)]))
        else:
            if not op.startswith("s_") and registers(operands) & result:
                return j, t
            heapq.heappush(queue, (t + 1, j + 1, free))
    return None


def too_early(text):
    found = []
    for name, (code, at) in parse(text).items():
        for i, c in enumerate(code):
            if "mfma" in c[0]:
                e = early(code, at, i)
                if e:
                    found.append((name, " ".join([c[0], *c[1]]), " ".join(
                        [code[e[0]][0], *code[e[0]][1]]), e[1]))
    return found


def test_the_walk_sees_a_missing_wait():
    def listing(nops, use):
        ins = ["v_mfma_f32_32x32x16_bf16 a[0:15], v[70:73], v[2:5], a[0:15]", "s_cbranch_scc0 3",
               "s_mov_b32 s2, s65", f"s_nop {nops}", use, "s_branch 65530 <f+0x8>", "s_endpgm"]
        out = ["0000000000000000 <f>:"]
        for i, x in enumerate(ins):
            op, target = x, ""
            if "cbranch" in x:
                target = " <f+0x18>"
            if "s_branch" in x:
                op, target = "s_branch 65530", " <f+0x8>"
            out.append(f"\t{op} // {4 * i:012X}: 00000000{target}")
        return "\n".join(out)

    assert not too_early(listing(7, "v_accvgpr_read_b32 v17, a15"))
    assert too_early(listing(6, "v_accvgpr_read_b32 v17, a15"))
    assert not too_early(listing(0, "v_accvgpr_read_b32 v17, a16"))
    assert too_early(listing(0, "global_store_dwordx4 v[0:1], a[12:15], off"))
    # the next product: of the result itself, or added to it
    assert too_early(listing(6, "v_mfma_f32_32x32x16_bf16 a[16:31], a[0:3], v[2:5], 0"))
    assert not too_early(listing(0, "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[2:5], a[0:15]"))


def test_no_result_is_used_too_early(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    from paper_1505_02890_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_1505_02890_amd.build import build
        build()
    lib = tmp_path / "lib.so"
    lib.write_bytes(open(_lib.LIB_PATH, "rb").read())
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True,
                   capture_output=True)
    parts = sorted(p for p in tmp_path.iterdir() if "gfx950" in p.name)
    assert parts
    products = 0
    for p in parts:
        text = subprocess.run([OBJDUMP, "-d", str(p)], check=True, capture_output=True,
                              text=True).stdout
        products += text.count("v_mfma")
        assert too_early(text) == [], p.name
    assert products > 1000
