"""The instructions that the kernels write out (products tied to their sums, loads straight to
LDS) in the library as built, without a GPU.  The compiler keeps the distances between its own
instructions, but does not look into those: here they are measured in the code of
libultraep.so, along every path that leads to such an instruction or away from it.

  - what the vector ALU writes, a matrix instruction takes (factors, sums, scales) 2 wait states
    later at the earliest;
  - a matrix instruction's sums are taken by anything but the matrix unit 4 wait states after its
    passes (PASSES) at the earliest;
  - a scalar register that the vector ALU writes is an address of a memory instruction 5 wait
    states later at the earliest;
  - m0 is written a wait state before a load to LDS takes its place from it.

A wait state is an instruction between, s_nop n are n + 1."""
import collections
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_04101_amd as uep

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
PASSES = {"v_mfma_f32_16x16x32_bf16": 4, "v_mfma_i32_16x16x64_i8": 4, "v_mfma_i32_32x32x32_i8": 8,
          "v_mfma_scale_f32_16x16x128_f8f6f4": 8}
REG = re.compile(r"\b([vas])\[(\d+):(\d+)\]|\b([vas])(\d+)\b|\b(vcc|m0)\b")
LINE = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):(?: [0-9A-F]{8})+(?: <\S+?(?:\+0x([0-9a-f]+))?>)?\s*$")
NO_RESULT = re.compile(r"(global|buffer|flat|scratch)_store|ds_write|global_load_lds|\w+_atomic|s_(cmp|bitcmp|wait|barrier|c?branch)")
MEMORY = ("global_", "buffer_", "flat_", "scratch_")

Instruction = collections.namedtuple("Instruction", "op text at to result taken states")


def registers(text):
    out = set()
    for kind, lo, hi, one, n, special in REG.findall(text):
        if kind:
            out.update((kind, i) for i in range(int(lo), int(hi) + 1))
        else:
            out.add((one, int(n)) if one else (special, 0))
    return out


def instruction(line, base):
    m = LINE.match(line)
    if not m:
        return None
    op, rest, at, to = m.groups()
    parts = re.split(r",\s*(?![^\[]*\])", rest)
    if NO_RESULT.match(op) or rest.endswith(" lds"):
        result, taken = set(), registers(rest)
    else:
        result, taken = registers(parts[0]), registers(",".join(parts[1:]))
        if re.match(r"v_(add|sub|subrev|addc|subb|subbrev)_co|v_div_scale|v_mad_[ui]64", op):
            result |= registers(parts[1])  # the carry
        if "fmac" in op:
            taken |= result
    return Instruction(op, f"{op} {rest}", int(at, 16), base + int(to or "0", 16) if "branch" in op else None, result, taken,
                       int(parts[0], 0) + 1 if op == "s_nop" else 1)


def kernels(text):
    """name, instructions of each function of a disassembly."""
    name, base, code = None, 0, []
    for line in text.splitlines():
        m = re.match(r"^([0-9a-f]+) <(\S+)>:", line)
        if m:
            if code:
                yield name, code
            name, base, code = m[2], int(m[1], 16), []
        elif name:
            i = instruction(line, base)
            if i:
                code.append(i)
            else:
                assert not line.startswith("\t") or line.strip() == "...", line
    if code:
        yield name, code


def edges(code):
    where = {i.at: n for n, i in enumerate(code)}
    after, before = [[] for _ in code], [[] for _ in code]
    for n, i in enumerate(code):
        if i.to is not None:
            after[n].append(where[i.to])
        if i.op not in ("s_branch", "s_endpgm") and n + 1 < len(code):
            after[n].append(n + 1)
        for k in after[n]:
            before[k].append(n)
    return before, after


def within(code, steps, n, states):
    """What lies less than `states` wait states from instruction n along the steps."""
    seen, todo = {}, [(k, 0) for k in steps[n]]
    while todo:
        k, d = todo.pop()
        if d >= states or seen.get(k, states) <= d:
            continue
        seen[k] = d
        yield code[k]
        todo += [(j, d + code[k].states) for j in steps[k]]


def close_ones(code):
    """(rule, earlier, later) of the instructions that lie too close, and how many were looked at."""
    before, after = edges(code)
    found, looked = [], collections.Counter()
    for n, i in enumerate(code):
        if i.op.startswith("v_mfma"):
            looked["matrix"] += 1
            for j in within(code, before, n, 2):
                if j.op.startswith("v_") and not j.op.startswith("v_mfma") and j.result & (i.taken | i.result):
                    found.append(("operand", j.text, i.text))
            for j in within(code, after, n, PASSES[i.op] + 4):
                if not j.op.startswith(("v_mfma", "s_")) and (j.result | j.taken) & i.result:
                    found.append(("sums", i.text, j.text))
        if i.op.startswith(MEMORY):
            address = {r for r in i.taken | i.result if r[0] in ("s", "vcc")}
            for j in within(code, before, n, 5) if address else ():
                if j.op.startswith("v_") and j.result & address:
                    found.append(("address", j.text, i.text))
            if i.op.startswith("global_load_lds") or i.text.endswith(" lds"):
                looked["to lds"] += 1
                for j in within(code, before, n, 1):
                    if ("m0", 0) in j.result:
                        found.append(("m0", j.text, i.text))
    return found, looked


@pytest.fixture(scope="module")
def disassembly(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    at = tmp_path_factory.mktemp("library")
    shutil.copy(uep.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    parts = sorted(p for p in os.listdir(at) if "gfx950" in p)
    assert parts
    return [subprocess.run([OBJDUMP, "-d", p], cwd=at, check=True, capture_output=True, text=True).stdout for p in parts]


def test_the_library_keeps_its_distances(disassembly):
    total, found = collections.Counter(), []
    for text in disassembly:
        for name, code in kernels(text):
            if any(i.op.startswith("v_mfma") or " lds" in i.text or "_lds_" in i.op for i in code):
                close, looked = close_ones(code)
                found += [(name, *c) for c in close]
                total += looked
    assert not found, (len(found), found[:5])
    assert total["matrix"] > 5000 and total["to lds"] > 2000


def listing(*lines):
    """Instructions of 4 bytes from 0x100 on; a branch's target as <k+0x..>."""
    out = ["0000000000000100 <k>:"]
    for n, line in enumerate(lines):
        text, _, to = line.partition(" -> ")
        out.append(f"\t{text} // {0x100 + 4 * n:012X}: 00000000" + (f" <k+0x{4 * int(to):x}>" if to else ""))
    ((_, code),) = kernels("\n".join(out))
    return [rule for rule, _, _ in close_ones(code)[0]]


MFMA = "v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]"
SCALED = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:7], v[8:15], a[0:3], v16, v17 op_sel_hi:[0,0,0]"


@pytest.mark.parametrize("lines,rules", [
    (["v_mov_b32_e32 v3, v9", MFMA], ["operand"]),
    (["v_mov_b32_e32 v3, v9", "s_nop 0", MFMA], ["operand"]),
    (["v_mov_b32_e32 v3, v9", "s_nop 1", MFMA], []),
    (["v_mov_b32_e32 v8, v9", MFMA], []),
    (["v_accvgpr_write_b32 a2, 0", "s_nop 0", MFMA], ["operand"]),
    (["v_lshrrev_b32_e32 v17, 8, v17", "s_nop 0", SCALED], ["operand"]),
    (["ds_read_b128 v[0:3], v20", MFMA], []),  # (s_waitcnt's to keep)
    ([MFMA, MFMA], []),
    ([MFMA, "s_nop 6", "v_accvgpr_read_b32 v9, a0"], ["sums"]),
    ([MFMA, "s_nop 7", "v_accvgpr_read_b32 v9, a0"], []),
    ([SCALED, "s_nop 10", "v_accvgpr_read_b32 v30, a0"], ["sums"]),
    ([SCALED, "s_nop 11", "v_accvgpr_read_b32 v30, a0"], []),
    ([MFMA, "s_nop 1", "global_store_dwordx4 v[8:9], a[0:3], off"], ["sums"]),
    # round a loop: the write at its end, the product at its beginning
    (["s_nop 4", MFMA, "s_nop 7", "v_mov_b32_e32 v7, v9", "s_cbranch_scc1 65532 -> 1"], ["operand"]),
    (["s_nop 4", MFMA, "s_nop 7", "v_mov_b32_e32 v7, v9", "s_nop 0", "s_cbranch_scc1 65532 -> 1"], []),
    (["s_branch 1 -> 2", "v_mov_b32_e32 v3, v9", MFMA], ["operand"]),
    (["v_mov_b32_e32 v3, v9", "s_branch 1 -> 3", "v_mov_b32_e32 v3, v9", MFMA], ["operand", "operand"]),
    (["v_readfirstlane_b32 s4, v0", "s_nop 3", "global_load_lds_dwordx4 v1, s[4:5]"], ["address"]),
    (["v_readfirstlane_b32 s4, v0", "s_nop 4", "global_load_lds_dwordx4 v1, s[4:5]"], []),
    (["s_mov_b32 s4, s9", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"], []),
    (["s_add_u32 m0, s9, 0x1000", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"], ["m0"]),
    (["s_add_u32 m0, s9, 0x1000", "s_nop 0", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"], [])])
def test_what_lies_too_close_is_seen(lines, rules):
    assert listing(*lines) == rules
