"""Scalar registers that the vector unit has written are old enough when a vector memory instruction reads them: the processor asks for five
wait states between the two and does not check.  The compiler sees to that for the loads that it makes, not for those in assembly text (memory
to LDS in the projections' kernels), so the built code is looked over."""
import os
import re
import struct
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
NEEDED = 5


def code_objects(path):
    with open(path, "rb") as f:
        data = f.read()
    for m in re.finditer(b"\x7fELF\x02\x01", data):
        base = m.start()
        if struct.unpack_from("<H", data, base + 18)[0] != 224:                  # EM_AMDGPU
            continue
        shoff, = struct.unpack_from("<Q", data, base + 40)
        size, count = struct.unpack_from("<HH", data, base + 58)
        yield data[base:base + shoff + size * count]


def functions(text):
    """name -> [(address, mnemonic, operands, target of a branch or None)], from a disassembly"""
    out, base, here = {}, {}, None
    for line in text.splitlines():
        m = re.match(r"([0-9a-f]+) <(.+)>:$", line)
        if m:
            here = out.setdefault(m.group(2), [])
            base[m.group(2)] = int(m.group(1), 16)
            continue
        m = re.match(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):[^<]*(?:<(.+?)(?:\+0x([0-9a-f]+))?>)?$", line)
        if m and here is not None:
            branch = m.group(1).startswith(("s_branch", "s_cbranch"))
            here.append((int(m.group(3), 16), m.group(1), m.group(2), base[m.group(4)] + int(m.group(5) or "0", 16) if branch else None))
    return out


def scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return range(int(m.group(1)), int(m.group(2)) + 1)
    m = re.fullmatch(r"s(\d+)", operand)
    return [int(m.group(1))] if m else []


def split(operands):
    return [o.strip() for o in re.split(r",(?![^\[]*\])", operands.split(" offen")[0])]


def too_early(code):
    """Instructions that read a scalar register less than NEEDED wait states after the vector unit wrote it, on any path."""
    index = {at: i for i, (at, *_rest) in enumerate(code)}
    facts = []                                               # (waits it gives, registers read by memory, written by VALU, written otherwise)
    for _, name, operands, _ in code:
        ops = split(operands)
        reads, by_valu, other = [], [], []
        if name.startswith(("buffer_", "global_", "flat_", "scratch_")):
            reads = [r for o in ops for word in o.split() for r in scalars(word)]
        elif name.startswith("v_"):
            by_valu = [r for o in ops[:2 if re.search(r"_co_|div_scale|mad_[ui]64", name) else 1] for r in scalars(o)]
        elif name.startswith("s_") and not name.startswith(("s_cmp", "s_bitcmp", "s_cbranch", "s_waitcnt", "s_nop", "s_store")):
            other = list(scalars(ops[0]))
        facts.append((1 + int(ops[0], 0) if name == "s_nop" else 1, reads, by_valu, other))
    young = [None] * len(code)                               # before an instruction: register -> the fewest wait states since the VALU wrote it
    work = {0}
    young[0] = {}
    while work:
        i = work.pop()
        waits, _, by_valu, other = facts[i]
        after = {r: n + waits for r, n in young[i].items() if n + waits < NEEDED and r not in other}
        after.update({r: 0 for r in by_valu})
        _, name, _, target = code[i]
        nexts = [] if name in ("s_branch", "s_endpgm", "s_setpc_b64") else [i + 1] if i + 1 < len(code) else []
        if target in index:
            nexts.append(index[target])
        for k in nexts:
            if young[k] is None:
                young[k] = dict(after)
                work.add(k)
            else:
                less = {r: n for r, n in after.items() if n < young[k].get(r, NEEDED)}
                if less:
                    young[k].update(less)
                    work.add(k)
    return [(code[i][1] + " " + code[i][2], r, young[i][r]) for i in range(len(code)) if young[i] for r in facts[i][1] if r in young[i]]


def test_the_check_finds_what_it_looks_for():
    line = "\t%s // %012X: 00000000"

    def text(*instructions):
        return "\n".join(["0000000000000000 <f>:"] + [line % (s, 4 * i) for i, s in enumerate(instructions)])
    load = "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"
    for early, instructions in ((True, ["v_readfirstlane_b32 s6, v0", "s_mov_b32 m0, s9", "s_nop 0", load]),
                                (True, ["v_readfirstlane_b32 s6, v0", "s_nop 3", load]),
                                (False, ["v_readfirstlane_b32 s6, v0", "s_nop 4", load]),
                                (False, ["v_readfirstlane_b32 s6, v0", "s_mov_b32 s6, 1", load]),
                                (False, ["v_readfirstlane_b32 s8, v0", load]),
                                (True, ["v_cmp_lt_i32_e64 s[6:7], v0, v1", load]),
                                (True, ["v_add_co_u32_e64 v0, s[4:5], v0, v1", load]),
                                (True, ["v_readlane_b32 s2, v0, 1", "global_load_dword v0, v1, s[2:3]"])):
        assert bool(too_early(functions(text(*instructions, "s_endpgm"))["f"])) == early, instructions
    # over a branch back
    loop = text("s_nop 4", load, "v_readfirstlane_b32 s6, v0") + "\n\ts_cbranch_scc1 65532 // 00000000000C: BF85FFFC <f+0x4>\n" + line % ("s_endpgm", 16)
    assert [r for _, r, _ in too_early(functions(loop)["f"])] == [6]


def test_loads_of_the_library(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    from paper_2110_09195_amd import binding
    binding.lib()
    seen, found = 0, {}
    for n, blob in enumerate(code_objects(binding.LIB_PATH)):
        path = tmp_path / ("%d.elf" % n)
        path.write_bytes(blob)
        text = subprocess.run([OBJDUMP, "-d", str(path)], check=True, capture_output=True, text=True).stdout
        if " lds " not in text:                              # (the compiler's own loads are its own business)
            continue
        for name, code in functions(text).items():
            loads = sum(1 for _, m, operands, _ in code if m.startswith("buffer_load") and operands.endswith("lds"))
            if loads:
                seen += 1
                early = too_early(code)
                if early:
                    found[name] = early[:3]
    assert seen >= 40, seen
    assert not found, found
