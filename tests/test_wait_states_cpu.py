"""Wait states in the built library's own kernels.

The gfx9 family leaves some waits between two instructions to whoever writes them.  The compiler keeps them between
instructions of its own; it cannot see into an asm statement, so what stands there, and what stands next to it, is checked
here, in the disassembled kernels of libsx.so, along every path that leads to an instruction:

  m0     a scalar instruction writes m0, a transfer to LDS reads it: 1
  base   a vector instruction writes a scalar register, a memory instruction reads it: 5
  dpp    a vector instruction writes a vector register, one that takes it from another lane (DPP) reads it: 2
  lane   a vector instruction writes a vector register, v_readlane or v_readfirstlane reads it: 1

An instruction counts as one wait state, s_nop n as n + 1."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2606_01751_amd as sx

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
REG = re.compile(r"^-?\|?(s|v|a)(?:(\d+)|\[(\d+):(\d+)\])\|?$")
LINE = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):")
TARGET = re.compile(r"<(.+)\+0x([0-9a-f]+)>$")
SYMBOL = re.compile(r"^([0-9a-f]+) <(.+)>:$")


def regs(operand):
    """The registers that an operand names, as (file, number)."""
    o = operand.strip().split(" ")[0]
    if o in ("m0", "vcc", "exec"):
        return {(o, 0)}
    m = REG.match(o)
    if not m:
        return set()
    lo, hi = (int(m[2]), int(m[2])) if m[2] else (int(m[3]), int(m[4]))
    return {(m[1], i) for i in range(lo, hi + 1)}


def split(text):
    return re.split(r",\s*", text) if text else []


def is_valu(op):
    return op.startswith("v_")


def is_memory(op):
    return op.startswith(("global_", "buffer_", "flat_", "scratch_"))


def valu_writes(op, args):
    """What a vector instruction writes (its second operand too where that is a carry or a flag)."""
    if not is_valu(op) or not args or op.startswith("v_nop"):
        return set()
    out = regs(args[0])
    if len(args) > 1 and ("_co_" in op or op.startswith("v_div_scale")):
        out |= regs(args[1])
    return out


def m0_write(op, args):
    return {("m0", 0)} if op.startswith("s_") and args and args[0] == "m0" and not op.startswith("s_cmp") else set()


def scalar_of(op, args):
    return {r for r in valu_writes(op, args) if r[0] in ("s", "vcc")}


def vector_of(op, args):
    return {r for r in valu_writes(op, args) if r[0] == "v"}


# name: (wait states, what is written by an instruction, what an instruction reads)
RULES = {
    "m0": (1, m0_write, lambda op, a: {("m0", 0)} if "_lds_" in op and is_memory(op) else set()),
    "base": (5, scalar_of, lambda op, a: {r for o in a for r in regs(o) if r[0] in ("s", "vcc")} if is_memory(op) else set()),
    "dpp": (2, vector_of, lambda op, a: {r for r in regs(a[1]) if r[0] == "v"} if op.endswith("_dpp") else set()),
    "lane": (1, vector_of, lambda op, a: {r for r in regs(a[1]) if r[0] == "v"} if op.startswith(("v_readlane", "v_readfirstlane")) else set()),
}


def states(op, args):
    return int(args[0], 0) + 1 if op == "s_nop" else 1


def kernels(text):
    """[(symbol, [(address, op, operands, where it may branch to or None)])] of a disassembly."""
    out, start = [], {}
    for line in text.splitlines():
        m = SYMBOL.match(line)
        if m:
            start[m[2]] = int(m[1], 16)
            out.append((m[2], []))
            continue
        m = LINE.match(line)
        if m and out:
            t = TARGET.search(line) if m[1].startswith(("s_cbranch", "s_branch")) else None
            to = start[t[1]] + int(t[2], 16) if t else None
            out[-1][1].append((int(m[3], 16), m[1], split(m[2]), to))
    return out


def missing(code, rule):
    """Instructions of a kernel that read a register too soon: (address of the write, of the read, wait states between)."""
    need, writes, reads = RULES[rule]
    index = {a: i for i, (a, _, _, _) in enumerate(code)}
    before = [[] for _ in code]
    for i, (_, op, _, to) in enumerate(code):
        if i + 1 < len(code) and op not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            before[i + 1].append(i)
        if to in index:
            before[index[to]].append(i)
    found = []
    for i, (addr, op, args, _) in enumerate(code):
        want = reads(op, args)
        todo = [(j, 0) for j in before[i]] if want else []
        seen = {}
        while todo:
            j, have = todo.pop()
            if have >= need or seen.get(j, need) <= have:
                continue
            seen[j] = have
            a, o, ar, _ = code[j]
            if writes(o, ar) & want:
                found.append((hex(a), hex(addr), have))
                continue
            todo += [(p, have + states(o, ar)) for p in before[j]]
    return found


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    sx.lib()
    at = tmp_path_factory.mktemp("kernels")
    shutil.copy(sx.RELEASE_LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    out = []
    for f in sorted(os.listdir(at)):
        if f.endswith("gfx950"):
            out += kernels(subprocess.run([OBJDUMP, "-d", f], cwd=at, check=True, capture_output=True, text=True).stdout)
    return out


@pytest.mark.parametrize("rule", RULES)
def test_wait_states(built, rule):
    assert sum(1 for _, code in built for _, op, _, _ in code if "_lds_" in op and is_memory(op)) > 100   # (the kernels are there)
    bad = {name: found for name, code in built if (found := missing(code, rule))}
    assert not bad, f"{rule}: {sum(map(len, bad.values()))} in {len(bad)} kernels, e.g. {[(n, f[0]) for n, f in bad.items()][:3]}"


def listing(*lines):
    return kernels("0000000000000000 <k>:\n" + "\n".join(f"\t{l} // {4 * i:012X}: 00000000" for i, l in enumerate(lines)))[0][1]


def test_the_check_finds_what_is_too_near():
    # a base read after four wait states, after five, and around a loop; m0 with and without a wait
    four = ["v_readfirstlane_b32 s4, v0", *["s_nop 0"] * 4, "global_load_lds_dwordx4 v1, s[4:5]"]
    assert missing(listing(*four), "base") == [("0x0", "0x14", 4)]
    assert missing(listing(four[0], "s_nop 4", four[-1]), "base") == []
    assert missing(listing("s_mov_b32 m0, s1", four[-1]), "m0") == [("0x0", "0x4", 0)]
    assert missing(listing("s_mov_b32 m0, s1", "s_nop 0", four[-1]), "m0") == []
    assert missing(listing("v_add_f32_e32 v1, v2, v3", "s_nop 0", "v_mov_b32_dpp v4, v1 row_ror:8 row_mask:0xf bank_mask:0xf"), "dpp") == [("0x0", "0x8", 1)]
    loop = "0000000000000000 <k>:\n\tglobal_load_dword v1, v2, s[4:5] // 000000000000: 0\n\tv_readlane_b32 s5, v0, 3 // 000000000004: 0\n" \
           "\ts_cbranch_scc1 65533 // 000000000008: 0 <k+0x0>\n\ts_endpgm // 00000000000C: 0\n"
    assert missing(kernels(loop)[0][1], "base") == [("0x4", "0x0", 1)]
