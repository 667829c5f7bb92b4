"""Idle slots that gfx950 asks for between two instructions, in the device code
of the built library.  The compiler puts them in for the instructions that it
knows, but not behind those written as inline assembly, which it does not look
into; a missing one can hand the second instruction a value that is not there
yet.  No GPU is needed."""
import functools
import os
import re
import shutil
import struct
import subprocess
import tempfile

import pytest

S = pytest.importorskip("paper_2511_18672_amd")

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _objdump():
    for c in (shutil.which("llvm-objdump"), "/opt/rocm/llvm/bin/llvm-objdump"):
        if c and os.path.exists(c):
            return c
    return None


def _code_objects(data):
    """The gfx950 code objects of a library: every translation unit left one in a bundle."""
    at = data.find(MAGIC)
    while at >= 0:
        (n,), p = struct.unpack_from("<Q", data, at + len(MAGIC)), at + len(MAGIC) + 8
        for _ in range(n):
            off, size, name = struct.unpack_from("<QQQ", data, p)
            if size and b"gfx950" in data[p + 24:p + 24 + name]:
                yield data[at + off:at + off + size]
            p += 24 + name
        at = data.find(MAGIC, at + len(MAGIC))


class Instr:
    """One instruction: its name, the vector registers of its first operand, of the others, and of the next two."""

    def __init__(self, line):
        text, _, note = line.partition("//")
        self.text = text.strip()
        self.op, _, operands = self.text.partition(" ")
        parts = [o.strip() for o in re.split(r",(?![^\[]*\])", operands)]
        self.first = _registers(parts[0]) if parts else frozenset()
        self.rest = frozenset().union(*[_registers(o) for o in parts[1:]])
        self.factors = frozenset().union(*[_registers(o) for o in parts[1:3]])  # of a product
        self.operands = parts
        m = re.search(r"<\S+\+0x([0-9a-f]+)>", note)
        self.target = int(m.group(1), 16) if m and self.op.startswith(("s_branch", "s_cbranch")) else None
        self.address = int(note.split(":")[0], 16)

    def slots(self):
        return int(self.operands[0]) + 1 if self.op == "s_nop" else 1


def _registers(operand):
    out = set()
    for a, b, c in re.findall(r"\bv(?:(\d+)|\[(\d+):(\d+)\])", operand):
        out |= {int(a)} if a else set(range(int(b), int(c) + 1))
    return frozenset(out)


@functools.lru_cache(None)
def kernels():
    """Kernel name -> its instructions, in order."""
    if not os.path.exists(S.binding.LIB_PATH):
        pytest.skip("libsphinx.so not built")
    if _objdump() is None:
        pytest.skip("llvm-objdump not available")
    with open(S.binding.LIB_PATH, "rb") as f:
        data = f.read()
    out = {}
    for code in _code_objects(data):
        with tempfile.NamedTemporaryFile(suffix=".o") as f:
            f.write(code)
            f.flush()
            r = subprocess.run([_objdump(), "-d", f.name], capture_output=True, text=True, check=True)
        name = None
        for line in r.stdout.splitlines():
            m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if m:
                name = m.group(1)
                out[name] = []
            elif name is not None and line.startswith("\t") and "//" in line:
                out[name].append(Instr(line))
    assert len(out) > 50
    return out


def following(code, i, slots):
    """Instructions that can run behind number i before `slots` slots have passed, on every path."""
    at = {x.address - code[0].address: j for j, x in enumerate(code)}
    todo, seen = [(i + 1, slots)], set()
    while todo:
        j, left = todo.pop()
        if left <= 0 or j >= len(code) or (j, left) in seen:
            continue
        seen.add((j, left))
        x = code[j]
        yield x
        if x.op.startswith("s_endpgm"):
            continue
        left -= x.slots()
        if x.target is not None:
            todo.append((at[x.target], left))
        if x.op != "s_branch":
            todo.append((j + 1, left))


def early_readers_of_dot_sums(code):
    """A dot product's sum takes three slots to be there for any instruction but the next dot product that adds to it."""
    bad = []
    for i, x in enumerate(code):
        if not x.op.startswith("v_dot"):
            continue
        for y in following(code, i, 3):
            if not y.op.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")):
                continue
            same = y.op == x.op  # may add to the sum, or start it anew, but not multiply by it
            if x.first & (y.factors if same else y.first | y.rest):
                bad.append((x.text, y.text))
    return bad


def early_copies_behind_m0(code):
    """A direct copy to LDS takes its place there from M0, which has to be written two instructions before it."""
    bad = []
    for i, x in enumerate(code):
        if not (x.op.startswith("s_") and x.operands[0] == "m0"):
            continue
        for y in following(code, i, 1):
            if y.op.startswith(("global_load_lds", "buffer_load_lds", "s_sendmsg", "s_movrel")) or " lds" in y.text:
                bad.append((x.text, y.text))
    return bad


def asm(*lines):
    return [Instr(f"{t} // {4 * i:012X}: 00000000" + (f" <k+0x{4 * to:x}>" if to is not None else ""))
            for i, (t, to) in enumerate((x, None) if isinstance(x, str) else x for x in lines)]


def test_the_search_finds_what_it_looks_for():
    dot, cmp_ = "v_dot2c_f32_bf16_e32 v3, 0x3f803f80, v1", "v_cmp_nge_f32_e32 vcc, s0, v3"
    find = early_readers_of_dot_sums
    assert find(asm(dot, cmp_)) and find(asm(dot, "s_nop 1", cmp_)) and find(asm(dot, "v_mov_b32_e32 v3, 0"))
    assert find(asm(dot, "s_nop 0", "v_mul_f32_e32 v7, v[2:3], v1")) and find(asm(dot, "global_store_dword v0, v3, s[2:3]"))
    assert find(asm(dot, ("s_cbranch_vccz 1", 3), "s_endpgm", cmp_))
    assert find(asm(dot, "v_dot2c_f32_bf16_e32 v4, v3, v1"))
    dot4 = "v_dot4_u32_u8 v3, v7, s7, v5"
    assert find(asm(dot4, "v_dot4_u32_u8 v6, v3, s6, v9")) and not find(asm(dot4, "v_dot4_u32_u8 v6, v6, s6, v3"))
    assert not find(asm(dot, dot, "s_nop 2", cmp_)) and not find(asm(dot, "s_nop 2", cmp_))
    assert not find(asm(dot, "v_add_f32_e32 v4, v1, v2", "s_nop 0", "s_mov_b32 s1, s2", cmp_))
    assert not find(asm(dot, ("s_branch 1", 3), cmp_, "s_endpgm"))
    copy = "global_load_lds_dwordx4 v4, s[0:1]"
    assert early_copies_behind_m0(asm("s_mov_b32 m0, s3", copy)) and early_copies_behind_m0(asm("s_movk_i32 m0, 0x10", copy))
    assert not early_copies_behind_m0(asm("s_mov_b32 m0, s3", "s_nop 0", copy, copy))


def test_sums_of_dot_products_are_there_when_they_are_read():
    bad = {k: early_readers_of_dot_sums(code) for k, code in kernels().items()}
    assert sum(x.op.startswith("v_dot") for code in kernels().values() for x in code) > 100
    assert not {k: v[:3] for k, v in bad.items() if v}


def test_copies_to_lds_do_not_follow_the_write_of_their_place_at_once():
    bad = {k: early_copies_behind_m0(code) for k, code in kernels().items()}
    assert sum("load_lds" in x.op for code in kernels().values() for x in code) > 100
    assert not {k: v[:3] for k, v in bad.items() if v}
