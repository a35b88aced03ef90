"""Wait states before the direct-to-LDS loads, in the machine code of the built library.

These loads are written as inline assembly, into which the compiler puts no wait states of its own.  On gfx950 one
instruction or s_nop has to stand between a scalar write of M0 (the LDS address) and the load, and five between a
vector instruction that writes a scalar register and a load that takes its address from it."""
import os
import re
import shutil
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_00049_amd", "librealq.so")
OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


def code_objects(path):
    """The gfx950 code objects of a library's offload bundles."""
    data, at = open(path, "rb").read(), 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        p = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            off, size, name = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + name] and size:
                yield data[at + off:at + off + size]
            p += 24 + name
        at += 1


def registers(operand):
    """Numbers of the scalar registers an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if not m:
        return set()
    return {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def early_loads(listing):
    """(number of direct-to-LDS loads, those that come too early with the instructions before them)."""
    code = [m[1] for m in (re.match(r"\t(\w+.*?)\s*(?://.*)?$", x) for x in listing.split("\n")) if m]
    loads, early = 0, []
    for i, text in enumerate(code):
        if not re.match(r"(global|buffer)_load_lds|buffer_load\S*\s.*\blds\b", text):
            continue
        loads += 1
        base = set().union(*(registers(x) for x in re.split(r",\s*|\s+", text)[1:]))
        waits = 0
        for before in reversed(code[max(0, i - 6):i]):
            op, *args = re.split(r",\s*|\s+", before)
            if op.startswith("s_") and args[:1] == ["m0"] and waits < 1:
                early.append((before, text))
            # a vector instruction's scalar results: its first operand, or the carry behind it
            wrote = registers(args[0]) if args and op.startswith("v_") else set()
            if re.match(r"v_(mad_[ui]64|div_scale|\w+_co_)", op):
                wrote |= registers(args[1])
            if wrote & base and waits < 5:
                early.append((before, text))
            waits += int(args[0], 0) + 1 if op == "s_nop" else 1
    return loads, early


def test_the_search_itself():
    listing = "\n".join("\t" + x for x in (
        "s_mov_b32 m0, s4", "global_load_lds_dwordx4 v1, s[8:9]",               # early
        "s_mov_b32 m0, s4", "s_nop 0", "global_load_lds_dwordx4 v1, s[8:9]",
        "v_readfirstlane_b32 s9, v2", "s_mov_b32 m0, s4", "s_nop 0", "global_load_lds_dwordx4 v1, s[8:9]",  # early
        "v_readfirstlane_b32 s9, v2", "s_mov_b32 m0, s4", "s_nop 3", "global_load_lds_dwordx4 v1, s[8:9]"))
    loads, early = early_loads(listing)
    assert loads == 4 and [e[0] for e in early] == ["s_mov_b32 m0, s4", "v_readfirstlane_b32 s9, v2"]


@pytest.mark.skipif(not os.path.exists(LIB) or not os.path.exists(OBJDUMP), reason="library or llvm-objdump not there")
def test_direct_to_lds_loads_wait_for_their_addresses(tmp_path):
    loads, early = 0, []
    for code in code_objects(LIB):
        (tmp_path / "code.o").write_bytes(code)
        res = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(tmp_path / "code.o")], capture_output=True,
                             text=True, check=True)
        n, bad = early_loads(res.stdout)
        loads, early = loads + n, early + bad
    assert loads > 0
    assert not early, f"{len(early)} of {loads} loads come too early, the first ones: {early[:4]}"
