"""Wait states around the loads to LDS in the built library (CPU).

The tiles' loads from memory to LDS are written in inline asm, inside which the
compiler does not look for hazards.  Two rules of gfx9 concern them: one wait
state between a scalar instruction's write of m0 and a load to LDS (which reads
m0), and five between a vector instruction's write of a scalar register and a
load that reads it.  Both are checked here in the disassembly of libmadd.so."""
import os
import re
import struct
import subprocess

import pytest

from paper_2607_10611_amd import _build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_objects(lib):
    """The gfx950 code objects in a library's offload bundles."""
    data = open(lib, "rb").read()
    for at in (m.start() for m in re.finditer(MAGIC, data)):
        pos = at + len(MAGIC)
        (count,) = struct.unpack_from("<Q", data, pos)
        pos += 8
        for _ in range(count):
            offset, size, named = struct.unpack_from("<3Q", data, pos)
            name = data[pos + 24:pos + 24 + named]
            pos += 24 + named
            if name.endswith(b"gfx950"):
                yield data[at + offset:at + offset + size]


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if not m:
        return set()
    lo, hi = (m[1], m[2]) if m[1] else (m[3], m[3])
    return set(range(int(lo), int(hi) + 1))


def parsed(line):
    """(mnemonic, operands) of a line of the disassembly, or None."""
    m = re.match(r"\s+([a-z]\w+)(?:\s+(.*?))?\s*(?://.*)?$", line)
    if not m:
        return None
    ops = [o.strip().split()[0] for o in (m[2] or "").split(",") if o.strip()]
    return m[1], ops, m[2] or ""


def violations(instructions):
    """(index, why) of loads to LDS that come too soon."""
    bad = []
    for i, (name, ops, text) in enumerate(instructions):
        if not (name.startswith(("buffer_load", "global_load")) and re.search(r"\blds\b", text)
                or name.startswith("global_load_lds")):
            continue
        if i and instructions[i - 1][0].startswith("s_") and instructions[i - 1][1][:1] == ["m0"]:
            bad.append((i, "m0 written directly before"))
        reads = set().union(*(scalars(o) for o in ops))
        waited, j = 0, i - 1
        while j >= 0 and waited < 5:
            n, o, _ = instructions[j]
            if n.startswith("v_"):
                wide = "_co_" in n or "div_scale" in n or "mad_u64" in n or "mad_i64" in n
                written = set().union(*(scalars(x) for x in o[:2 if wide else 1]))
                if written & reads:
                    bad.append((i, f"{n} {o} writes a scalar register {waited} wait states before"))
            waited += int(o[0], 0) + 1 if n == "s_nop" else 1
            j -= 1
    return bad


def test_the_check_sees_violations():
    """The rules above, on made-up listings."""
    load = "\tbuffer_load_dwordx4 v1, s[12:15], s23 offen lds // 0000: E05D1000"
    listing = lambda *lines: [parsed(x) for x in (*lines, load)]  # noqa: E731
    assert violations(listing("\ts_mov_b32 m0, s54"))
    assert violations(listing("\ts_add_i32 m0, s54, 0x1000"))
    assert not violations(listing("\ts_mov_b32 m0, s54", "\ts_nop 0"))
    assert violations(listing("\tv_readlane_b32 s13, v9, 2", "\ts_nop 0"))
    assert violations(listing("\tv_readfirstlane_b32 s23, v9", "\ts_nop 3"))
    assert not violations(listing("\tv_readfirstlane_b32 s23, v9", "\ts_nop 4"))
    assert not violations(listing("\tv_readfirstlane_b32 s22, v9"))
    assert not violations(listing("\tv_add_u32_e32 v1, s13, v2"))


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")
def test_loads_to_lds_come_late_enough(tmp_path):
    if not os.path.exists(_build.LIB):
        _build.build()
    loads, bad = 0, []
    for k, obj in enumerate(device_objects(_build.LIB)):
        if b"matmul_tile_kernel" not in obj:
            continue
        path = tmp_path / f"{k}.o"
        path.write_bytes(obj)
        out = subprocess.run([OBJDUMP, "-d", str(path)], check=True, capture_output=True,
                             text=True).stdout
        code = [p for p in map(parsed, out.splitlines()) if p]
        loads += sum("lds" in t.split() for _, _, t in code)
        bad += violations(code)
    assert loads > 0
    assert not bad, (len(bad), bad[:5])
