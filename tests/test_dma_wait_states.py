"""Wait states around the loads into LDS that the kernels write as inline assembly (CPU only: the built code is listed,
nothing runs).

gfx9 does not hold such a load back until the scalars that it reads are written: M0 needs one wait state after a scalar
write, any scalar register five after a vector instruction's.  The compiler keeps these distances for its own instructions
and does not look into inline assembly."""
import os
import re
import struct
import subprocess
from collections import defaultdict

import pytest

from paper_2606_06302_amd import build

OBJDUMP = os.path.join(build.ROCM, "llvm", "bin", "llvm-objdump")
BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(library):
    """The GPU code of every source file: a bundle's header is its number of entries, then offset, size and name of each."""
    at = library.find(BUNDLE)
    while at >= 0:
        count, = struct.unpack_from("<Q", library, at + len(BUNDLE))
        entry = at + len(BUNDLE) + 8
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", library, entry)
            if library[entry + 24:entry + 24 + n].startswith(b"hip") and size:
                yield library[at + offset:at + offset + size]
            entry += 24 + n
        at = library.find(BUNDLE, at + 1)


def functions(listing):
    """name -> [(address, instruction, address that it branches to or None)]"""
    out, name = {}, None
    for line in listing.splitlines():
        head = re.match(r"([0-9a-f]+) <(.+)>:$", line)
        if head:
            base, name = int(head[1], 16), head[2]
            out[name] = []
            continue
        ins = re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+):(.*)", line)
        if ins and name:
            to = re.search(r"<[^+>]+(?:\+0x([0-9a-f]+))?>", ins[3])
            out[name].append((int(ins[2], 16), ins[1], base + int(to[1] or "0", 16) if to else None))
    return out


def scalars(operands):
    regs = {int(x) for x in re.findall(r"\bs(\d+)\b", operands)}
    for lo, hi in re.findall(r"\bs\[(\d+):(\d+)\]", operands):
        regs |= set(range(int(lo), int(hi) + 1))
    return regs


def early_reads(code):
    """(loads into LDS, those of them that come too early after a write, as text) of one function."""
    index = {a: i for i, (a, _, _) in enumerate(code)}
    before = defaultdict(list)
    for i, (_, text, to) in enumerate(code):
        if text.startswith(("s_branch", "s_cbranch")) and to in index:
            before[index[to]].append(i)
        if i + 1 < len(code) and not text.startswith(("s_branch", "s_endpgm")):
            before[i + 1].append(i)
    loads, bad = 0, []
    for i, (_, load, _) in enumerate(code):
        if not (load.startswith("global_load_lds") or (load.startswith("buffer_load") and load.endswith(" lds"))):
            continue
        loads += 1
        reads = scalars(load.partition(" ")[2])
        todo, seen = [(i, 0)], set()
        while todo:
            at, states = todo.pop()
            for p in before[at]:
                op, _, rest = code[p][1].partition(" ")
                written = rest.partition(",")[0].strip()
                if states < 1 and op.startswith("s_") and written == "m0":
                    bad.append(f"{code[p][1]}; {load}")
                if op.startswith("v_") and (scalars(written) & reads or written == "m0"):
                    bad.append(f"{code[p][1]}; {load}")
                far = states + (1 + int(rest, 0) if op == "s_nop" else 1)
                if far < 5 and (p, far) not in seen:
                    seen.add((p, far))
                    todo.append((p, far))
    return loads, bad


def listings():
    if not os.path.exists(OBJDUMP) or not os.path.exists(build.LIB):
        pytest.skip("needs the built library and llvm-objdump")
    with open(build.LIB, "rb") as f:
        library = f.read()
    for code in code_objects(library):
        yield subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "-"], input=code, capture_output=True,
                             check=True).stdout.decode()


def test_the_scan_sees_early_reads():
    """The scan itself, on code made for it."""
    make = lambda *ins: [(4 * i, x, None) for i, x in enumerate(ins)]
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    assert early_reads(make("s_mov_b32 m0, s1", load)) == (1, [f"s_mov_b32 m0, s1; {load}"])
    assert early_reads(make("s_mov_b32 m0, s1", "s_nop 0", load)) == (1, [])
    assert len(early_reads(make("v_readlane_b32 s5, v2, 3", "s_nop 3", load))[1]) == 1
    assert early_reads(make("v_readlane_b32 s5, v2, 3", "s_nop 4", load)) == (1, [])
    assert early_reads(make("v_readlane_b32 s6, v2, 3", load)) == (1, [])
    # along a branch
    code = [(0, "s_add_i32 m0, s1, s2", None), (4, "v_readfirstlane_b32 s4, v1", None), (8, "s_branch 1", 16),
            (12, "s_endpgm", None), (16, load, None)]
    assert early_reads(code) == (1, [f"v_readfirstlane_b32 s4, v1; {load}"])


def test_scalars_are_written_before_the_loads_that_read_them():
    loads = 0
    for listing in listings():
        for name, code in functions(listing).items():
            n, bad = early_reads(code)
            loads += n
            assert not bad, f"{name}: {len(bad)} of {n} loads, first: {bad[0]}"
    assert loads > 0
