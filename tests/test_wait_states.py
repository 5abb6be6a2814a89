"""Loads from memory straight into LDS are written as assembler text, into which the compiler's hazard checks do not see (no GPU).

What the instruction set leaves to software there: one wait state between a scalar write of M0 and a load to LDS, which reads M0, and five between a
vector instruction's write of a scalar register and a memory instruction that reads it.  (Scalar instructions wait for vector ones by themselves, so where
one has written the register in between, the memory instruction reads that.)  Looked for in the machine code of the built library, along every path that
leads to such a load.
"""
import os
import re
import shutil
import struct
import subprocess

import pytest

OBJDUMP = shutil.which("llvm-objdump", path=os.pathsep.join(["/opt/rocm/llvm/bin", os.environ.get("PATH", "")]))
M0_STATES, SGPR_STATES = 1, 5


def _code_objects(data):
    """The gfx950 code objects of an offload bundle's file."""
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + length]:
                yield data[at + off:at + off + size]
            p += 24 + length
        at = data.find(magic, at + 1)


def _registers(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    return {int(m[1])} if m else set()


def _parse(listing):
    """Functions as lists of (address, mnemonic, operands, branch target's offset or None)."""
    functions, body = [], None
    for line in listing.splitlines():
        if re.fullmatch(r"[0-9a-f]+ <.*>:", line):
            body = []
            functions.append((int(line.split()[0], 16), body))
            continue
        m = re.match(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)$", line)
        if m and body is not None:
            target = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$", m[4]) if m[1].startswith(("s_branch", "s_cbranch")) else None
            body.append((int(m[3], 16), m[1], [x.strip() for x in m[2].split(",")], int(target[1] or "0", 16) if target else None))
    return functions


def _scalar_writes_of_vector(name, ops):
    name = re.sub(r"_e(32|64)$", "", name)
    if name.startswith(("v_readfirstlane", "v_readlane", "v_cmp_")):
        return _registers(ops[0])
    if re.match(r"v_(mad_[ui]64_[ui]32|\w+_co_|div_scale)", name):
        return _registers(ops[1])
    return set()


def _scalar_writes(name, ops):
    if not name.startswith("s_") or name.startswith(("s_cmp", "s_bitcmp", "s_nop", "s_wait", "s_branch", "s_cbranch", "s_load", "s_set")):
        return set()
    return _registers(ops[0])


def hazards(functions):
    """(loads looked at, [(address, what)])."""
    loads, found = 0, []
    for base, body in functions:
        place = {address: i for i, (address, *_) in enumerate(body)}
        before = [[i - 1] if i and body[i - 1][1] not in ("s_branch", "s_endpgm", "s_setpc_b64") else [] for i in range(len(body))]
        for i, (_, _, _, target) in enumerate(body):
            if target is not None:
                before[place[base + target]].append(i)
        for i, (address, name, ops, _) in enumerate(body):
            if not (name.startswith("global_load_lds") or (name.startswith("buffer_load") and any(o.split()[-1] == "lds" for o in ops if o))):
                continue
            loads += 1
            read = set().union(*(_registers(o.split()[0]) for o in ops if o))
            what, seen, todo = set(), set(), [(j, 0, frozenset(read)) for j in before[i]]
            while todo:
                at = j, states, waits_for = todo.pop()
                if states >= SGPR_STATES or at in seen:
                    continue
                seen.add(at)
                _, n, o, _ = body[j]
                if n.startswith("s_") and o[0] == "m0" and states < M0_STATES:
                    what.add("M0")
                if _scalar_writes_of_vector(n, o) & waits_for:
                    what.add("address")
                states += int(o[0], 0) + 1 if n == "s_nop" else 1
                todo += [(k, states, waits_for - _scalar_writes(n, o)) for k in before[j]]
            found += [(address, w) for w in sorted(what)]
    return loads, found


def test_the_search_finds_what_it_looks_for():
    """Itself first: on listings with the hazards planted."""
    def listing(*lines):
        return "0000000000001000 <f>:\n" + "\n".join(f"\t{text}    // {0x1000 + 4 * i:012X}: 00000000 {note}" for i, (text, note) in enumerate(lines))

    load = ("global_load_lds_dwordx4 v1, s[2:3]", "")
    nop, m0 = ("s_nop 0", ""), ("s_mov_b32 m0, s4", "")
    assert hazards(_parse(listing(m0, load)))[1] == [(0x1004, "M0")]
    assert hazards(_parse(listing(m0, nop, load))) == (1, [])
    assert hazards(_parse(listing(("v_readfirstlane_b32 s2, v0", ""), m0, nop, load)))[1] == [(0x100C, "address")]
    assert hazards(_parse(listing(("v_readfirstlane_b32 s4, v0", ""), m0, nop, load)))[1] == []
    assert hazards(_parse(listing(("v_readfirstlane_b32 s2, v0", ""), ("s_nop 2", ""), m0, nop, load)))[1] == []
    assert hazards(_parse(listing(("v_readlane_b32 s3, v0, 5", ""), ("s_addc_u32 s3, s9, s3", ""), m0, nop, load)))[1] == []
    assert hazards(_parse(listing(("v_readlane_b32 s3, v0, 5", ""), ("s_add_u32 s2, s9, s2", ""), m0, nop, load)))[1] == [(0x1010, "address")]
    assert hazards(_parse(listing(("v_mad_u64_u32 v[4:5], s[2:3], v0, s9, v[2:3]", ""), load)))[1] == [(0x1004, "address")]
    # along a branch: the load follows the label, the write comes before the jump
    around = listing(m0, ("s_cbranch_scc1 2", "<f+0x10>"), ("v_mov_b32 v0, v1", ""), ("v_cmp_lt_i32_e64 s[2:3], v0, v1", ""), load)
    assert hazards(_parse(around))[1] == [(0x1010, "address")]
    assert hazards(_parse(listing(m0, ("s_branch 1", "<f+0xc>"), nop, load)))[1] == []       # the jump itself is a wait state


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_loads_to_lds_wait_for_their_registers(tmp_path):
    import paper_1806_11248_amd as g
    if not os.path.exists(g.LIB_PATH):
        from paper_1806_11248_amd import build
        build.build()
    total = 0
    with open(g.LIB_PATH, "rb") as f:
        objects = list(_code_objects(f.read()))
    assert objects
    for n, code in enumerate(objects):
        path = tmp_path / f"{n}.co"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True, check=True).stdout
        if "_lds_" not in listing and " lds" not in listing:
            continue
        loads, found = hazards(_parse(listing))
        total += loads
        assert not found, f"{len(found)} of {loads} loads: {[(hex(a), what) for a, what in found[:8]]}"
    assert total > 0
