"""Wait states in the built library's gfx950 code, from its disassembly: needs
no GPU, but the toolchain's llvm-objdump.

The compiler keeps them between its own instructions and does not look inside
inline asm, from which the kernels issue their copies from memory to LDS.  On
gfx950

* a vector memory operation that writes LDS reads m0: one wait state after a
  scalar instruction wrote m0;
* a vector memory operation that reads a scalar register: five wait states after
  a vector instruction (v_readlane, v_readfirstlane) wrote it.

An instruction in between is one wait state, s_nop n is n + 1.
"""
import collections
import os
import re
import subprocess

import pytest

from paper_2503_12450_amd import binding as B
from paper_2503_12450_amd import build
from test_code_objects import _code_objects

LINE = re.compile(r"^\s+(\S+)\s*(.*?)\s+// ([0-9A-F]+):")
SCALARS = re.compile(r"s\[(\d+):(\d+)\]|\bs(\d+)\b")
VECTOR_MEMORY = ("buffer_", "global_", "flat_", "scratch_")

Ins = collections.namedtuple("Ins", "op args")


def _objdump():
    return os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc()))), "llvm", "bin",
                        "llvm-objdump")


def _functions(text):
    """(name, [(address, Ins)]) of a disassembly."""
    name, body = None, []
    for line in text.splitlines():
        head = re.match(r"^[0-9a-f]+ <(.+)>:$", line)
        at = LINE.match(line)
        if head:
            if name:
                yield name, body
            name, body = head[1], []
        elif at and name:
            body.append((int(at[3], 16), Ins(at[1], at[2])))
    if name:
        yield name, body


def _scalars(args):
    found = set()
    for lo, hi, one in SCALARS.findall(args):
        found.update(range(int(lo), int(hi) + 1) if lo else [int(one)])
    return found


def _predecessors(body):
    index = {address: i for i, (address, _) in enumerate(body)}
    before = [[] for _ in body]
    for i, (address, ins) in enumerate(body):
        if ins.op == "s_branch" or ins.op.startswith("s_cbranch"):
            offset = int(ins.args.split()[-1])
            target = index.get(address + 4 + 4 * (offset - 65536 if offset > 32767 else offset))
            if target is not None:
                before[target].append(i)
        if ins.op not in ("s_branch", "s_endpgm") and i + 1 < len(body):
            before[i + 1].append(i)
    return before


def _too_close(body, before, i, need, writes):
    """An instruction that `writes` within fewer than `need` wait states before
    instruction i, on any way to it."""
    todo, seen = [(p, 0) for p in before[i]], set()
    while todo:
        j, waited = todo.pop()
        if waited >= need or (j, waited) in seen:
            continue
        seen.add((j, waited))
        ins = body[j][1]
        if writes(ins):
            return ins
        waited += int(ins.args, 0) + 1 if ins.op == "s_nop" else 1
        todo += [(p, waited) for p in before[j]]
    return None


def _hazards(body):
    """(copies into LDS, hazards) of a function."""
    before, copies, found = _predecessors(body), 0, []
    for i, (address, ins) in enumerate(body):
        if not ins.op.startswith(VECTOR_MEMORY):
            continue
        if "_lds_" in ins.op or ins.args.endswith(" lds"):
            copies += 1
            w = _too_close(body, before, i, 1, lambda x: x.op.startswith("s_") and x.args.startswith("m0"))
            if w:
                found.append((hex(address), w, ins))
        used = _scalars(ins.args)
        if used:
            w = _too_close(body, before, i, 5,
                           lambda x: x.op.startswith("v_") and bool(_scalars(x.args.split(",")[0]) & used))
            if w:
                found.append((hex(address), w, ins))
    return copies, found


@pytest.fixture(scope="module")
def hazards(tmp_path_factory):
    """{kernel: (copies into LDS, hazards)} of the library."""
    with open(B.LIB_PATH, "rb") as f:
        images = list(_code_objects(f.read()))
    out = {}
    for i, elf in enumerate(images):
        path = tmp_path_factory.mktemp("elf") / f"{i}.elf"
        path.write_bytes(elf)
        text = subprocess.run([_objdump(), "-d", "--mcpu=gfx950", str(path)], check=True, capture_output=True,
                              text=True).stdout
        for name, body in _functions(text):
            out[name] = _hazards(body)
    return out


def test_the_search_finds_what_it_looks_for():
    """Hazards written down by hand: straight, over a branch, and ended by
    s_nop."""
    def run(*lines):
        return _hazards([(4 * i, Ins(*line)) for i, line in enumerate(lines)])

    m0, load = ("s_mov_b32", "m0, s4"), ("global_load_lds_dwordx4", "v0, s[2:3]")
    assert run(m0, load)[0] == 1 and len(run(m0, load)[1]) == 1
    assert not run(m0, ("s_nop", "0"), load)[1]
    lane = ("v_readlane_b32", "s3, v9, 2")
    assert len(run(lane, ("s_nop", "3"), load)[1]) == 1 and not run(lane, ("s_nop", "4"), load)[1]
    assert not run(("v_readlane_b32", "s4, v9, 2"), load)[1]
    # the branch at 4 jumps over the s_nop at 8 to the load at 12
    over = run(lane, ("s_cbranch_scc0", "1"), ("s_nop", "4"), load)
    assert len(over[1]) == 1
    assert len(run(("s_branch", "0"), lane, ("s_cbranch_scc0", "65533"), load)[1]) == 1


def _check(hazards, pattern):
    mine = {name: h for name, h in hazards.items() if re.search(pattern, name) and h[0]}
    assert mine
    assert {name: h[1][:2] for name, h in mine.items() if h[1]} == {}


def test_copies_of_the_paged_attention(hazards):
    _check(hazards, "attn_many")


def test_copies_of_every_kernel(hazards):
    """The products' operand tiles among them."""
    assert sum("gemm" in name for name, (copies, _) in hazards.items() if copies) > 100
    _check(hazards, "")
