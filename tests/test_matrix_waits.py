"""Results of matrix instructions are read late enough, on every way through the delta rule's kernels: in the built library's own machine code (no GPU needed).

The hardware does not hold back an instruction that reads, or writes over, the registers that a matrix instruction has not written yet: so many instructions, or idle steps of s_nop, have
to lie between.  The compiler counts them within straight code, but has left some out where branches lay between.  Here every way is counted, branches as one."""
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_1803_09926_amd as dw
from paper_1803_09926_amd import build

OBJDUMP = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin", "llvm-objdump")
# what the compiler keeps in straight code
STEPS = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x4_f32": 10}


def code_objects(path):
    """The GPU's ELF files in a library: each compilation's bundle begins with a magic, the number of entries, and each one's place, size and name."""
    blob, magic = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__"
    at = blob.find(magic)
    while at >= 0:
        p = at + len(magic)
        (n,) = struct.unpack_from("<Q", blob, p)
        p += 8
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", blob, p)
            name = blob[p + 24:p + 24 + length].decode()
            p += 24 + length
            if "gfx950" in name and size:
                yield blob[at + offset:at + offset + size]
        at = blob.find(magic, at + 1)


def registers(text):
    out = set()
    for kind, lo, hi, one, n in re.findall(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        out |= {(kind, k) for k in range(int(lo), int(hi) + 1)} if kind else {(one, int(n))}
    return out


def kernels(listing):
    """(name, instructions) of a disassembly; an instruction: its address, operation, operands, and where it branches to"""
    for part in re.split(r"\n(?=[0-9a-f]{16} <)", listing)[1:]:
        name, code = re.match(r"[0-9a-f]+ <([^>]+)>", part).group(1), []
        start = int(part[:16], 16)
        for line in part.split("\n")[1:]:
            m = re.match(r"\s+(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)$", line)
            if not m:
                continue
            op, operands, address, rest = m.groups()
            to = re.search(r"<[^>+]+(?:\+0x([0-9a-f]+))?>\s*$", rest)
            code.append((int(address, 16), op, operands, start + int(to.group(1) or "0", 16) if to and op.startswith(("s_cbranch", "s_branch")) else None))
        yield name, code


def steps_to_readers(code):
    """(operation, steps, whether over a branch, the reader's text) of each instruction that touches a matrix instruction's registers soon behind it"""
    index = {address: i for i, (address, _, _, _) in enumerate(code)}
    regs = [registers(operands) for _, _, operands, _ in code]
    first = [registers(operands.split(",")[0]) for _, _, operands, _ in code]
    for k, (_, op, operands, _) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        seen, todo = {}, [(k + 1, 0, False, frozenset(first[k]))]
        while todo:
            i, steps, over, live = todo.pop()
            if i >= len(code) or steps >= 12 or not live or seen.get((i, over, live), 99) <= steps:
                continue
            seen[i, over, live] = steps
            _, what, text, to = code[i]
            if what == "s_endpgm":
                continue
            if what.startswith("v_mfma"):
                # (what it adds to comes the same way out of the unit as it goes in, and needs no steps; its factors do)
                parts = re.findall(r"[va]\[\d+:\d+\]|[va]\d+", text)
                if (registers(parts[1]) | registers(parts[2])) & live:
                    yield op, steps, over, what + " " + text
                todo.append((i + 1, steps + 1, over, live - first[i]))
                continue
            if regs[i] & live and not what.startswith("s_"):
                yield op, steps, over, what + " " + text
                continue
            if to is not None:
                todo.append((index[to], steps + 1, True, live))
                if what == "s_branch":
                    continue
            todo.append((i + 1, steps + (int(text, 0) + 1 if what == "s_nop" else 1), over or to is not None, live))


@pytest.mark.skipif(not shutil.which(OBJDUMP), reason="no disassembler beside the compiler")
def test_results_of_matrix_instructions_are_waited_for(tmp_path):
    if not os.path.exists(build.LIB):
        dw.load()
    found, least, early = set(), {}, []
    for i, elf in enumerate(code_objects(build.LIB)):
        if b"k_gdelta" not in elf:
            continue
        path = tmp_path / ("%d.elf" % i)
        path.write_bytes(elf)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
        for name, code in kernels(listing):
            if "k_gdelta" not in name:
                continue
            found.add(name)
            for op, steps, over, reader in steps_to_readers(code):
                least[op, over] = min(least.get((op, over), 99), steps)
                if steps < STEPS[op]:
                    early.append("%s: %d steps of %d behind %s%s: %s" % (name, steps, STEPS[op], op, ", over a branch" if over else "", reader))
    print(len(found), "kernels;", sorted(least.items()))
    assert len(found) > 50 and {op for op, _ in least} == set(STEPS)
    assert not early, "\n".join(early)


def test_the_count_sees_a_short_way_over_a_branch():
    """One way round a branch is short, the other long enough; and a factor of the next matrix instruction counts, what it adds to does not."""
    def of(*lines):
        listing = "\n0000000000001000 <k>:\n" + "\n".join("\t%s // %012X: 00%s" % (l, 0x1000 + 4 * i, " <k+0x%x>" % (4 * to) if to is not None else "")
                                                          for i, (l, to) in enumerate(lines))
        (_, code), = kernels(listing)
        return sorted((steps, over) for _, steps, over, _ in steps_to_readers(code))

    mfma, use = ("v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]", None), ("v_add_f32_e32 v20, v2, v21", None)
    nop = ("s_nop 5", None)
    assert of(mfma, ("s_nop 7", None), use) == [(8, False)]
    assert of(mfma, ("s_cbranch_scc1 2", 3), nop, use) == [(1, True), (7, True)]
    assert of(mfma, mfma, ("s_nop 7", None), use) == [(8, False)]
    assert of(mfma, ("v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], 0", None), ("s_endpgm", None)) == [(0, False)]
