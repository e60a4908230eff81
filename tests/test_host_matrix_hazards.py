"""The matrix instructions that alcs_tile.h writes out are not known to the compiler as such, and neither are the
accumulation registers they use, so it keeps no distance between them and the instructions around.  What has to hold is
read off the built kernels: a register that a vector instruction wrote is a matrix instruction's operand two
states later at the earliest; an accumulator is read no earlier than behind the waits of matrix_done(); and nothing but
those instructions, the clearing and the reading of each accumulator once touches accumulation registers."""
import os
import re
import struct
import subprocess
import tempfile

import pytest

import paper_2109_00170_amd as alcs
from kernel_metadata import LLVM, MAGIC

pytestmark = pytest.mark.skipif(not (os.path.exists(os.path.join(LLVM, "llvm-objdump")) and os.path.exists(alcs.library_path())),
                                reason="needs the built library and llvm-objdump")


def code_objects():
    """The gfx950 code objects of libalcs.so, as bytes."""
    with tempfile.TemporaryDirectory() as d:
        section = os.path.join(d, "fatbin")
        subprocess.check_call(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", alcs.library_path(), section])
        with open(section, "rb") as f:
            data = f.read()
    at = data.find(MAGIC)
    while at >= 0:
        entry = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            target = data[entry + 24:entry + 24 + length].decode()
            entry += 24 + length
            if "gfx950" in target and size:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + len(MAGIC))


def registers(text):
    """{("v", 3), ...} that an operand text names."""
    out = set()
    for kind, one, a, b in re.findall(r"\b([va])(?:(\d+)|\[(\d+):(\d+)\])", text):
        lo, hi = (int(one), int(one)) if one else (int(a), int(b))
        out |= {(kind, r) for r in range(lo, hi + 1)}
    return out


def states(line):
    m = re.match(r"s_nop (\d+)", line)
    return int(m[1]) + 1 if m else 1


def check(name, lines):
    seen = 0
    for i, l in enumerate(lines):
        if not l.startswith("v_mfma"):
            continue
        seen += 1
        _, operands = l.split(None, 1)
        reads = registers(operands)
        apart, k = 0, i - 1
        while k >= 0 and apart < 2 and not lines[k].startswith("s_cbranch") and not lines[k].startswith("s_branch"):
            p = lines[k]
            if p.startswith("v_") and not p.startswith("v_mfma") and not p.startswith("v_cmp"):
                wrote = registers(p.split(None, 1)[1].split(",")[0])
                assert not wrote & reads, "%s: %r %d states before %r" % (name, p, apart, l)
            apart += states(p)
            k -= 1
    touch = [l for l in lines if not l.startswith("v_mfma") and any(k == "a" for k, _ in registers(l))]
    clears = [l for l in touch if re.match(r"v_accvgpr_write_b32 a\d+, 0$", l)]
    reads = [l for l in touch if re.match(r"v_accvgpr_read_b32 v\d+, a\d+$", l)]
    assert len(touch) == 512 and len(set(clears)) == 256 and len({l.split()[-1] for l in reads}) == 256, name
    last = max(i for i, l in enumerate(lines) if l.startswith("v_mfma"))
    nops = [i for i, l in enumerate(lines) if l == "s_nop 15"]
    read = min(i for i, l in enumerate(lines) if l in set(reads))
    assert sum(last < i < read for i in nops) >= 2, name
    return seen


def test_distances_in_the_large_tiles():
    kernels = 0
    with tempfile.TemporaryDirectory() as d:
        for n, data in enumerate(code_objects()):
            if b"k_big" not in data:
                continue
            path = os.path.join(d, "object%d" % n)
            with open(path, "wb") as f:
                f.write(data)
            table = subprocess.check_output([os.path.join(LLVM, "llvm-readelf"), "--symbols", "--wide", path], text=True)
            names = sorted({w[-1] for w in (l.split() for l in table.splitlines()) if len(w) > 7 and w[3] == "FUNC" and "k_big" in w[-1]})
            for name in names:
                text = subprocess.check_output([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", "--disassemble-symbols=" + name, path], text=True)
                lines = [m[1].strip() for m in re.finditer(r"^\s+([a-z]\S+.*?)(?:\s*//.*)?$", text, re.M)]
                lines = [l for l in lines if re.match(r"[sv]_|ds_|global_|buffer_|scratch_|flat_", l)]
                assert check(name, lines) == 192
                kernels += 1
    assert kernels == 9   # forward, dX and dW of two 16-bit types, the 4-bit product to three
