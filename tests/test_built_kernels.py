"""What the compiler made of the kernels: read from the descriptors in the built library (host only)."""
import os
import re
import shutil
import struct
import subprocess

import pytest

LIB = os.path.join(os.path.dirname(__file__), "..", "paper_2607_05116_amd", "libcap.so")


def _sections(elf):
    """(name, type, address, offset, size, link) of an ELF file's sections."""
    table = struct.unpack_from("<Q", elf, 0x28)[0]
    each, n, names = struct.unpack_from("<HHH", elf, 0x3A)
    rows = [struct.unpack_from("<IIQQQQI", elf, table + i * each) for i in range(n)]
    at = rows[names][4]
    text = lambda o: elf[at + o:elf.index(b"\0", at + o)].decode()
    return [(text(r[0]), r[1], r[3], r[4], r[5], r[6]) for r in rows]


def code_objects(path=LIB):
    """The gfx950 code objects of a library: entries of the bundles in its .hip_fatbin section."""
    elf = open(path, "rb").read()
    (at, size), = [(s[3], s[4]) for s in _sections(elf) if s[0] == ".hip_fatbin"]
    fat, start, found = elf[at:at + size], 0, []
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    while (start := fat.find(magic, start)) >= 0:
        p = start + len(magic) + 8
        for _ in range(struct.unpack_from("<Q", fat, p - 8)[0]):
            offset, length, n = struct.unpack_from("<QQQ", fat, p)
            if "gfx950" in fat[p + 24:p + 24 + n].decode() and length:
                found.append(fat[start + offset:start + offset + length])
            p += 24 + n
        start += len(magic)
    return found


def descriptors(obj):
    """Per kernel: bytes of LDS and of private memory, and whether it asks for the dispatch packet's address."""
    sections, out = _sections(obj), {}
    for _, kind, _, at, size, link in sections:
        if kind != 11:                                  # the dynamic symbols
            continue
        names = sections[link][3]
        for p in range(at, at + size, 24):
            name, _, _, index, value, _ = struct.unpack_from("<IBBHQQ", obj, p)
            symbol = obj[names + name:obj.index(b"\0", names + name)].decode()
            if not symbol.endswith(".kd"):
                continue
            d = sections[index][3] + value - sections[index][2]
            lds, private = struct.unpack_from("<II", obj, d)
            out[symbol[:-3]] = dict(lds=lds, private=private, dispatch=bool(struct.unpack_from("<H", obj, d + 56)[0] & 2))
    return out


@pytest.fixture(scope="module")
def kernels():
    found = {}
    for obj in code_objects():
        found.update(descriptors(obj))
    return found


def test_routing_by_scores_has_no_private_memory(kernels):
    """A private array that is indexed at run time lies in scratch, or in LDS at a place worked out from the dispatch
    packet, which every wave then reads from host memory."""
    mine = {n: d for n, d in kernels.items() if "route_scores_kernel" in n}
    assert len(mine) > 100
    assert [n for n, d in mine.items() if d["private"] or d["dispatch"]] == []


def test_no_kernel_shifts_64_bits_by_a_vector_register(tmp_path):
    """Such a shift whose amount is the last register of the kernel's now and then gives wrong results in whole waves, and
    which register it is, is the compiler's choice (cap_device.hpp has the forms that are used instead)."""
    objdump = shutil.which("llvm-objdump") or os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
    objects, found, seen = code_objects(), [], 0
    assert len(objects) > 10
    for i, obj in enumerate(objects):
        path = tmp_path / f"{i}.o"
        path.write_bytes(obj)
        text = subprocess.run([objdump, "-d", "--no-show-raw-insn", "--mcpu=gfx950", path], capture_output=True, text=True, check=True).stdout
        name = ""
        for line in text.splitlines():
            if line.endswith(">:"):
                name = line
            elif "_b64" in line or "_i64" in line:
                seen += 1
                if re.search(r"\bv_(lshlrev|lshrrev|ashrrev)_[bi]64\w* v\[\d+:\d+\], v\d+,", line):
                    found.append((name, line.strip()))
    assert seen > 1000                                  # the pattern has lines to look at
    assert found == []
