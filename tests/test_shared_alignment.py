"""Shared memory that kernels move in pieces wider than its elements is declared with the alignment of the pieces.  Without that it is where the compiler puts
it, and a new array beside it may turn the accesses into misaligned ones: the declarations are checked, since a test on a GPU sees only today's places."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1806_04090_b200", "csrc")
SIZE = {"uint8_t": 1, "char": 1, "uint16_t": 2, "float": 4, "int": 4, "uint32_t": 4, "int32_t": 4, "double": 8, "uint64_t": 8, "int64_t": 8, "float2": 8, "uint2": 8, "int2": 8,
        "float4": 16, "uint4": 16, "int4": 16, "double2": 16, "ulonglong2": 16}


def _declared(src, name, before):
    """Alignment of the shared array `name` by the declaration that stands last before a place; None where the name is no shared array (there)."""
    found, at = None, -1
    for m in re.finditer(r"__shared__\s+(?:(?:__align__|alignas)\((\d+)\)\s+)?(?:unsigned\s+)?(\w+)\s+([^;]*);", src):
        names = re.findall(r"(\w+)\s*(?:\[[^\]]*\])+", m.group(3))
        if name in names and m.start() < before:
            found, at = int(m.group(1)) if m.group(1) else SIZE.get(m.group(2)), m.start()
    pointers = [m.start() for m in re.finditer(r"\*\s*%s\s*=" % name, src) if m.start() < before]      # a pointer of that name in a later kernel
    return None if pointers and pointers[-1] > at else found


def test_shared_arrays_are_as_aligned_as_their_accesses():
    seen, bad = 0, []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        with open(path) as f:
            src = re.sub(r"//[^\n]*", "", f.read())
        for m in re.finditer(r"reinterpret_cast<(?:const )?(\w+)\s*\*(?: const)?>\(&?(\w+)", src):
            have, need = _declared(src, m.group(2), m.start()), SIZE.get(m.group(1))
            if have is None or need is None:
                continue
            seen += 1
            if have < need:
                bad.append((os.path.basename(path), m.group(2), have, need))
    assert seen > 5 and not bad, bad
