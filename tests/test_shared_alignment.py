"""Arrays in shared memory that kernels read or write in wider pieces than their elements are declared with the
alignment that such an access needs: where the compiler places them does not give it."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_07565_gb300", "csrc")
SIZES = {"uint8_t": 1, "int8_t": 1, "uint16_t": 2, "uint32_t": 4, "float": 4, "int": 4, "uint64_t": 8, "double": 8,
         "uint2": 8, "float2": 8, "int2": 8, "uint4": 16, "float4": 16, "int4": 16, "QPiece": 8}
SHARED = re.compile(r"__shared__\s+(?:__align__\((\d+)\)\s+)?(?:static\s+)?(\w+)\s+([^;]+);")
CAST = re.compile(r"reinterpret_cast<(?:const\s+)?(?:volatile\s+)?(\w+)\s*\*>\(\s*&?(\w+)\b")


def too_wide(source):
    """(name, access, alignment) of accesses past an array's declared alignment."""
    arrays = {}
    for align, element, names in SHARED.findall(source):
        for name in re.findall(r"(\w+)(?:\[[^\]]*\])+", names):
            # (An array of a name that several kernels use: the least of their alignments.)
            arrays[name] = min(arrays.get(name, 1 << 10), max(int(align or 0), SIZES.get(element, 1 << 10)))
    return [(name, cast, arrays[name]) for cast, name in CAST.findall(source)
            if name in arrays and SIZES.get(cast, 0) > arrays[name]]


def test_finds_what_it_looks_for():
    text = "__shared__ uint32_t a[4][8];\n x = *reinterpret_cast<const uint4 *>(&a[0][4]);"
    assert too_wide(text) == [("a", "uint4", 4)]
    assert too_wide(text.replace("uint32_t a", "__align__(16) uint32_t a")) == []
    assert too_wide(text.replace("uint32_t a", "uint4 a")) == []


def test_wide_accesses_are_aligned_by_declaration():
    files = glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))
    assert files
    found = {os.path.basename(f): hits for f in files if (hits := too_wide(open(f).read()))}
    assert not found, found
