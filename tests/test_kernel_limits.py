"""Limits that belong to a kernel and not to a call, by reading the sources."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_11498_b200", "csrc")


def test_the_limit_of_shared_memory_is_one_constant_for_a_kernel():
    """It is the function's, for all host threads: a call that sets it to its own size can lower it between another call's setting and that
    call's launch.  allow_smem takes it as a template argument; the other place is a kernel that is never launched."""
    found = {}
    for path in glob.glob(os.path.join(CSRC, "*")):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        uses = re.findall(r"cudaFuncSetAttribute\(\s*(\w+),\s*cudaFuncAttributeMaxDynamicSharedMemorySize,\s*([^)]*)\)", text)
        assert len(uses) == text.count("MaxDynamicSharedMemorySize"), path
        if uses:
            found[os.path.basename(path)] = uses
    assert found == {"lrsa_internal.h": [("kern", "BYTES")], "lrsa_api.cu": [("room_kernel", "200 << 10")]}


def test_operand_tiles_that_are_not_aligned_are_told():
    """The swizzled tiles want 1024 bytes.  A kernel that finds its shared memory elsewhere does nothing, and says so by its status."""
    places = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"& 1023u", text):
            places += 1
            line = text[text.rfind("\n", 0, m.start()):text.find("\n", m.end())]
            block = text[m.end():text.find("}", m.end())] if line.rstrip().endswith("{") else line
            assert "abort" in block or "status" in block, (path, line)
    assert places >= 3
